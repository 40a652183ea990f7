"""Rotary positions with several axes against their definition in 64 bits."""
import pytest
import torch

import block_reference as ref

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def setup(seed, T, H, D, dtype, wide, at=0):
    g = torch.Generator("cuda")
    g.manual_seed(seed)
    X = torch.randn(T, H * D + wide + at, generator=g, device="cuda").to(dtype)[:, at:at + H * D].unflatten(1, (H, D))
    return g, X


@pytest.mark.parametrize("T,H,D,R,sections,wide,at", [
    (1, 1, 2, 2, (1,), 0, 0), (1, 12, 64, 64, (32,), 0, 0), (197, 24, 64, 64, (16, 16), 768, 0), (33, 3, 128, 96, (16, 20, 12), 0, 0),
    (5, 2, 80, 40, (10, 10), 8, 8), (7, 5, 33, 30, (5, 4, 3, 3), 1, 1), (300, 1, 128, 128, (64,), 3, 0), (9, 2, 96, 96, (0, 48), 0, 0),
    (2, 1, 2048, 2048, (600, 424), 0, 0), (3, 2, 1100, 1096, (548,), 4, 0), (70000, 1, 32, 32, (16,), 0, 0), (64, 2, 72, 72, (20, 16), 0, 0)])
@pytest.mark.parametrize("x_type,y_type", [(BF16, BF16), (F32, F32), (F32, BF16), (BF16, F32)])
def test_turn(T, H, D, R, sections, wide, at, x_type, y_type):
    import paper_2409_09708_amd as nm
    g, X = setup(T + D, T, H, D, x_type, wide, at)
    axes = len(sections)
    freqs = 10000.0 ** (-torch.arange(R // 2, device="cuda") / (R // 2))
    for positions in (torch.randint(0, 9000, (T, axes), generator=g, device="cuda", dtype=torch.int32),
                      torch.randn(T, axes, generator=g, device="cuda") * 50):
        for interleaved in (False, True):
            for inverse in (False, True):
                y = nm.nm_rotary(X, positions, freqs, sections, interleaved, inverse, out_dtype=y_type)
                want, bound = ref.rotary(X.double(), positions, freqs, sections, interleaved, inverse, y_type)
                assert y.dtype == y_type
                ref.close(y, want, bound, (interleaved, inverse))


def test_one_axis_and_the_way_back_in_place():
    import paper_2409_09708_amd as nm
    g, X = setup(3, 211, 6, 64, F32, 128)
    at = torch.arange(211, device="cuda", dtype=torch.int32)
    freqs = 10000.0 ** (-torch.arange(24, device="cuda") / 24)  # (the last 16 elements are not turned)
    want = nm.nm_rotary(X, at[:, None].contiguous(), freqs, (24,))
    assert torch.equal(nm.nm_rotary(X, at, freqs), want)
    assert torch.equal(want[..., 48:], X[..., 48:])
    kept = X.clone()
    out = nm.nm_rotary(X, at, freqs, out=X)
    assert out is X and torch.equal(X, want)
    back = nm.nm_rotary(X, at, freqs, inverse=True)
    size = kept.abs()
    pair = torch.cat([size[..., :24] + size[..., 24:48]] * 2 + [size[..., 48:]], -1)
    assert bool(((back - kept).abs() <= 24 * ref.U32 * pair.double()).all())


def test_backward_is_the_transposed_turn():
    """<dY, turn(X)> = <turn^-1(dY), X>."""
    import paper_2409_09708_amd as nm
    g, X = setup(4, 50, 3, 64, F32, 0)
    dY = torch.randn(50, 3, 64, generator=g, device="cuda")
    pos = torch.randint(0, 100, (50, 2), generator=g, device="cuda", dtype=torch.int32)
    freqs = torch.rand(32, generator=g, device="cuda")
    a = (dY.double() * nm.nm_rotary(X, pos, freqs, (16, 16)).double()).sum()
    b = (nm.nm_rotary(dY, pos, freqs, (16, 16), inverse=True).double() * X.double()).sum()
    assert abs(float(a - b)) <= 16 * ref.U32 * 2 * float((dY.double().abs().sum() + X.double().abs().sum())) * 5
