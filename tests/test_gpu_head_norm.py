"""Norm of heads with its rotary turn, and the backward pass, against the definition in 64 bits."""
import pytest
import torch

import block_reference as ref
import pages_reference as pages

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-6


def setup(seed, T, H, D, dtype, wide=0, at=0, scale=1.0, offset=0.0):
    g = torch.Generator("cuda").manual_seed(seed)
    X = torch.randn(T, H * D + wide + at, generator=g, device="cuda").mul_(scale).add_(offset).to(dtype)
    return g, X[:, at:at + H * D].unflatten(1, (H, D))


def turned(g, T, R, sections, interleaved, far=9000):
    if not R:
        return None, None, None, False
    freqs = 10000.0 ** (-torch.arange(R // 2, device="cuda") / (R // 2))
    return torch.randint(-far, far, (T, len(sections)), generator=g, device="cuda", dtype=torch.int32), freqs, sections, interleaved


def named(t):
    return dict(zip(("positions", "freqs", "sections", "interleaved"), t))


def weights(g, H, heads, D):
    shape = (2, D) if heads < H else (D,)
    return 1 + 0.3 * torch.randn(shape, generator=g, device="cuda")


def check(seed, T, H, heads, D, R, sections, x_type, y_type, wide=0, at=0, interleaved=False, centred=False, weight=True, backward=True, **how):
    import paper_2409_09708_amd as nm
    g, X = setup(seed, T, H, D, x_type, wide, at, **how)
    t = turned(g, T, R, sections, interleaved)
    w = weights(g, H, heads, D) if weight else None
    y = nm.nm_head_norm(X, w, heads, EPS, centred, out_dtype=y_type, **named(t))
    want, bound = pages.head_norm(X, w, heads, EPS, centred, t, y_type)
    assert y.dtype == y_type
    ref.close(y, want, bound, "y")
    if not backward:
        return
    dY = setup(seed + 1, T, H, D, y_type, at, wide)[1]
    dx, dw = nm.nm_head_norm_backward(dY, X, w, heads, EPS, centred, out_dtype=x_type, **named(t))
    (want, bound), params = pages.head_norm_grad(dY, X, w, heads, EPS, centred, t, x_type)
    ref.close(dx, want, bound, "dx")
    assert (dw is None) == (params is None)
    if params:
        assert dw.shape == w.shape
        ref.close(dw, *params, "dw")
        again = nm.nm_head_norm_backward(dY, X, w, heads, EPS, centred, out_dtype=x_type, **named(t))
        assert torch.equal(again[0], dx) and torch.equal(again[1], dw)
        assert nm.nm_head_norm_backward(dY, X, w, heads, EPS, centred, params=False, **named(t))[1] is None


SHAPES = [  # T, H, heads, D, R, sections, wide, at
    (1, 1, 1, 1, 0, (), 0, 0), (1, 2, 1, 2, 2, (1,), 0, 0), (1, 40, 32, 128, 128, (64,), 0, 0), (2, 3, 3, 7, 4, (2,), 1, 1),
    (197, 24, 12, 64, 64, (16, 16), 768, 0), (33, 3, 2, 128, 96, (16, 20, 12), 0, 0), (5, 2, 1, 80, 40, (10, 10), 8, 8),
    (7, 5, 4, 33, 30, (5, 4, 3, 3), 1, 1), (9, 2, 2, 96, 96, (0, 48), 0, 0), (3, 2, 1, 512, 512, (256,), 0, 0), (4, 3, 1, 500, 2, (1,), 3, 5),
    (5, 2, 1, 257, 0, (), 0, 0), (64, 2, 1, 72, 72, (20, 16), 0, 0), (2300, 3, 2, 16, 16, (8,), 0, 0), (1500, 6, 4, 64, 0, (), 64, 0),
    (11, 1, 1, 256, 130, (65,), 2, 0)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("x_type,y_type", [(BF16, BF16), (F32, F32), (F32, BF16), (BF16, F32)])
def test_values_and_gradients(shape, x_type, y_type):
    T, H, heads, D, R, sections, wide, at = shape
    for interleaved in (False, True) if R else (False,):
        for centred in (False, True):
            check(T + D, T, H, heads, D, R, sections, x_type, y_type, wide, at, interleaved, centred)


def test_many_tokens_in_few_blocks():
    check(1, 9000, 5, 3, 128, 128, (64,), BF16, BF16, wide=256)
    check(2, 3001, 10, 7, 80, 72, (12, 12, 12), F32, F32, interleaved=True, centred=True)


@pytest.mark.parametrize("centred", [False, True])
def test_without_weights_and_without_turn(centred):
    check(3, 50, 4, 4, 64, 64, (32,), BF16, BF16, centred=centred, weight=False)
    check(4, 50, 4, 2, 64, 0, (), F32, F32, centred=centred, weight=False)
    check(5, 50, 4, 4, 100, 0, (), F32, BF16, centred=centred)


def test_sizes_of_values():
    """Offsets far above the spread, heads of zeros, and magnitudes whose squares are near the ends of a float."""
    import paper_2409_09708_amd as nm
    check(6, 20, 3, 2, 64, 64, (32,), F32, F32, centred=True, offset=1000.0, backward=False)
    check(7, 20, 3, 2, 64, 64, (32,), BF16, F32, scale=1e15)
    check(8, 20, 3, 2, 64, 64, (32,), F32, F32, scale=1e-12, centred=True)
    X = torch.zeros(3, 2, 64, device="cuda")
    X[1, 1] = 5.0  # (constant: nothing is left of it once centred)
    y = nm.nm_head_norm(X, centred=True)
    assert torch.equal(y, torch.zeros_like(y))
    dx, _ = nm.nm_head_norm_backward(torch.ones_like(X), X, centred=True)
    assert torch.equal(dx, torch.zeros_like(dx))
    X[2, 0, 5] = float("nan")
    y = nm.nm_head_norm(X)
    assert bool(y[2, 0].isnan().all()) and not bool(y[:2].isnan().any()) and not bool(y[2, 1].isnan().any())


def test_far_positions():
    """Angles of many turns: a product in 32 bits would be off by 60 radians."""
    import paper_2409_09708_amd as nm
    g, X = setup(9, 40, 2, 64, F32)
    freqs = torch.rand(32, generator=g, device="cuda")
    for positions in (torch.randint(1 << 29, (1 << 30) - 1, (40,), generator=g, device="cuda", dtype=torch.int32),
                      torch.rand(40, generator=g, device="cuda") * 1e6):
        y = nm.nm_head_norm(X, positions=positions, freqs=freqs)
        want, bound = pages.head_norm(X, None, 2, EPS, False, (positions, freqs, (32,), False), F32)
        ref.close(y, want, bound)


def test_in_place_and_into_views():
    import paper_2409_09708_amd as nm
    g, X = setup(10, 211, 6, 64, BF16, wide=128)
    t = turned(g, 211, 48, (24,), False)
    w = weights(g, 6, 4, 64)
    whole = X.clone()
    want = nm.nm_head_norm(X, w, 4, **named(t))
    dY = setup(11, 211, 6, 64, BF16, wide=64)[1]
    dx, dw = nm.nm_head_norm_backward(dY, X, w, 4, **named(t))
    row = torch.full((211, 8 * 64), 7.0, dtype=BF16, device="cuda")
    view = row[:, :384].unflatten(1, (6, 64))
    out, dw2 = nm.nm_head_norm_backward(dY, X, w, 4, out=view, **named(t))
    assert out is view and torch.equal(view, dx) and torch.equal(dw2, dw) and bool((row[:, 384:] == 7).all())
    kept = dY.clone()
    out, _ = nm.nm_head_norm_backward(dY, X, w, 4, out=dY, **named(t))
    assert out is dY and torch.equal(dY, dx)
    x2 = whole.clone()
    out, _ = nm.nm_head_norm_backward(kept, x2, w, 4, out=x2, **named(t))
    assert torch.equal(x2, dx)
    assert nm.nm_head_norm(X, w, 4, out=X, **named(t)) is X and torch.equal(X, want)
    heads_first = whole.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(nm.nm_head_norm(heads_first, w, 4, **named(t)), want)
    one = whole[:, :1].expand(-1, 6, -1)  # (one head read six times)
    ref.close(nm.nm_head_norm(one, w, 4, **named(t)), *pages.head_norm(one, w, 4, 1e-6, False, t, BF16))


@pytest.mark.parametrize("centred", [False, True])
def test_gradient_against_differences(centred):
    """(f(x + h v) - f(x - h v)) / 2 h in 64 bits along directions, of the definition, which the kernels are held to above."""
    g, X = setup(12, 6, 3, 16, F32)
    t = turned(g, 6, 12, (6,), True)
    w = weights(g, 3, 2, 16)
    X, dY = X.double(), setup(13, 6, 3, 16, F32)[1].double()
    (dx, _), (dw, _) = pages.head_norm_grad(dY, X, w, 2, EPS, centred, t, F32)
    h = 1e-5

    def f(x, weight):
        return (pages.head_norm(x, weight, 2, EPS, centred, t, F32)[0] * dY).sum()

    for k in range(4):
        v = torch.randn(X.shape, generator=g, device="cuda").double()
        num = (f(X + h * v, w) - f(X - h * v, w)) / (2 * h)
        # (the third derivative's part is h^2 / 6 of sums of size 1e3 at most; rounding 1e3 2^-53 / h)
        assert abs(float(num - (dx * v).sum())) <= 1e-6 * (1 + abs(float(num)))
        u = torch.randn(w.shape, generator=g, device="cuda").double()
        num = (f(X, w.double() + h * u) - f(X, w.double() - h * u)) / (2 * h)
        assert abs(float(num - (dw * u).sum())) <= 1e-6 * (1 + abs(float(num)))


def test_captured_and_replayed():
    import paper_2409_09708_amd as nm
    g, X = setup(14, 3000, 6, 64, BF16)
    t = turned(g, 3000, 64, (32,), False)
    w, dY = weights(g, 6, 4, 64), setup(15, 3000, 6, 64, BF16)[1].clone()

    def step():
        return (nm.nm_head_norm(X, w, 4, **named(t)),) + nm.nm_head_norm_backward(dY, X, w, 4, **named(t))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for k in range(4):
        X.copy_(torch.randn(X.shape, generator=g, device="cuda"))
        dY.copy_(torch.randn(X.shape, generator=g, device="cuda"))
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want)), k
