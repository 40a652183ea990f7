"""Whole numbers of any size in the arguments of the norm of heads and of a cache in pages: what a field of the C interface does not hold
stays too large for it, and is taken or refused as such."""
import ctypes

import pytest
import torch

import paper_2409_09708_amd as nm
from paper_2409_09708_amd import binding

BF16 = torch.bfloat16
MOST = 2 ** 31 - 1


@pytest.mark.parametrize("value,held", [(0, 0), (5, 5), (-1, -1), (MOST, MOST), (MOST + 1, MOST), (2 ** 32 + 5, MOST), (10 ** 12, MOST), (2 ** 64, MOST),
                                        (-2 ** 31, -2 ** 31), (-2 ** 31 - 1, -2 ** 31), (-2 ** 32 + 5, -2 ** 31), (-2 ** 64 + 5, -2 ** 31)])
def test_fields_of_32_bits(value, held):
    d, p = binding.PagedDesc(), binding.Pages()
    d.window, d.sinks, d.heads_q, p.head_size, p.table_width = (value,) * 5
    assert [d.window, d.sinks, d.heads_q, p.head_size, p.table_width] == [held] * 5
    assert list(binding._ints([value, 3])) == [held, 3]


def test_fields_of_64_bits():
    d = binding.HeadNormDesc()
    d.heads, d.D = 2 ** 64 + 3, -2 ** 64 + 3
    assert d.heads == 2 ** 63 - 1 and d.D == -2 ** 63
    d.eps, d.weight, d.freqs = 0.5, None, 2 ** 63 + 16  # (no whole numbers, and an address)
    assert d.eps == 0.5 and d.weight is None and d.freqs == 2 ** 63 + 16
    with pytest.raises(TypeError):
        d.heads = 1.5


def test_refused_on_the_host():
    lib = binding.load_library()
    TH, at = binding.TypedHeads, 0x1000
    for heads, sections in ((2 ** 64 + 3, (16, 16)), (3, (2 ** 32 + 16, 16)), (3, (16, -2 ** 32 + 16))):
        d = binding.HeadNormDesc()
        d.X = d.Y = TH(at, 256, 64, 1, 0)
        d.positions = d.freqs = at
        kept = binding._ints(sections)
        d.sections = ctypes.addressof(kept)
        d.T, d.H, d.heads, d.D, d.rotated, d.axes, d.eps = 5000, 4, heads, 64, 64, 2, 1e-6
        assert lib.nm_head_norm(ctypes.byref(d), None) == 2  # (a shape)


@pytest.mark.gpu
@pytest.mark.parametrize("new", [1, 40])
def test_attention_over_pages(new):
    from pages_reference import Cache
    cache = Cache([90, 60], 96, 2, 64, 16, True).fill(1)
    g = torch.Generator("cuda").manual_seed(2)
    Q = torch.randn(2 * new, 4, 64, generator=g, device="cuda").to(BF16)

    def o(**how):
        return nm.nm_attention_paged(Q, *cache.args, **cache.scales, **how)

    every, some = o(), o(window=5)
    assert not torch.equal(every, some)
    for window in (2 ** 31 + 5, 2 ** 32 + 5, 10 ** 12, 2 ** 64 + 5):
        assert torch.equal(o(window=window), every), window
        assert torch.equal(o(window=5, sinks=window), every), window
    for wrong in (-1, -2 ** 31, -2 ** 32 + 5, -2 ** 64 + 5):
        with pytest.raises(nm.NmError):
            o(window=wrong)
        with pytest.raises(nm.NmError):
            o(window=5, sinks=wrong)
