"""The norm of heads and attention over pages at the ends of what their arguments may be."""
import pytest
import torch

import paper_2409_09708_amd as nm
from pages_reference import Cache
from test_gpu_paged import check

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("window", [2 ** 30, 2 ** 31 - 1])
@pytest.mark.parametrize("counts", [[6, 3], [40, 90], [200, 70]])
def test_widest_window_where_queries_stand_before_the_first_token(counts, window, codes):
    """(more new tokens than the sequence is said to have: the first of them have negative positions and see nothing)"""
    cache = Cache([4, 66], 300, 2, 64, 16, codes).fill(window % 97)
    o = check(cache, counts, 4, window=window, sinks=3, max_q=max(counts))
    assert torch.equal(o, check(cache, counts, 4, max_q=max(counts)))
    check(cache, counts, 4, sinks=2 ** 31 - 1, window=1, max_q=max(counts))


def test_norm_gradient_of_very_many_heads():
    H, T = 2 ** 17, 768 * 20
    g = torch.Generator("cuda").manual_seed(5)
    x, dy = (torch.randn(1, H, 1, generator=g, device="cuda").to(BF16) for _ in range(2))
    w = torch.full((1,), 1.5, device="cuda")
    one, _ = nm.nm_head_norm_backward(dy, x, w, eps=1.0, params=False)
    n = x.double() * (x.double().square() + 1).rsqrt()
    want = (x.double().square() + 1).rsqrt() * (dy.double() * 1.5) * (1 - n * n)
    # (the difference of 1 and n^2 = x^2 rstd^2 in 32 bits, then the rounding)
    assert ((one.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -20 * dy.double().abs()).all()
    every, _ = nm.nm_head_norm_backward(dy.expand(T, H, 1), x.expand(T, H, 1), w, eps=1.0, params=False)
    for t in range(0, T, 1024):
        assert torch.equal(every[t:t + 1024], one.expand_as(every[t:t + 1024])), t


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("L", [4, 7, 8, 9, 12, 15, 16, 17, 20])
def test_one_size_of_workspace_for_both_types(L, codes):
    """(sixteen to eighty pairs of query and head: where one kernel takes over from the other, which is by the pages' type)"""
    cache = Cache([3000, 40, L], 3000, 2, 64, 16, codes).fill(L)
    size = nm.binding.load_library().nm_attention_paged_workspace_bytes(3 * L, 3, 8, 2, 64, L)
    plain = check(cache, [L] * 3, 8, L)
    assert torch.equal(plain, check(cache, [L] * 3, 8, L, workspace=torch.empty(size, dtype=torch.uint8, device="cuda")))
    check(cache, [L, 1, 0], 8, L, max_q=L, window=300, sinks=5)


@pytest.mark.parametrize("codes", [False, True])
def test_units_left_whole_where_they_are_many(codes):
    lens = [(37 * i) % 700 for i in range(500)]
    cache = Cache(lens, 700, 1, 32, 16, codes).fill(6)
    counts = [min(n, 1 + i % 2) for i, n in enumerate(lens)]
    for max_k in (624, 626, 700):  # (both sides of five keys for four units, whatever the lengths are)
        check(cache, counts, 2, max_q=2, max_k=max_k)
