"""Attention over pages for few queries is as exact as the rounding of its output: probabilities enter as two bfloat16 each.  The bound leaves
no room for one."""
import pytest
import torch

import block_reference as ref
import paper_2409_09708_amd as nm
from block_reference import U16, U32
from pages_reference import Cache
from test_gpu_paged import offsets, queries


def sharp(Q, keys, counts, lens, scale, window=0, sinks=0):
    """(O, bound, O where probabilities are rounded to one bfloat16) in 64 bits; keys(b, at): keys and values of tokens `at` of sequence b.
    A probability's first half is off by U16 of it, the second half of that by U16 again."""
    Q = Q.double()
    O, bound, one = (torch.zeros_like(Q) for _ in range(3))
    q0 = 0
    for b, (L, n) in enumerate(zip(counts, lens)):
        rows = slice(q0, q0 + L)
        q0 += L
        at, p = torch.arange(n, device=Q.device), torch.arange(n - L, n, device=Q.device)[:, None]
        seen = (at <= p) & ((at > p - window) | (at < sinks)) if window else at <= p
        at = at[seen.any(0)]
        seen = seen[:, at]
        k_all, v_all = keys(b, at)
        group = Q.shape[1] // k_all.shape[1]
        for h in range(Q.shape[1]):
            k, v = k_all[:, h // group].contiguous(), v_all[:, h // group].contiguous()
            s, ds = ref._scores(Q[rows, h], k, scale, seen)
            e = torch.exp(s - s.amax(1, keepdim=True))
            pr = e / e.sum(1, keepdim=True)
            # (scores, their exponent, the sum that it is divided by, as in the bound for any number of queries)
            off = torch.where(seen, ds, 0.0).amax(1, keepdim=True) * 2 + (len(at) + 16) * U32 + 64 * U32
            o = pr @ v
            off = (U16 * U16 * (1 + 2 * off) + 2 * off + (len(at) + 8) * U32) * (pr @ v.abs())
            O[rows, h], bound[rows, h] = o, off + U16 * (o.abs() + off)
            one[rows, h] = (e.float().to(torch.bfloat16).double() @ v) / e.sum(1, keepdim=True)
    return O, bound, one


def test_bound_tells_one_bfloat16_from_two():
    g = torch.Generator().manual_seed(1)
    lens = [200, 333]
    Q, K, V = (torch.randn(n, h, 64, generator=g).to(torch.bfloat16) for n, h in ((2, 4), (533, 2), (533, 2)))
    start = [0, 200]
    O, bound, one = sharp(Q, lambda b, at: (K[start[b] + at].double(), V[start[b] + at].double()), [1, 1], lens, 0.125)
    ref.close(O.to(torch.bfloat16), O, bound)
    with pytest.raises(AssertionError):
        ref.close(one.to(torch.bfloat16), O, bound)


@pytest.mark.gpu
@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [32, 64, 100, 128])
def test_few_queries(D, codes):
    """Up to 32 pairs of a query and a head of a key head's, 64 in 8 bits: units whole, dealt out, and under a window."""
    lens = [3000, 333, 70]
    cache = Cache(lens, 3000, 2, D, 16, codes).fill(D)
    for L in (1, 4, 8) + ((16,) if codes else ()):
        counts = [L, L, max(1, L - 3)]
        Q = queries(L, sum(counts), 8, D)
        for hints in (dict(max_k=400), dict(max_k=3000), dict(max_k=3000, window=700, sinks=5)):
            how = {k: v for k, v in hints.items() if k != "max_k"}
            O, bound, one = sharp(Q, cache.rows, counts, lens, D ** -0.5, **how)
            o = nm.nm_attention_paged(Q, *cache.args, offsets_q=offsets(counts), max_q=L, **hints, **cache.scales)
            ref.close(o, O, bound, (L, hints))
