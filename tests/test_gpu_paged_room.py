"""Sequences that are longer than their tables have room for: what fits is kept, and is seen from where it stands."""
import pytest
import torch

import paper_2409_09708_amd as nm
import block_reference as ref
import pages_reference as pages
from pages_reference import Cache
from paper_2409_09708_amd.block import PagedCache
from test_gpu_paged import offsets, queries

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
LENS, PAGE, WIDTH = [50, 61, 20], 16, 3  # (room for 48)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("window,sinks", [(0, 0), (7, 0), (13, 3), (1, 1)])
@pytest.mark.parametrize("counts", [[1, 1, 1], [5, 14, 3], [50, 61, 20]])
def test_queries_stand_where_their_tokens_do(counts, window, sinks, codes):
    cache = Cache(LENS, 64, 2, 64, PAGE, codes).fill(1)
    Q = queries(1, sum(counts), 4, 64)
    want = pages.paged(Q, cache, counts, 0.125, window, sinks, gone=[(0, WIDTH), (1, WIDTH)])  # (the tokens behind the room are not there)
    table = cache.table[:, :WIDTH].contiguous()
    for hints in (dict(), dict(max_q=max(counts)), dict(max_q=max(counts), max_k=3000), dict(max_q=200)):
        o, lse = nm.nm_attention_paged(Q, cache.K, cache.V, table, cache.lengths, offsets_q=offsets(counts), window=window, sinks=sinks, lse=True,
                                       **cache.scales, **hints)
        ref.close(o, want[0], want[1], (counts, hints))
        ref.close(lse, want[2], want[3], (counts, hints))


@pytest.mark.parametrize("length", [2 ** 30, 2 ** 31 - 1])
def test_longest_lengths(length):
    """New tokens far behind all that is kept see it, but for what their window has left behind."""
    cache = Cache([48], 48, 2, 64, PAGE, False).fill(2)
    Q = queries(2, 40, 4, 64)
    want = pages.paged(Q[:1], cache, [1], 0.125)
    first = pages.paged(Q[:1], cache, [1], 0.125, gone=[(0, 1), (0, 2)])  # (the first page's keys)
    cache.lengths.fill_(length)
    for L in (1, 40):
        o = nm.nm_attention_paged(Q[:L], *cache.args)
        ref.close(o[:1], want[0], want[1], L)
        assert not bool(nm.nm_attention_paged(Q[:L], *cache.args, window=1000).any())
        o = nm.nm_attention_paged(Q[:L], *cache.args, window=1000, sinks=PAGE)
        ref.close(o[:1], first[0], first[1], L)


@pytest.mark.parametrize("eight_bits", [False, True])
def test_written_past_the_room_and_attended(eight_bits):
    """As a replayed graph does it, whose host does not know the lengths: the token that fits is seen by its own query."""
    small, large = (PagedCache.empty(1, room, 2, 64, PAGE, eight_bits=eight_bits) for room in (48, 64))
    k, v, q = queries(3, 50, 2, 64), queries(4, 50, 2, 64), queries(5, 3, 4, 64)
    got = []
    for cache in (small, large):
        cache.keep(k[:47], v[:47], offsets([47]))
        cache.keep(k[47:], v[47:], offsets([3]))
        assert cache.lengths.tolist() == [50]
        got.append(cache.attend(q, offsets([3]), 3, 48))
    assert torch.equal(got[0][0], got[1][0])
    without, _ = small.read(offsets([48]), 48)
    assert torch.equal(without, large.read(offsets([48]), 48)[0])
