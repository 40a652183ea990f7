"""Chunks on a cache in pages where a call's column tiles are not listed: as many new tokens in each sequence as was said, in sum, or very many
sequences."""
import pytest
import torch

import paper_2409_09708_amd as nm
from pages_reference import Cache
from test_gpu_paged import check, offsets, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("counts", [[300, 0, 60], [0, 360, 0], [1, 2, 357], [120, 120, 120], [121, 119, 120]])
def test_longer_than_was_said(counts, codes):
    cache = Cache([max(n, 200) for n in counts], 400, 2, 64, 16, codes).fill(1)
    check(cache, counts, 4, max_q=120)
    check(cache, counts, 4, max_q=120, window=70, sinks=3)
    check(cache, counts, 40, max_q=120)


@pytest.mark.parametrize("codes", [False, True])
def test_more_sequences_than_are_listed(codes):
    lens = [(37 * i) % 40 for i in range(530)]
    lens[7], lens[300], lens[529] = 300, 290, 299
    counts = [min(n, i % 3) for i, n in enumerate(lens)]
    counts[7], counts[300], counts[529] = 200, 70, 299
    cache = Cache(lens, 300, 1, 32, 16, codes).fill(2)
    check(cache, counts, 2, max_q=40)  # (longer ones than was said among them)
    check(cache, counts, 2, max_q=299)
    check(cache, counts, 3, max_q=33, window=50, sinks=2)


def test_as_fast_as_a_listed_call():
    """500 chunks of 64 on caches of 200, all as long, or one of them a token shorter: blocks do not go through the tiles of other sequences."""
    B, L = 500, 64
    cache = Cache([200] * B, 200, 2, 64, 16, False, waste=0.0)
    Q = queries(1, B * L, 8, 64)

    def us(counts):
        of = offsets(counts)
        out = torch.empty_like(Q)
        times = []
        for _ in range(12):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            for _ in range(4):
                nm.nm_attention_paged(Q[:sum(counts)], *cache.args, offsets_q=of, max_q=L, max_k=200, out=out[:sum(counts)])
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b) * 250)
        return sorted(times)[len(times) // 2]

    listed, equal = us([L] * (B - 1) + [L - 1]), us([L] * B)
    print(f"listed {listed:.1f} us, equal {equal:.1f} us")
    assert equal <= 1.5 * listed
