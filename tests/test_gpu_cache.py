"""A cache of keys and values in pages: what is written, where, and what is read back."""
import math

import pytest
import torch

from pages_reference import Cache, E4M3, rounded

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def offsets(counts):
    return torch.tensor([0] + list(counts)).cumsum(0).to(torch.int32).cuda()


def tokens(seed, T, H, D, pad=0, scale=1.0):
    g = torch.Generator("cuda").manual_seed(seed)
    return [torch.randn(T, H, D + pad, generator=g, device="cuda").mul_(scale).to(BF16)[..., :D] for _ in range(2)]


def same(a, b):
    """Bit for bit, any NaN being as good as another."""
    if a.dtype == E4M3:
        a, b = a.float(), b.float()
    if a.is_floating_point():
        assert torch.equal(a.isnan(), b.isnan())
        a, b = a.nan_to_num(), b.nan_to_num()
    assert torch.equal(a, b)


def check(lens, counts, room, H, D, page, codes, order="heads", seed=0, pad=0, given=True, K=None, V=None):
    """New tokens written as by indexing with the definition's values; nothing else changes; and read back."""
    import paper_2409_09708_amd as nm
    ours, want = (Cache(lens, room, H, D, page, codes, seed, order, waste=3.0) for _ in range(2))
    if K is None:
        K, V = tokens(seed, sum(counts), H, D, pad)
    at = 0
    for b, (n, new) in enumerate(zip(lens, counts)):
        where = torch.arange(n - new, n, device="cuda")
        keep = (where >= 0) & (where < want.table.shape[1] * page)
        want.put(b, where[keep], K[at:at + new][keep], V[at:at + new][keep])
        at += new
    of = offsets(counts) if given else None
    assert nm.nm_cache_write(K, V, *ours.args, offsets=of, **ours.scales) is None
    for name in ("K", "V", "K_scales", "V_scales"):
        if getattr(ours, name) is not None:
            same(getattr(ours, name), getattr(want, name))
    first = (ours.lengths - torch.tensor(counts, device="cuda")).to(torch.int32)
    k, v = nm.nm_cache_read(*ours.args, of, tokens=sum(counts), first=first, **ours.scales)
    at = 0
    for b, (n, new) in enumerate(zip(lens, counts)):
        where = torch.arange(n - new, n, device="cuda")
        keep = (where >= 0) & (where < ours.table.shape[1] * page)  # (the other rows are left as they were)
        for got, x in ((k, K), (v, V)):
            x = x[at:at + new][keep]
            same(got[at:at + new][keep], rounded(x)[0].to(BF16) if codes else x)
        at += new
    return ours


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("page", [1, 2, 7, 16, 64, 100, 256])
def test_pages(page, codes):
    check([300, 1, 64, 65, 5], [300, 1, 0, 64, 2], 300, 3, 64, page, codes)
    check([300, 17, 64], [1, 1, 1], 300, 8, 128, page, codes, order="tokens", given=False)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("order", ["heads", "tokens"])
@pytest.mark.parametrize("D", [1, 7, 8, 15, 16, 17, 24, 32, 40, 64, 80, 100, 127, 128])
def test_head_sizes(D, order, codes):
    check([40, 33], [40, 20], 45, 2, D, 8, codes, order, pad=D % 3)


@pytest.mark.parametrize("codes", [False, True])
def test_many_sequences(codes):
    """More than a wave finds at once; several of them empty."""
    lens = [(7 * i) % 23 for i in range(200)]
    check(lens, [min(n, i % 4) for i, n in enumerate(lens)], 23, 1, 32, 4, codes)
    lens = [1 + i % 3 for i in range(5000)]
    check(lens, [int(i % 7 == 0) for i in range(5000)], 3, 2, 16, 2, codes)


def test_every_bfloat16():
    """All patterns, beside maxima that put the power of two anywhere: zeros, subnormals, infinities and NaN among them."""
    x = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(BF16).cuda().view(-1, 2, 16)
    check([2048], [2048], 2048, 2, 16, 64, True, K=x, V=x.flip(0).contiguous())
    g = torch.Generator("cuda").manual_seed(1)
    mixed = x.flatten()[torch.randperm(65536, generator=g, device="cuda")].view(-1, 1, 64)
    check([512, 512], [512, 512], 512, 1, 64, 16, True, K=mixed, V=mixed)
    top = torch.full((4, 1, 32), 3.3895e38, dtype=BF16, device="cuda")
    top[1], top[2, 0, 3], top[3] = -1e-40, math.inf, 0.0
    cache = check([4], [4], 4, 1, 32, 4, True, K=top, V=-top)
    assert cache.K_scales[cache.table[0, 0].item(), :, 0].tolist() == [246, 27, 246, 27]


def test_values_read_back_are_near():
    """Within half a step of three bits of mantissa, and of the smallest multiple beside the row's largest."""
    import paper_2409_09708_amd as nm
    K, V = tokens(3, 500, 4, 128, scale=5.0)
    cache = Cache([500], 500, 4, 128, 16, True)
    nm.nm_cache_write(K, V, *cache.args, **cache.scales)
    for got, x in zip(nm.nm_cache_read(*cache.args, tokens=500, **cache.scales), (K, V)):
        x = x.double()
        power = torch.exp2(torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / 448)))
        assert bool(((got.double() - x).abs() <= torch.maximum(x.abs() * 2.0 ** -4, power * 2.0 ** -10)).all())


@pytest.mark.parametrize("codes", [False, True])
def test_what_does_not_fit_is_dropped(codes):
    """Tokens before the first or behind the table's last, and on pages that are not there; and lengths of nothing."""
    import paper_2409_09708_amd as nm
    check([10, 3, 0, 20], [10, 5, 0, 6], 16, 2, 32, 4, codes)  # (the second has more new tokens than tokens, the last one's end is behind the table)
    cache, before = (Cache([16, 16, 16], 16, 2, 32, 4, codes, waste=2.0) for _ in range(2))
    cache.table[0, 1], cache.table[1, 0], cache.table[2, 3] = -1, cache.count, 2 ** 31 - 1
    K, V = tokens(5, 48, 2, 32)
    nm.nm_cache_write(K, V, *cache.args, **cache.scales)
    k, v = nm.nm_cache_read(*cache.args, tokens=48, **cache.scales)
    gone = [range(4, 8), range(16, 20), range(44, 48)]
    kept = torch.ones(48, dtype=torch.bool)
    for r in gone:
        kept[list(r)] = False
    kept = kept.cuda()
    for got, x in ((k, K), (v, V)):
        same(got[kept], (rounded(x)[0].to(BF16) if codes else x)[kept])
        assert not bool(got[~kept].any())
    pages = torch.ones(cache.count, dtype=torch.bool)
    pages[[p for p in cache.table.flatten().tolist() if 0 <= p < cache.count]] = False
    pages = pages.cuda()
    raw = (lambda t: t.float()) if codes else (lambda t: t)
    assert torch.equal(raw(cache.K)[pages], raw(before.K)[pages]) and torch.equal(raw(cache.V)[pages], raw(before.V)[pages])


@pytest.mark.parametrize("codes", [False, True])
def test_rows_that_no_token_fills_stay(codes):
    import paper_2409_09708_amd as nm
    cache = Cache([9, 0, 5], 12, 2, 48, 4, codes).fill(1)
    out = tuple(torch.full((30, 2, 60), 9.0, dtype=BF16, device="cuda")[..., :48] for _ in range(2))
    of = torch.tensor([2, 14, 16, 25], dtype=torch.int32, device="cuda")
    first = torch.tensor([6, 0, -1], dtype=torch.int32, device="cuda")
    assert nm.nm_cache_read(*cache.args, of, first=first, out=out, **cache.scales) == out
    for got, i in ((out[0], 0), (out[1], 1)):
        same(got[2:5].double(), cache.rows(0, torch.arange(6, 9, device="cuda"))[i])
        same(got[17:22].double(), cache.rows(2, torch.arange(5, device="cuda"))[i])  # (its row 16 would be token -1)
        rest = torch.ones(30, dtype=torch.bool, device="cuda")
        rest[2:5] = rest[17:22] = False
        assert bool((got[rest] == 9).all())
    whole = nm.nm_cache_read(*cache.args, offsets([9, 0, 5]), tokens=14, **cache.scales)
    same(whole[0][9:].double(), cache.rows(2, torch.arange(5, device="cuda"))[0])


def test_offsets_that_lie_stay_inside():
    """Whatever offsets and lengths hold, nothing outside the tensors is touched, and sequences that are right are kept."""
    import paper_2409_09708_amd as nm
    K, V = tokens(6, 12, 2, 32)
    for of in ([0, 4, 900, 12], [-50, 4, 8, 12], [0, 8, 4, 12], [2 ** 31 - 1] * 4, [-2 ** 31] * 4, [0, 0, 0, 0]):
        for lens in ([4, 4, 4], [2 ** 31 - 1, -5, 4], [-2 ** 31, 2 ** 31 - 1, 0]):
            cache = Cache(lens, 8, 2, 32, 4, False, waste=1.0)
            at = torch.tensor(of, dtype=torch.int32, device="cuda")
            nm.nm_cache_write(K, V, *cache.args, offsets=at)
            nm.nm_cache_read(*cache.args, at, tokens=12)
            torch.cuda.synchronize()
            spare = torch.ones(cache.count, dtype=torch.bool, device="cuda")
            spare[cache.table.flatten().long()] = False
            assert bool((cache.K[spare] == 1).all())


def test_long_cache_past_32_bits():
    """Pages whose offsets pass 2^31 elements."""
    import paper_2409_09708_amd as nm
    pages = torch.empty(70000, 64, 4, 128, dtype=torch.uint8, device="cuda").view(E4M3)
    scales = torch.empty(70000, 64, 4, dtype=torch.uint8, device="cuda")
    table = torch.tensor([[69999, 3], [40000, 69998]], dtype=torch.int32, device="cuda")
    K, V = tokens(7, 200, 4, 128)
    lengths = torch.tensor([100, 100], dtype=torch.int32, device="cuda")
    at = (pages, pages.clone(), table, lengths)
    both = dict(K_scales=scales, V_scales=scales.clone())
    nm.nm_cache_write(K, V, *at, **both)
    k, v = nm.nm_cache_read(*at, tokens=200, **both)
    same(k, rounded(K)[0].to(BF16))
    same(v, rounded(V)[0].to(BF16))
    Q = tokens(8, 2, 8, 128)[0]
    o = nm.nm_attention_paged(Q, *at, **both)
    want = nm.nm_attention(Q, k, v, True, offsets_q=offsets([1, 1]), offsets_k=offsets([100, 100]))
    assert float((o.float() - want.float()).abs().max()) <= 2.0 ** -6 * float(want.float().abs().max())
