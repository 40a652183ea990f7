"""Attention and its backward pass against their definitions in 64 bits."""
import pytest
import torch

import block_reference as ref

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def offsets(lengths):
    return torch.tensor([0] + lengths).cumsum(0).to(torch.int32).cuda()


def tensors(seed, Tq, Tk, Hq, Hkv, D, fused=False, pad=0, scale=1.0):
    g = torch.Generator("cuda")
    g.manual_seed(seed)

    def heads(T, H):
        t = torch.randn(T, H, D + pad, generator=g, device="cuda").mul_(scale).to(BF16)
        return t[..., :D]

    if fused:
        row = torch.randn(Tq, (Hq + 2 * Hkv) * D, generator=g, device="cuda").mul_(scale).to(BF16)
        return [t.unflatten(1, (-1, D)) for t in row.split([Hq * D, Hkv * D, Hkv * D], 1)] + [heads(Tq, Hq)]
    return [heads(Tq, Hq), heads(Tk, Hkv), heads(Tk, Hkv), heads(Tq, Hq)]


def check(Q, K, V, dO, causal, scale=None, q_lens=None, k_lens=None, lengths_k=None, backward=True, **hints):
    import paper_2409_09708_amd as nm
    oq = None if q_lens is None else offsets(q_lens)
    ok = None if k_lens is None else offsets(k_lens)
    n = len(q_lens) if q_lens else 1
    at = dict(scale=scale, offsets_q=oq, offsets_k=ok, lengths_k=lengths_k, **hints)
    O, lse = nm.nm_attention(Q, K, V, causal, lse=True, **at)
    s = scale if scale is not None else Q.shape[2] ** -0.5
    qs, ks = ref.spans(Q.shape[0], oq, None, n), ref.spans(K.shape[0], ok, lengths_k, n)
    o, bo, l, bl = ref.attention(Q, K, V, causal, s, qs, ks)
    ref.close(O, o, bo, "O")
    ref.close(lse, l, bl, "lse")
    assert torch.equal(nm.nm_attention(Q, K, V, causal, **at), O)
    if not backward:
        return
    got = nm.nm_attention_backward(dO, Q, K, V, O, lse, causal, **at)
    for name, t, (v, b) in zip(("dQ", "dK", "dV"), got, ref.attention_grad(dO, Q, K, V, O, lse, causal, s, qs, ks)):
        ref.close(t, v, b, name)
    again = nm.nm_attention_backward(dO, Q, K, V, O, lse, causal, **at)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("L", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 130, 197, 256, 300, 700])
def test_one_sequence(L, causal):
    check(*tensors(L, L, L, 3, 3, 64), causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D", [1, 7, 8, 24, 31, 32, 40, 64, 72, 80, 96, 100, 127, 128])
def test_head_sizes(D, causal):
    check(*tensors(D, 150, 150, 4, 2, D), causal)
    check(*tensors(D, 20, 333, 4, 2, D), causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (6, 1), (8, 2), (12, 4), (40, 8)])
def test_shared_heads(Hq, Hkv, causal):
    check(*tensors(Hq, 140, 140, Hq, Hkv, 64, fused=True), causal)
    check(*tensors(Hq, 3, 270, Hq, Hkv, 64), causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("Lq,Lk", [(1, 1), (1, 5), (1, 1000), (4, 1000), (5, 3), (200, 130), (130, 200), (300, 1), (1, 0), (260, 0), (64, 2100),
                                   (131, 700)])
def test_queries_and_keys_of_different_lengths(Lq, Lk, causal):
    check(*tensors(Lq * 1009 + Lk, Lq, Lk, 4, 2, 128), causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D", [64, 80, 128])
def test_packed(D, causal):
    lens = [197, 0, 1, 64, 65, 333, 0, 128, 2]
    T = sum(lens)
    check(*tensors(D, T, T, 4, 2, D, fused=True), causal, q_lens=lens, k_lens=lens, max_q=max(lens), max_k=max(lens))
    check(*tensors(D, T, T, 4, 2, D), causal, q_lens=lens, k_lens=lens)             # no word about the lengths
    check(*tensors(D, T, T, 4, 2, D), causal, q_lens=lens, k_lens=lens, max_q=1, max_k=1)  # a wrong one
    check(*tensors(D, T, T, 4, 2, D), causal, q_lens=lens, k_lens=lens[::-1], max_q=333, max_k=333)


@pytest.mark.parametrize("group", [1, 4, 8])
@pytest.mark.parametrize("Lq", [1, 3, 17])
@pytest.mark.parametrize("D", [64, 128, 50])
def test_cache(D, Lq, group):
    """New tokens against caches of fixed capacity, what lies past their lengths being anything."""
    B, room, Hkv = 5, 1500, 2
    lens = [1500, 17, 0, 33, 700]
    Q, K, V, dO = tensors(D + Lq, B * Lq, B * room, Hkv * group, Hkv, D)
    for b, n in enumerate(lens):
        K[b * room + n:(b + 1) * room] = float("nan")
        V[b * room + n:(b + 1) * room] = float("inf")
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for hints in (dict(max_q=Lq, max_k=room), dict(max_q=Lq, max_k=40), dict()):
        check(Q, K, V, dO, True, q_lens=[Lq] * B, k_lens=[room] * B, lengths_k=lengths, backward=Lq == 3, **hints)


def test_many_long_chunks():
    """Keys cut into many chunks, joined in order; a first chunk of scores far below the rest."""
    Q, K, V, dO = tensors(1, 2, 40000, 8, 1, 128)
    K[:5000] = -K[5000:10000].abs() * torch.sign(Q[0, 0])
    check(Q, K, V, dO, True, backward=False)


@pytest.mark.parametrize("pad", [1, 3, 8])
@pytest.mark.parametrize("D", [64, 96])
def test_strides(D, pad):
    check(*tensors(pad, 170, 170, 4, 2, D, pad=pad), True)
    check(*tensors(pad, 5, 170, 4, 2, D, pad=pad), True)


def test_other_orders_and_broadcast_keys():
    """Heads before tokens, and one key head expanded to all heads (its gradient comes per head)."""
    import paper_2409_09708_amd as nm
    Q, K, V, dO = tensors(7, 150, 150, 4, 1, 64)
    order = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (Q, K, V, dO)]
    check(*order, True)
    K4, V4 = K.expand(-1, 4, -1), V.expand(-1, 4, -1)
    check(Q, K4, V4, dO, True)
    O, lse = nm.nm_attention(Q, K, V, True, lse=True)
    out = torch.empty(4, 150, 64, dtype=BF16, device="cuda").transpose(0, 1)
    assert nm.nm_attention(Q, K4, V4, True, out=out) is out and torch.equal(out, O)


def test_gradients_into_a_joint_projection():
    import paper_2409_09708_amd as nm
    Q, K, V, dO = tensors(8, 200, 200, 6, 2, 64, fused=True)
    O, lse = nm.nm_attention(Q, K, V, True, lse=True)
    want = nm.nm_attention_backward(dO, Q, K, V, O, lse, True)
    row = torch.full((200, 10 * 64), float("nan"), dtype=BF16, device="cuda")
    views = [t.unflatten(1, (-1, 64)) for t in row.split([384, 128, 128], 1)]
    nm.nm_attention_backward(dO, Q, K, V, O, lse, True, out=views)
    assert torch.equal(row, torch.cat([t.flatten(1) for t in want], 1))


def test_large_scores():
    """Rows decided by one key, and scores whose exponentials would overflow without the running maximum."""
    for scale in (1.0, 8.0):
        check(*tensors(21, 180, 180, 2, 2, 64, scale=2.0), False, scale=scale, backward=scale == 1.0)
    check(*tensors(22, 2, 3000, 2, 2, 64, scale=2.0), True, scale=8.0, backward=False)


def test_keys_of_minus_infinity_do_not_count():
    """A key whose score is -infinity (the lowest there is) has no weight; with nothing but such keys there is no output."""
    import paper_2409_09708_amd as nm
    for Lq in (150, 2):
        Q, K, V, _ = tensors(23, Lq, 150, 2, 2, 64)
        Q[...] = Q.abs() + 0.1
        kept = torch.arange(150, device="cuda") % 3 == 0
        Kinf = torch.where(kept[:, None, None], K, torch.tensor(float("-inf"), dtype=BF16, device="cuda"))
        got, lse = nm.nm_attention(Q, Kinf, V, lse=True)
        o, bo, l, bl = ref.attention(Q, K[kept], V[kept], False, 0.125, [(0, Lq)], [(0, 50)])
        ref.close(got, o, bo)
        ref.close(lse, l, bl)
        none, lse = nm.nm_attention(Q, torch.full_like(K, float("-inf")), V, lse=True)
        assert float(none.abs().max()) == 0 and bool((lse == -float("inf")).all())


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D", [32, 40, 64, 100, 128])
def test_many_sequences(D, causal):
    """More query tiles than blocks: some with no queries, no keys, fewer keys than queries, and more tiles than the hint says."""
    lens = [(0, 5), (1, 1), (130, 0), (300, 300), (127, 64), (0, 0), (64, 200), (257, 31), (128, 128), (3, 65), (200, 129)] * 9
    Tq, Tk = sum(q for q, _ in lens), sum(k for _, k in lens)
    Q, K, V, dO = tensors(27, Tq, Tk, 8, 4, D)
    for hint in (300, 150):
        check(Q, K, V, dO, causal, q_lens=[q for q, _ in lens], k_lens=[k for _, k in lens], backward=hint == 300, max_q=hint, max_k=300)


@pytest.mark.parametrize("Lq,Lk,H", [(2, 3000, 2), (150, 150, 2), (2500, 130, 8)])
def test_nan_stays_in_its_row(Lq, Lk, H):
    """A query that holds a NaN has an output and a log-sum of NaN; the other queries have their own."""
    import paper_2409_09708_amd as nm
    Q, K, V, _ = tensors(25, Lq, Lk, H, H, 64)
    o, bo, l, bl = ref.attention(Q, K, V, False, 0.125, [(0, Lq)], [(0, Lk)])
    Q[1, 0, 5] = float("nan")
    got, lse = nm.nm_attention(Q, K, V, lse=True)
    assert bool(got[1, 0].isnan().all()) and bool(lse[0, 1].isnan())
    got[1, 0], lse[0, 1] = o[1, 0], l[0, 1]
    ref.close(got, o, bo)
    ref.close(lse, l, bl)


def test_offsets_past_32_bits():
    """A cache of over 2^31 elements, its last sequence behind them."""
    import paper_2409_09708_amd as nm
    room, Hkv, D, B = 1 << 20, 8, 128, 3  # 3 x 2^30 elements
    K = torch.zeros(B * room, Hkv, D, dtype=BF16, device="cuda")
    V = torch.zeros(B * room, Hkv, D, dtype=BF16, device="cuda")
    Q, k, v, _ = tensors(31, B, 500, 16, Hkv, D)
    first = [room - 500, 2 * room - 500, 3 * room - 500]
    for at in first:
        K[at:at + 500], V[at:at + 500] = k, v
    at = torch.tensor([0] + first[:2] + [3 * room], dtype=torch.int32, device="cuda")
    o = nm.nm_attention(Q[:1], K[first[2]:], V[first[2]:], True)
    lens = torch.tensor([500, 500, 500], dtype=torch.int32, device="cuda")
    offs = torch.tensor(first + [3 * room], dtype=torch.int32, device="cuda")
    got = nm.nm_attention(Q, K, V, True, offsets_q=offsets([1, 1, 1]), offsets_k=offs, lengths_k=lens, max_q=1, max_k=500)
    assert torch.equal(got[0], o[0])
    for b in range(3):
        assert torch.equal(got[b], nm.nm_attention(Q[b:b + 1], k, v, True)[0])


def test_offsets_that_lie():
    """Offsets outside the tensors are taken as their ends: nothing outside is read or written."""
    import paper_2409_09708_amd as nm
    Q, K, V, dO = tensors(33, 100, 100, 2, 2, 64)
    bad = torch.tensor([-50, 1000], dtype=torch.int32, device="cuda")
    lens = torch.tensor([1 << 30], dtype=torch.int32, device="cuda")
    want, lse = nm.nm_attention(Q, K, V, lse=True)
    assert torch.equal(nm.nm_attention(Q, K, V, offsets_q=bad, offsets_k=bad, lengths_k=lens), want)
    back = torch.tensor([80, 20], dtype=torch.int32, device="cuda")
    nm.nm_attention(Q, K, V, offsets_q=back, offsets_k=back)
    got = nm.nm_attention_backward(dO, Q, K, V, want, lse, offsets_q=bad, offsets_k=bad, lengths_k=lens)
    assert all(torch.equal(a, b) for a, b in zip(got, nm.nm_attention_backward(dO, Q, K, V, want, lse)))


def test_gradient_is_that_of_differences():
    """Along random directions, against differences of the definition in 64 bits."""
    import paper_2409_09708_amd as nm
    Q, K, V, dO = tensors(41, 70, 90, 4, 2, 64)
    O, lse = nm.nm_attention(Q, K, V, True, lse=True)
    got = nm.nm_attention_backward(dO, Q, K, V, O, lse, True)
    bounds = ref.attention_grad(dO, Q, K, V, O, lse, True, 0.125, [(0, 70)], [(0, 90)])
    base = [t.double() for t in (Q, K, V)]
    # the O given is rounded: dO . o is off by up to 2^-8 |dO| |O|, which p and the keys (queries) carry into dQ (dK)
    rough = (dO.double().abs() * O.double().abs()).sum(-1).max() * ref.U16
    for n in range(3):
        way = torch.randn(base[n].shape, dtype=torch.float64, device="cuda", generator=torch.Generator("cuda").manual_seed(n))

        def loss(h):
            x = [t + h * way if i == n else t for i, t in enumerate(base)]
            return (ref.attention(*x, True, 0.125, [(0, 70)], [(0, 90)])[0] * dO.double()).sum()

        diff = (loss(1e-4) - loss(-1e-4)) / 2e-4
        along = (got[n].double() * way).sum()
        slack = (bounds[n][1] * way.abs()).sum()
        if n < 2:  # sum over rows of |rough| p_ij |k_j| scale (p sums to one), or over columns
            slack = slack + rough * 0.125 * base[1 - n].abs().amax() * way.abs().sum() * (1 if n == 0 else 4 * 70 / 90)
        assert abs(float(along - diff)) <= float(slack) + 1e-6 * abs(float(diff)), n


def test_other_stream_and_capture():
    import paper_2409_09708_amd as nm
    Q, K, V, dO = tensors(51, 3, 5000, 8, 2, 128)
    want = nm.nm_attention(Q, K, V, True, lse=True)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = nm.nm_attention(Q, K, V, True, lse=True, stream=stream)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")

    def step():
        O, lse = nm.nm_attention(Q, K, V, True, lse=True, workspace=ws)
        return (O, *nm.nm_attention_backward(dO, Q, K, V, O, lse, True, workspace=ws))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for n in range(3):
        Q.copy_(tensors(60 + n, 3, 1, 8, 2, 128)[0])
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in outs]
        assert all(torch.equal(a, b) for a, b in zip(kept, step()))
