"""Infinities in the last row of a sequence: its tile's rest is no part of the sums, whatever the last row holds."""
import pytest
import torch

import block_reference as ref
from test_gpu_attention import offsets, tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("D,pad", [(32, 0), (64, 0), (128, 0), (64, 1), (80, 0)])
@pytest.mark.parametrize("Lq,Lk,Hq,Hkv", [(150, 150, 4, 2), (2, 333, 4, 2), (2, 5001, 8, 1), (2500, 130, 8, 8), (700, 65, 40, 8)])
def test_value_of_the_last_key(Lq, Lk, Hq, Hkv, D, pad, sign):
    """All queries see it: their output is infinite in that element, and what it is without it in the others."""
    import paper_2409_09708_amd as nm
    Q, K, V, _ = tensors(Lq + Lk + D, Lq, Lk, Hq, Hkv, D, pad=pad)
    V[-1, 0, 5] = sign * float("inf")
    got, lse = nm.nm_attention(Q, K, V, lse=True)
    o, bo, l, bl = ref.attention(Q, K, V, False, D ** -0.5, [(0, Lq)], [(0, Lk)])
    assert bool((o[:, :Hq // Hkv, 5] == sign * float("inf")).all())
    ref.close(got, o, bo, "O")
    ref.close(lse, l, bl, "lse")


def test_value_of_the_last_key_in_use():
    """Of packed caches of fixed capacity, what lies behind it being anything."""
    import paper_2409_09708_amd as nm
    lens, room = [70, 33, 1500, 1], 1500
    Q, K, V, _ = tensors(3, 4, 4 * room, 8, 2, 128)
    for b, n in enumerate(lens):
        V[b * room + n - 1, 1, 9] = float("inf")
        K[b * room + n:(b + 1) * room] = float("nan")
        V[b * room + n:(b + 1) * room] = float("nan")
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    at = dict(offsets_q=offsets([1] * 4), offsets_k=offsets([room] * 4), lengths_k=lengths)
    for causal in (False, True):
        for max_k in (room, 40):
            got = nm.nm_attention(Q, K, V, causal, max_q=1, max_k=max_k, **at)
            o, bo, *_ = ref.attention(Q, K, V, causal, 128 ** -0.5, ref.spans(4, at["offsets_q"], None, 4), ref.spans(4 * room, at["offsets_k"], lengths, 4))
            assert bool((o[:, 4:, 9] == float("inf")).all())
            ref.close(got, o, bo)


@pytest.mark.parametrize("D,pad", [(32, 0), (64, 0), (128, 0), (64, 1), (80, 0)])
@pytest.mark.parametrize("Lq,Lk", [(150, 150), (65, 300), (2049, 70)])
def test_gradient_of_the_last_query(Lq, Lk, D, pad):
    """An infinity in the last row of dO: dV is infinite in that element, and what it is without it in the others."""
    import paper_2409_09708_amd as nm
    Q, K, V, dO = tensors(Lq + Lk + D, Lq, Lk, 4, 2, D, pad=pad)
    O, lse = nm.nm_attention(Q, K, V, lse=True)
    dO[-1, 1, 5] = float("inf")
    dV = nm.nm_attention_backward(dO, Q, K, V, O, lse)[2]
    want, bound = ref.attention_grad(dO, Q, K, V, O, lse, False, D ** -0.5, [(0, Lq)], [(0, Lk)])[2]
    assert bool((want[:, 0, 5] == float("inf")).all()) and bool(torch.isfinite(want[:, 1]).all())
    ref.close(dV, want, bound)
