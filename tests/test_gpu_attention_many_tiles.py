"""Sequences of so many query tiles that these go round the chip by other rules, with few key tiles cut for several blocks."""
import pytest

from test_gpu_attention import check, tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D,pad", [(64, 0), (128, 0), (64, 1), (128, 8), (96, 0)])
@pytest.mark.parametrize("lens", [[2049, 1, 0, 2305, 300], [1920, 333], [40, 1921], [2177]])
def test_on_both_sides_of_sixteen_tiles(lens, D, pad, causal):
    """19, 15, 16 and 18 tiles of the longest sequence, four query heads to a key head."""
    T = sum(lens)
    check(*tensors(T + D, T, T, 4, 1, D, pad=pad), causal, q_lens=lens, k_lens=lens, max_q=max(lens), max_k=max(lens))


@pytest.mark.parametrize("causal", [False, True])
def test_many_heads(causal):
    lens = [2050, 130, 2176]
    T = sum(lens)
    check(*tensors(17, T, T, 6, 3, 64, fused=True), causal, q_lens=lens, k_lens=lens, max_q=2176, max_k=2176)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("q_lens,k_lens", [([2100, 77], [300, 2200]), ([200, 2300], [2600, 2000])])
def test_queries_and_keys_of_different_lengths(q_lens, k_lens, causal):
    check(*tensors(19, sum(q_lens), sum(k_lens), 4, 1, 128), causal, q_lens=q_lens, k_lens=k_lens, max_q=max(q_lens), max_k=max(k_lens))
