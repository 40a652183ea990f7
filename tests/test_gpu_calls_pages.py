"""Native marshalling of the norm of heads and of a cache in pages against the Python functions it stands in for."""
import pytest
import torch

import paper_2409_09708_amd as nm
from pages_reference import Cache
from paper_2409_09708_amd import binding
from test_gpu_calls_block import both_ways

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("T,D", [(1, 64), (300, 80)])
@pytest.mark.parametrize("dtype", [torch.float32, BF16])
def test_head_norm(monkeypatch, T, D, dtype):
    X, dY = (torch.randn(T, 6 * D, device="cuda").to(dtype)[:, :5 * D].unflatten(1, (5, D)) for _ in range(2))
    w, w1 = torch.randn(2, D, device="cuda"), torch.randn(D, device="cuda")
    pos, freqs = torch.randint(0, 50, (T, 2), device="cuda", dtype=torch.int32), torch.rand(D // 4, device="cuda")
    turn = dict(positions=pos, freqs=freqs, sections=(D // 8, D // 8))
    at = pos[:, 0].float().contiguous()
    own = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()

    def run(stream):
        out, dx = torch.zeros(T, 5, D, device="cuda"), torch.zeros(T, 5, D, device="cuda")
        torch.cuda.synchronize()
        assert nm.nm_head_norm(X, w, 3, 1e-5, True, **turn, interleaved=True, out=out, stream=stream) is out
        back = nm.nm_head_norm_backward(dY, X, w, 3, 1e-5, True, **turn, interleaved=True, out=dx, stream=stream)
        assert back[0] is dx
        return [out, back, nm.nm_head_norm(X, stream=stream), nm.nm_head_norm(X, w1, out_dtype=BF16, stream=stream),
                nm.nm_head_norm(X, w1, positions=at, freqs=freqs, stream=stream),
                nm.nm_head_norm_backward(dY, X, w1, out_dtype=BF16, workspace=own, stream=stream),
                nm.nm_head_norm_backward(dY, X, stream=stream), nm.nm_head_norm_backward(dY, X, w, 3, params=False, stream=stream)]

    both_ways(monkeypatch, run)
    assert binding._CALLS.head_norm(X, w, 3, 1e-5, True, pos, freqs, (D // 8, D // 8), True, None, None, None) is not NotImplemented


@pytest.mark.parametrize("codes", [False, True])
def test_cache_and_attention(monkeypatch, codes):
    cache = Cache([700, 20], 700, 2, 64, 16, codes, waste=0.0).fill(1)
    K, V, Q = (torch.randn(8, h, 64, device="cuda").to(BF16) for h in (2, 2, 4))
    of = torch.tensor([0, 5, 8], dtype=torch.int32, device="cuda")
    first = torch.tensor([695, 17], dtype=torch.int32, device="cuda")
    own = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()

    def run(stream):
        out, read = torch.zeros_like(Q), (torch.zeros_like(K), torch.zeros_like(V))
        torch.cuda.synchronize()
        assert nm.nm_cache_write(K, V, *cache.args, offsets=of, **cache.scales, stream=stream) is None
        assert nm.nm_cache_read(*cache.args, of, first=first, out=read, **cache.scales, stream=stream) == read
        o, lse = nm.nm_attention_paged(Q, *cache.args, 0.25, of, 90, 3, max_q=5, max_k=700, lse=True, out=out, **cache.scales, stream=stream)
        assert o is out
        return [o, lse, read, nm.nm_cache_read(*cache.args, of, 8, first, **cache.scales, stream=stream),
                nm.nm_attention_paged(Q, *cache.args, **cache.scales, stream=stream),
                nm.nm_attention_paged(Q, *cache.args, offsets_q=of, workspace=own, **cache.scales, stream=stream)]

    both_ways(monkeypatch, run)
    assert binding._CALLS.attention_paged(Q, *cache.args, None, of, 0, 0, cache.K_scales, cache.V_scales, None, None, False, None, None,
                                          None) is not NotImplemented
    assert binding._CALLS.cache_write(K, V, *cache.args, of, cache.K_scales, cache.V_scales, None) is None


def test_refusals_reach_the_caller():
    cache = Cache([30], 32, 2, 64, 16, True)
    x = torch.zeros(4, 2, 64, dtype=BF16, device="cuda")
    with pytest.raises(nm.NmError):
        nm.nm_head_norm(x, eps=-1.0)
    with pytest.raises(ValueError, match="weight"):
        nm.nm_head_norm(x, torch.ones(2, 64, device="cuda"))
    with pytest.raises(ValueError, match="positions"):
        nm.nm_head_norm(x, freqs=torch.ones(32, device="cuda"))
    with pytest.raises(nm.NmError):
        nm.nm_attention_paged(x, *cache.args, scale=-1.0, **cache.scales)
    with pytest.raises(ValueError, match="scales"):
        nm.nm_attention_paged(x, *cache.args)
    with pytest.raises(ValueError, match="K must be"):
        nm.nm_cache_write(x[:, :1], x, *cache.args, **cache.scales)
    with pytest.raises(ValueError, match="tokens"):
        nm.nm_cache_read(*cache.args, **cache.scales)
    with pytest.raises(nm.NmError):
        nm.nm_cache_write(x, x, cache.K[:, :1].expand(-1, 16, -1, -1), cache.V[:, :1].expand(-1, 16, -1, -1), cache.table, cache.lengths, **cache.scales)
