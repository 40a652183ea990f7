"""A workspace of the size that the library names does for the call, and for calls with shorter caches."""
import pytest
import torch

from paper_2409_09708_amd import binding

CAPACITIES = sorted({*range(1, 3000, 97), *range(3000, 140001, 1711), *(512 * n + d for n in range(1, 100, 7) for d in (-1, 0, 1)),
                     8192, 9000, 10240, 12288, 13000, 16384, 98304, 120000, 131072})


@pytest.mark.parametrize("Tq,B,Hq,Hkv,D,max_q", [(1, 1, 32, 8, 128, 1), (24, 24, 32, 8, 128, 1), (16, 16, 8, 8, 128, 1), (16, 1, 32, 8, 128, 16),
                                                 (600, 1, 4, 2, 64, 600), (37, 5, 12, 12, 64, 9), (512, 512, 8, 1, 80, 1), (513, 513, 8, 1, 80, 1)])
def test_size_does_not_fall_with_the_longest_length(Tq, B, Hq, Hkv, D, max_q):
    size = binding.load_library().nm_attention_workspace_bytes
    sizes = [size(Tq, B, Hq, Hkv, D, max_q, n) for n in CAPACITIES]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))


@pytest.mark.gpu
@pytest.mark.parametrize("B,Lq,Hq,Hkv,D,room,capacity,used", [
    (16, 1, 8, 8, 128, 12288, 16384, 12288), (1, 1, 8, 8, 128, 12288, 13000, 13000), (16, 1, 8, 8, 128, 768, 13000, 13000),
    (1, 16, 32, 8, 128, 98304, 120000, 120000), (3, 2, 4, 2, 64, 5000, 131072, 4100)])
def test_named_size_does(B, Lq, Hq, Hkv, D, room, capacity, used):
    import paper_2409_09708_amd as nm
    g = torch.Generator("cuda").manual_seed(B + room)
    Q = torch.randn(B * Lq, Hq, D, generator=g, device="cuda").to(torch.bfloat16)
    K, V = (torch.randn(B * room, Hkv, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    need = binding.load_library().nm_attention_workspace_bytes(B * Lq, B, Hq, Hkv, D, Lq, capacity)
    ws = torch.zeros(max(need, 256), dtype=torch.uint8, device="cuda")
    at = dict(offsets_q=torch.arange(B + 1, dtype=torch.int32, device="cuda") * Lq, max_q=Lq, max_k=used,
              offsets_k=torch.arange(B + 1, dtype=torch.int32, device="cuda") * room)
    assert torch.equal(nm.nm_attention(Q, K, V, True, workspace=ws, **at), nm.nm_attention(Q, K, V, True, **at))
    O = torch.empty_like(Q)
    d = binding._attention_desc(Q, K, V, True, None, at["offsets_q"], at["offsets_k"], None, Lq, used)
    d.O = binding._heads(O, "O", Q.shape)
    status = binding.load_library().nm_attention(d, ws.data_ptr(), need, binding._stream_handle(None))
    assert status == binding.NM_OK
    assert torch.equal(O, nm.nm_attention(Q, K, V, True, **at))
