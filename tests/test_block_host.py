"""Refusals and sizes of the operators between the linear layers: reported on the host, before anything is launched."""
import ctypes

import pytest
import torch

from paper_2409_09708_amd import binding

FAKE = 0x1000  # a non-NULL, well aligned address that is never dereferenced on the error paths
OK, NULL, SHAPE, ALIGN, DTYPE, WORKSPACE = 0, 1, 2, 4, 5, 6
F32, BF16, I32 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def norm(lib, **kw):
    a = dict(X=FAKE, ldx=64, xt=BF16, R=None, ldr=0, T=8, C=64, w=FAKE, b=FAKE, eps=1e-5, Y=FAKE, ldy=64, yt=BF16, S=None,
             lds=0, stats=None, stream=None)
    a.update(kw)
    return lib.nm_layer_norm(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(X=None), NULL), (dict(Y=None), NULL), (dict(T=0), SHAPE), (dict(C=0), SHAPE), (dict(T=-1), SHAPE), (dict(T=2 ** 31 + 1), SHAPE),
    (dict(C=2 ** 24 + 1, ldx=2 ** 25, ldy=2 ** 25), SHAPE), (dict(T=2 ** 31, C=1024, ldx=1024, ldy=1024), SHAPE), (dict(ldx=63), SHAPE),
    (dict(ldy=63), SHAPE), (dict(R=FAKE, ldr=63), SHAPE), (dict(R=FAKE, ldr=64, S=FAKE, lds=63), SHAPE), (dict(eps=-1.0), SHAPE),
    (dict(eps=float("nan")), SHAPE), (dict(xt=I32), DTYPE), (dict(yt=7), DTYPE), (dict(X=FAKE + 1), ALIGN), (dict(xt=F32, X=FAKE + 2), ALIGN),
    (dict(yt=F32, Y=FAKE + 2), ALIGN), (dict(w=FAKE + 2), ALIGN), (dict(b=FAKE + 1), ALIGN), (dict(stats=FAKE + 4), ALIGN),
    (dict(R=FAKE + 1, ldr=64), ALIGN)])
def test_layer_norm_refusals(lib, kw, status):
    assert norm(lib, **kw) == status


def norm_backward(lib, **kw):
    a = dict(dY=FAKE, lddy=64, yt=BF16, S=FAKE, lds=64, st=BF16, stats=FAKE, w=FAKE, dS=None, ldds=0, T=8, C=64, dX=FAKE, lddx=64,
             xt=F32, dw=FAKE, db=FAKE, ws=FAKE, bytes=1 << 30, stream=None)
    a.update(kw)
    return lib.nm_layer_norm_backward(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(dY=None), NULL), (dict(S=None), NULL), (dict(stats=None), NULL), (dict(dX=None), NULL), (dict(dw=None), NULL), (dict(db=None), NULL),
    (dict(T=0), SHAPE), (dict(C=-4), SHAPE), (dict(lddy=63), SHAPE), (dict(lds=63), SHAPE), (dict(lddx=63), SHAPE),
    (dict(dS=FAKE, ldds=1), SHAPE), (dict(yt=2), DTYPE), (dict(st=3), DTYPE), (dict(xt=-1), DTYPE), (dict(stats=FAKE + 4), ALIGN),
    (dict(dX=FAKE + 2), ALIGN), (dict(dw=FAKE + 2), ALIGN), (dict(T=999, ws=None), WORKSPACE), (dict(T=999, bytes=16), WORKSPACE),
    (dict(T=999, ws=FAKE + 64), WORKSPACE)])
def test_layer_norm_backward_refusals(lib, kw, status):
    assert norm_backward(lib, **kw) == status


def test_layer_norm_backward_workspace(lib):
    size = lib.nm_layer_norm_backward_workspace_bytes
    assert size(4, 768) == 0 and size(0, 768) == 0 and size(8, 0) == 0
    assert size(50432, 768) == size(200000, 768) > 0
    assert size(50432, 768) % (2 * 768 * 4) == 0


def rotary(lib, sections=(16, 16), **kw):
    a = dict(X=FAKE, xt=BF16, T=8, H=2, D=64, xk=128, xh=64, pos=FAKE, pf=0, freqs=FAKE, sections=binding._ints(sections), axes=len(sections),
             rotated=64, inter=0, inv=0, Y=FAKE, yt=BF16, yk=128, yh=64, stream=None)
    a.update(kw)
    return lib.nm_rotary(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(X=None), NULL), (dict(Y=None), NULL), (dict(pos=None), NULL), (dict(freqs=None), NULL), (dict(T=0), SHAPE), (dict(H=0), SHAPE),
    (dict(D=0), SHAPE), (dict(rotated=63), SHAPE), (dict(rotated=0), SHAPE), (dict(rotated=66), SHAPE), (dict(axes=0), SHAPE),
    (dict(sections=(4,) * 5), SHAPE), (dict(sections=(16, 15)), SHAPE), (dict(sections=(33, -1)), SHAPE), (dict(xk=-128), SHAPE),
    (dict(yk=127), SHAPE), (dict(yh=63), SHAPE), (dict(xt=2), DTYPE), (dict(yt=2), DTYPE), (dict(X=FAKE + 1), ALIGN), (dict(pos=FAKE + 2), ALIGN),
    (dict(freqs=FAKE + 2), ALIGN), (dict(yt=F32, Y=FAKE + 2), ALIGN)])
def test_rotary_refusals(lib, kw, status):
    assert rotary(lib, **kw) == status


def attention(lib, backward=False, ws=FAKE, bytes=1 << 40, **kw):
    d = binding.AttentionDesc()
    for name in ("Q", "O", "dO", "dQ"):
        setattr(d, name, binding.Heads(FAKE, 4 * 64, 64))
    for name in ("K", "V", "dK", "dV"):
        setattr(d, name, binding.Heads(FAKE, 2 * 64, 64))
    d.lse = FAKE
    d.Tq = d.Tk = d.max_q = d.max_k = 100
    d.sequences, d.heads_q, d.heads_kv, d.head_size, d.scale = 1, 4, 2, 64, 0.125
    for k, v in kw.items():
        setattr(d, k, v)
    return (lib.nm_attention_backward if backward else lib.nm_attention)(ctypes.byref(d), ws, bytes, None)


H = binding.Heads


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(Q=H(None, 256, 64)), NULL), (dict(K=H(None, 128, 64)), NULL), (dict(V=H(None, 128, 64)), NULL), (dict(O=H(None, 256, 64)), NULL),
    (dict(sequences=2), NULL), (dict(Tq=0), SHAPE), (dict(Tk=-1), SHAPE), (dict(Tq=2 ** 30 + 1), SHAPE), (dict(Tk=2 ** 30 + 1), SHAPE),
    (dict(sequences=0), SHAPE), (dict(sequences=65536, offsets_q=FAKE, offsets_k=FAKE), SHAPE), (dict(heads_q=5), SHAPE), (dict(heads_kv=0), SHAPE),
    (dict(sequences=60000, heads_q=32, offsets_q=FAKE, offsets_k=FAKE), SHAPE), (dict(head_size=0), SHAPE), (dict(head_size=129), SHAPE),
    (dict(max_q=-1), SHAPE), (dict(scale=0.0), SHAPE), (dict(scale=-1.0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE),
    (dict(Q=H(FAKE, -256, 64)), SHAPE), (dict(Q=H(FAKE + 1, 256, 64)), ALIGN), (dict(lse=FAKE + 2), ALIGN),
    (dict(sequences=3, offsets_q=FAKE + 2, offsets_k=FAKE), ALIGN), (dict(lengths_k=FAKE + 1), ALIGN)])
def test_attention_refusals(lib, backward, kw, status):
    assert attention(lib, backward, **kw) == status


def test_attention_refuses_outputs_that_overlap(lib):
    assert attention(lib, O=H(FAKE, 255, 64)) == SHAPE
    assert attention(lib, O=H(FAKE, 256, 63)) == SHAPE
    assert attention(lib, O=H(FAKE, 64, 64 * 99)) == SHAPE
    assert attention(lib, True, dK=H(FAKE, 0, 64)) == SHAPE
    assert attention(lib, True, dV=H(FAKE, 128, 0)) == SHAPE
    assert attention(lib, True, dQ=H(None, 256, 64)) == NULL
    assert attention(lib, True, lse=None) == NULL
    assert lib.nm_attention(None, None, 0, None) == NULL and lib.nm_attention_backward(None, None, 0, None) == NULL


def test_attention_workspace(lib):
    size = lib.nm_attention_workspace_bytes
    assert size(50432, 256, 12, 12, 64, 197, 197) == 0            # whole prompts: none
    assert size(1, 1, 32, 8, 128, 1, 200) == 0                    # a short cache: one chunk
    need = size(1, 1, 32, 8, 128, 1, 16384)
    assert need > 0
    assert attention(lib, ws=None, bytes=0, Tq=1, Tk=16384, max_q=1, max_k=16384, heads_q=32, heads_kv=8, Q=H(FAKE, 4096, 128), O=H(FAKE, 4096, 128),
                     K=H(FAKE, 1024, 128), V=H(FAKE, 1024, 128), head_size=128) == WORKSPACE
    assert size(0, 1, 32, 8, 128, 1, 16384) == 0 and size(1, 1, 32, 7, 128, 1, 16384) == 0
    back = lib.nm_attention_backward_workspace_bytes
    assert back(100, 100, 1, 4, 2, 64, 100, 100, 0) == 1792 and back(0, 100, 1, 4, 2, 64, 100, 100, 0) == 0
    assert back(8192, 8192, 1, 16, 4, 128, 8192, 8192, 1) > 8192 * 16 * 4
    assert back(65536, 65536, 65535, 1, 1, 64, 8192, 0, 0) == 65536 * 4   # no keys: nothing to cut
    assert attention(lib, True, ws=None, bytes=0) == WORKSPACE


def test_python_calls_name_what_is_wrong():
    import paper_2409_09708_amd as nm
    x = torch.zeros(4, 8)
    for call in (lambda: nm.nm_layer_norm(x), lambda: nm.nm_layer_norm_backward(x, x, x), lambda: nm.nm_rotary(x, x, x),
                 lambda: nm.nm_attention(x, x, x), lambda: nm.nm_attention_backward(x, x, x, x, x, x)):
        with pytest.raises(ValueError, match="device tensor"):
            call()
