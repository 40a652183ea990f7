"""Refusals and sizes of the norm of heads and of a cache in pages: reported on the host, before anything is launched."""
import ctypes

import pytest
import torch

from paper_2409_09708_amd import binding

FAKE = 0x1000  # a non-NULL, well aligned address that is never dereferenced on the error paths
OK, NULL, SHAPE, ALIGN, DTYPE, WORKSPACE = 0, 1, 2, 4, 5, 6
F32, BF16, I32, E4M3 = 0, 1, 2, 3
TH, H = binding.TypedHeads, binding.Heads


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def head_norm(lib, backward=False, ws=FAKE, bytes=1 << 40, sections=(16, 16), **kw):
    d = binding.HeadNormDesc()
    d.X, d.Y, d.dY = (TH(FAKE, 256, 64, BF16, 0) for _ in range(3))
    d.weight = d.positions = d.freqs = FAKE
    if backward:
        d.dweight = FAKE
    d.T, d.H, d.heads, d.D, d.rotated, d.axes, d.eps = 5000, 4, 3, 64, 64, len(sections), 1e-6
    kept = binding._ints(sections)
    d.sections = ctypes.addressof(kept)
    for k, v in kw.items():
        setattr(d, k, v)
    return lib.nm_head_norm_backward(ctypes.byref(d), ws, bytes, None) if backward else lib.nm_head_norm(ctypes.byref(d), None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(X=TH(None, 256, 64, BF16, 0)), NULL), (dict(Y=TH(None, 256, 64, BF16, 0)), NULL), (dict(freqs=None), NULL),
    (dict(T=0), SHAPE), (dict(T=2 ** 31 + 1), SHAPE), (dict(H=0), SHAPE), (dict(D=0), SHAPE), (dict(D=513), SHAPE),
    (dict(H=2 ** 15, D=512, heads=1), SHAPE), (dict(heads=0), SHAPE), (dict(heads=5), SHAPE), (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE),
    (dict(rotated=66), SHAPE), (dict(rotated=63), SHAPE), (dict(rotated=0), SHAPE), (dict(axes=0), SHAPE), (dict(axes=5), SHAPE),
    (dict(sections=(16, 15)), SHAPE), (dict(sections=(33, -1)), SHAPE), (dict(X=TH(FAKE, -256, 64, BF16, 0)), SHAPE),
    (dict(Y=TH(FAKE, 255, 64, BF16, 0)), SHAPE), (dict(X=TH(FAKE, 2 ** 31, 64, BF16, 0)), SHAPE), (dict(Y=TH(FAKE, 256, 63, BF16, 0)), SHAPE), (dict(X=TH(FAKE, 256, 64, I32, 0)), DTYPE),
    (dict(Y=TH(FAKE, 256, 64, E4M3, 0)), DTYPE), (dict(X=TH(FAKE + 1, 256, 64, BF16, 0)), ALIGN), (dict(Y=TH(FAKE + 2, 256, 64, F32, 0)), ALIGN),
    (dict(weight=FAKE + 2), ALIGN), (dict(positions=FAKE + 1), ALIGN), (dict(freqs=FAKE + 2), ALIGN)])
def test_head_norm_refusals(lib, backward, kw, status):
    assert head_norm(lib, backward, **kw) == status


def test_head_norm_backward_refusals(lib):
    assert lib.nm_head_norm(None, None) == NULL and lib.nm_head_norm_backward(None, None, 0, None) == NULL
    assert head_norm(lib, True, dY=TH(None, 256, 64, BF16, 0)) == NULL
    assert head_norm(lib, True, weight=None) == NULL  # (a gradient of what is not there)
    assert head_norm(lib, True, dY=TH(FAKE, 256, -64, BF16, 0)) == SHAPE
    assert head_norm(lib, True, dY=TH(FAKE, 256, 64, 7, 0)) == DTYPE
    assert head_norm(lib, True, dY=TH(FAKE + 1, 256, 64, BF16, 0)) == ALIGN
    assert head_norm(lib, True, dweight=FAKE + 2) == ALIGN
    assert head_norm(lib, True, ws=None) == WORKSPACE
    assert head_norm(lib, True, bytes=64) == WORKSPACE
    assert head_norm(lib, True, ws=FAKE + 64) == WORKSPACE


def test_head_norm_workspace(lib):
    size = lib.nm_head_norm_backward_workspace_bytes
    assert size(1, 4, 4, 64, 64) == 256 and size(0, 4, 3, 64, 64) == 0 and size(9, 4, 5, 64, 64) == 0 and size(9, 4, 3, 64, 65) == 0
    assert size(9, 4, 3, 513, 0) == 0 and size(9, 4, 3, 64, 66) == 0 and size(9, 0, 0, 64, 0) == 0
    many = size(10 ** 6, 4, 3, 64, 64)
    assert many > 0 and many % (64 * 4) == 0 and size(10 ** 7, 4, 3, 64, 64) <= 2 * many  # (a row of sums to each of so many blocks)


def pages(codes=True, **kw):
    p = binding.Pages()
    p.K = p.V = p.table = p.lengths = FAKE
    p.page, p.token, p.head = 2 * 16 * 64, 64, 16 * 64
    p.scale_page, p.scale_token, p.scale_head = 32, 1, 16
    if codes:
        p.K_scales = p.V_scales = FAKE
    p.pages, p.page_size, p.table_width, p.sequences, p.heads, p.head_size, p.dtype = 100, 16, 8, 3, 2, 64, E4M3 if codes else BF16
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def write(lib, p, K=H(FAKE, 128, 64), V=H(FAKE, 128, 64), offsets=FAKE, T=6):
    return lib.nm_cache_write(ctypes.byref(p), K and ctypes.byref(K), V and ctypes.byref(V), offsets, T, None)


def read(lib, p, K=H(FAKE, 128, 64), V=H(FAKE, 128, 64), offsets=FAKE, T=6, first=None):
    return lib.nm_cache_read(ctypes.byref(p), K and ctypes.byref(K), V and ctypes.byref(V), offsets, first, T, None)


def attend(lib, p, ws=FAKE, bytes=1 << 40, **kw):
    d = binding.PagedDesc()
    d.pages = p
    d.Q, d.O = H(FAKE, 256, 64), H(FAKE, 256, 64)
    d.lse = d.offsets_q = FAKE
    d.Tq, d.max_q, d.max_k, d.heads_q, d.scale = 6, 3, 100, 4, 0.125
    for k, v in kw.items():
        setattr(d, k, v)
    return lib.nm_attention_paged(ctypes.byref(d), ws, bytes, None)


PAGES_REFUSED = [
    (dict(K=None), NULL), (dict(V=None), NULL), (dict(table=None), NULL), (dict(lengths=None), NULL), (dict(K_scales=None), NULL),
    (dict(V_scales=None), NULL), (dict(dtype=F32), DTYPE), (dict(dtype=I32), DTYPE), (dict(dtype=4), DTYPE), (dict(pages=0), SHAPE),
    (dict(pages=2 ** 31), SHAPE), (dict(page_size=0), SHAPE), (dict(page_size=2 ** 20 + 1), SHAPE), (dict(table_width=0), SHAPE),
    (dict(table_width=2 ** 26 + 1), SHAPE), (dict(sequences=0), SHAPE), (dict(sequences=65536), SHAPE), (dict(heads=0), SHAPE),
    (dict(sequences=60000, heads=32), SHAPE), (dict(head_size=0), SHAPE), (dict(head_size=129), SHAPE), (dict(page=-1), SHAPE), (dict(head=-64), SHAPE),
    (dict(scale_token=-1), SHAPE), (dict(page=2 ** 41), SHAPE), (dict(table=FAKE + 2), ALIGN), (dict(lengths=FAKE + 1), ALIGN)]


@pytest.mark.parametrize("call", [write, read, attend])
@pytest.mark.parametrize("kw,status", PAGES_REFUSED)
def test_pages_refusals(lib, call, kw, status):
    assert call(lib, pages(**kw)) == status


@pytest.mark.parametrize("call", [write, read])
def test_cache_refusals(lib, call):
    assert lib.nm_cache_write(None, None, None, None, 1, None) == NULL and lib.nm_cache_read(None, None, None, None, None, 1, None) == NULL
    p = pages()
    assert call(lib, p, K=None) == NULL and call(lib, p, V=None) == NULL and call(lib, p, K=H(None, 128, 64)) == NULL
    assert call(lib, p, T=0) == SHAPE and call(lib, p, T=2 ** 30 + 1) == SHAPE and call(lib, p, offsets=None, T=7) == SHAPE
    assert call(lib, p, K=H(FAKE, -128, 64)) == SHAPE and call(lib, p, V=H(FAKE + 1, 128, 64)) == ALIGN and call(lib, p, offsets=FAKE + 2) == ALIGN
    assert call(lib, pages(False, K=FAKE + 1)) == ALIGN


def test_what_is_written_must_not_overlap(lib):
    for kw in (dict(token=63), dict(head=15 * 64), dict(page=31 * 64), dict(token=0), dict(scale_token=0), dict(scale_head=15), dict(scale_page=31)):
        assert write(lib, pages(**kw)) == SHAPE, kw
    assert write(lib, pages(False, scale_token=0, K=None)) == NULL  # (no scales: their strides do not count)
    assert write(lib, pages(False, scale_token=0, K=FAKE + 1)) == ALIGN
    assert read(lib, pages(), K=H(FAKE, 127, 64)) == SHAPE and read(lib, pages(), V=H(FAKE, 128, 63)) == SHAPE
    assert read(lib, pages(), first=FAKE + 2) == ALIGN


def test_paged_refusals(lib):
    p = pages()
    assert lib.nm_attention_paged(None, None, 0, None) == NULL
    for kw, status in [
            (dict(Q=H(None, 256, 64)), NULL), (dict(O=H(None, 256, 64)), NULL), (dict(Tq=0), SHAPE), (dict(Tq=2 ** 30, heads_q=4), SHAPE),
            (dict(heads_q=5), SHAPE), (dict(heads_q=0), SHAPE), (dict(max_q=-1), SHAPE), (dict(max_k=-1), SHAPE), (dict(window=-1), SHAPE),
            (dict(sinks=-1), SHAPE), (dict(scale=0.0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE),
            (dict(offsets_q=None, Tq=7), SHAPE), (dict(Q=H(FAKE, -256, 64)), SHAPE), (dict(O=H(FAKE, 255, 64)), SHAPE), (dict(O=H(FAKE, 256, 63)), SHAPE),
            (dict(Q=H(FAKE + 1, 256, 64)), ALIGN), (dict(lse=FAKE + 2), ALIGN), (dict(offsets_q=FAKE + 2), ALIGN)]:
        assert attend(lib, p, **kw) == status, kw
    many = pages(table_width=4096)
    assert attend(lib, many, ws=None, max_k=60000) == WORKSPACE and attend(lib, many, bytes=256, max_k=60000) == WORKSPACE
    assert attend(lib, many, ws=FAKE + 64, max_k=60000) == WORKSPACE


def test_paged_workspace(lib):
    size = lib.nm_attention_paged_workspace_bytes
    assert size(0, 1, 4, 2, 64, 1) == 0 and size(4, 1, 5, 2, 64, 1) == 0 and size(4, 1, 4, 2, 129, 1) == 0 and size(2 ** 30, 1, 4, 2, 64, 1) == 0
    assert size(24, 24, 32, 8, 128, 1) > 0
    assert size(700, 700, 4, 4, 64, 1) == 0                 # units enough: none is cut
    assert size(8 * 2048, 8, 16, 4, 128, 2048) == 0         # chunks enough
    assert size(300, 1, 16, 4, 128, 300) > 0


def test_python_calls_name_what_is_wrong():
    import paper_2409_09708_amd as nm
    x = torch.zeros(4, 2, 8)
    p = torch.zeros(3, 4, 2, 8, dtype=torch.bfloat16)
    t = torch.zeros(1, 3, dtype=torch.int32)
    for call in (lambda: nm.nm_head_norm(x), lambda: nm.nm_head_norm_backward(x, x), lambda: nm.nm_cache_write(x, x, p, p, t, t),
                 lambda: nm.nm_cache_read(p, p, t, t, tokens=4), lambda: nm.nm_attention_paged(x, p, p, t, t)):
        with pytest.raises(ValueError, match="device tensor"):
            call()


def test_native_calls_decline_what_python_has_to_judge():
    calls = binding._native()
    x = torch.zeros(4, 2, 8, dtype=torch.bfloat16)
    p, t = torch.zeros(3, 4, 2, 8, dtype=torch.bfloat16), torch.zeros(1, 3, dtype=torch.int32)
    for done in (calls.head_norm(x, None, None, 1e-6, False, None, None, None, False, None, None, None),
                 calls.head_norm_backward(x, x, None, None, 1e-6, False, None, None, None, False, None, None, True, None, None),
                 calls.cache_write(x, x, p, p, t, t, None, None, None, None), calls.cache_read(p, p, t, t, None, 4, None, None, None, None, None),
                 calls.attention_paged(x, p, p, t, t, None, None, 0, 0, None, None, None, None, False, None, None, None),
                 calls.head_norm(x), calls.head_norm_backward(), calls.cache_write(x), calls.cache_read(), calls.attention_paged(x)):
        assert done is NotImplemented
