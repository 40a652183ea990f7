"""Layer norm and its backward pass against their definitions in 64 bits."""
import pytest
import torch

import block_reference as ref

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def rows(g, T, C, dtype, pad=0, at=0, scale=1.0):
    t = torch.randn(T, C + pad + at, generator=g, device="cuda").mul_(scale).to(dtype)
    return t[:, at:at + C]


def setup(seed):
    g = torch.Generator("cuda")
    g.manual_seed(seed)
    return g


# widths on both sides of every form that a row is held in, rows from one to more than the blocks that walk them
SHAPES = [(1, 768, 0, 0), (3, 1, 0, 0), (5, 8, 0, 0), (17, 128, 0, 0), (33, 136, 8, 0), (2049, 512, 0, 0), (130, 520, 0, 0),
          (67, 1024, 8, 8), (9, 1032, 0, 0), (7, 2048, 0, 0), (6, 2056, 0, 0), (5, 4096, 0, 0), (4, 4104, 0, 0), (3, 8192, 0, 0),
          (2, 8200, 0, 0), (700, 9001, 3, 0), (19, 255, 2, 1), (21, 257, 1, 0), (520, 1000, 0, 1), (5, 1025, 3, 0),
          (3, 4097, 0, 0), (5, 5003, 5, 0), (2, 8191, 0, 0)]


@pytest.mark.parametrize("T,C,pad,at", SHAPES)
@pytest.mark.parametrize("x_type,y_type", [(BF16, BF16), (F32, BF16), (F32, F32), (BF16, F32)])
def test_forward(T, C, pad, at, x_type, y_type):
    import paper_2409_09708_amd as nm
    g = setup(T * 7919 + C)
    X, R = rows(g, T, C, x_type, pad, at), rows(g, T, C, x_type, pad, at, 2.0)
    w, b = (torch.randn(C, generator=g, device="cuda") for _ in range(2))
    for residual, affine in ((None, True), (R, True), (R, False)):
        wd, bd = (w, b) if affine else (None, None)
        got = nm.nm_layer_norm(X, wd, bd, 1e-5, residual=residual, train=True, out_dtype=y_type)
        exact = X.double() + (0 if residual is None else residual.double())
        one, zero = torch.ones(C, device="cuda").double(), torch.zeros(C, device="cuda").double()
        y, bound, mean, rstd, d_mean, d_rstd = ref.norm(exact, w.double() if affine else one, b.double() if affine else zero, 1e-5, y_type)
        extra = ref.U32 * exact.abs() * rstd * (w.abs().double() if affine else one) * 2  # the 32-bit sum x + r
        assert got[0].dtype == y_type
        ref.close(got[0], y, bound + extra, "y")
        stats = got[-1]
        ref.close(stats[:, :1], mean, d_mean + 2 * ref.U32 * exact.abs().mean(1, keepdim=True), "mean")
        ref.close(stats[:, 1:], rstd, rstd * (d_rstd + 8 * ref.U32), "rstd")
        if residual is not None:
            assert got[1].dtype == x_type
            ref.close(got[1], exact, (ref.rounding(x_type) + ref.U32) * exact.abs(), "sum")
        plain = nm.nm_layer_norm(X, wd, bd, 1e-5, residual=residual, out_dtype=y_type)
        assert torch.equal(plain if residual is None else plain[0], got[0])


@pytest.mark.parametrize("T,C,pad,at", SHAPES)
@pytest.mark.parametrize("y_type,x_type,out_type", [(BF16, BF16, BF16), (F32, F32, F32), (BF16, F32, F32), (F32, BF16, BF16)])
def test_backward(T, C, pad, at, y_type, x_type, out_type):
    import paper_2409_09708_amd as nm
    g = setup(T * 31 + C)
    X, dY, dS = rows(g, T, C, x_type, pad, at), rows(g, T, C, y_type, pad, at), rows(g, T, C, y_type, pad, at)
    w = torch.randn(C, generator=g, device="cuda")
    stats = nm.nm_layer_norm(X, train=True)[1]
    mean, rstd = stats.double().split(1, 1)
    for affine, extra in ((True, dS), (False, None)):
        got = nm.nm_layer_norm_backward(dY, X, stats, w if affine else None, dS=extra, out_dtype=out_type)
        want = ref.norm_grad(dY.double(), X.double(), mean, rstd, w.double() if affine else torch.ones_like(w).double(),
                             extra if extra is None else extra.double(), out_type)
        for name, t, (v, bound) in zip(("dX", "dweight", "dbias"), got, want):
            ref.close(t, v, bound, name)
        again = nm.nm_layer_norm_backward(dY, X, stats, w if affine else None, dS=extra, out_dtype=out_type)
        assert all(torch.equal(a, b) for a, b in zip(got, again))
        alone = nm.nm_layer_norm_backward(dY, X, stats, w if affine else None, dS=extra, out_dtype=out_type, params=False)
        assert torch.equal(alone[0], got[0]) and alone[1] is None and alone[2] is None


def test_gradient_is_that_of_differences():
    """Along a random direction, against differences of the definition in 64 bits."""
    import paper_2409_09708_amd as nm
    g = setup(5)
    T, C = 13, 200
    X, dY = rows(g, T, C, F32), rows(g, T, C, F32)
    w, b, way = torch.randn(C, generator=g, device="cuda"), torch.randn(C, generator=g, device="cuda"), rows(g, T, C, F32).double()
    stats = nm.nm_layer_norm(X, w, b, 1e-5, train=True)[1]
    dX, dw, db = nm.nm_layer_norm_backward(dY, X, stats, w)

    def loss(x, w, b):
        m = x.mean(1, keepdim=True)
        return (((x - m) * ((x - m).square().mean(1, keepdim=True) + 1e-5).rsqrt() * w + b) * dY.double()).sum()

    h, x, wd, bd = 1e-5, X.double(), w.double(), b.double()
    for got, diff, size in (
            ((dX.double() * way).sum(), (loss(x + h * way, wd, bd) - loss(x - h * way, wd, bd)) / (2 * h), (dX.double() * way).abs().sum()),
            ((dw.double() * way[0]).sum(), (loss(x, wd + h * way[0], bd) - loss(x, wd - h * way[0], bd)) / (2 * h), (dw.double() * way[0]).abs().sum()),
            ((db.double() * way[0]).sum(), (loss(x, wd, bd + h * way[0]) - loss(x, wd, bd - h * way[0])) / (2 * h), (db.double() * way[0]).abs().sum())):
        assert abs(float(got - diff)) <= (C + 64) * ref.U32 * float(size) * 4 + 1e-7 * float(size)


def test_large_offset_keeps_the_variance():
    """Rows around 1000 with a spread of 1: a variance from sums of squares would lose it."""
    import paper_2409_09708_amd as nm
    g = setup(9)
    X = rows(g, 64, 768, F32) + 1000
    y = nm.nm_layer_norm(X, eps=0.0).double()
    x = X.double()
    want, bound, *_ = ref.norm(x, torch.ones(768, device="cuda").double(), torch.zeros(768, device="cuda").double(), 0.0, F32)
    ref.close(y, want, bound)
    assert float((y - want).abs().max()) < 1e-2


def test_rows_that_are_constant_or_not_finite():
    import paper_2409_09708_amd as nm
    X = torch.full((4, 768), 3.0, device="cuda")
    X[1, 5], X[2, 7] = float("inf"), float("nan")
    y = nm.nm_layer_norm(X, eps=1e-5)
    assert float(y[0].abs().max()) == 0 and float(y[3].abs().max()) == 0
    assert bool(torch.isnan(y[1]).any()) and bool(torch.isnan(y[2]).all())


def test_residual_stream_in_place_and_on_another_stream():
    import paper_2409_09708_amd as nm
    g = setup(11)
    for C in (768, 9000, 131):
        X, R = rows(g, 300, C, F32), rows(g, 300, C, F32)
        want = nm.nm_layer_norm(X, residual=R)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            kept = R.clone()
            got = nm.nm_layer_norm(X, residual=kept, sum_out=kept)
        stream.synchronize()
        assert got[1] is kept and torch.equal(kept, want[1]) and torch.equal(got[0], want[0])


def test_captured():
    import paper_2409_09708_amd as nm
    g = setup(13)
    X, dY, w = rows(g, 1000, 768, BF16), rows(g, 1000, 768, BF16), torch.randn(768, generator=g, device="cuda")
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")

    def step():
        y, stats = nm.nm_layer_norm(X, w, train=True, out_dtype=BF16)
        return (y, *nm.nm_layer_norm_backward(dY, X, stats, w, out_dtype=BF16, workspace=ws))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for n in range(3):
        X.copy_(rows(g, 1000, 768, BF16))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        assert all(torch.equal(a, b) for a, b in zip(got, step()))
