"""Rows of one value: nothing is left of them but the bias, also where their 32-bit sum is rounded many times."""
import pytest
import torch

import block_reference as ref

pytestmark = pytest.mark.gpu
VALUES = [0.1, -1000.1, 10000.1, 33333.3, 3.0, -1e-3, 123456.7]
WIDTHS = [1, 3, 100, 128, 136, 500, 512, 768, 1000, 1024, 2000, 2048, 4000, 5003, 6144, 8000, 8192, 9000]
# roundings on the way of an element into a sum: at most 40 elements of a lane, the tree over the lanes, the quotient
DEPTH = 64


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("residual", [False, True])
def test_constant_rows(C, residual):
    import paper_2409_09708_amd as nm
    eps = 1e-6
    values = torch.tensor(VALUES, dtype=torch.float32, device="cuda")
    X = values[:, None].expand(-1, C).contiguous()
    R = (values.flip(0) * 0.7)[:, None].expand(-1, C).contiguous() if residual else None
    total = values if R is None else values + R[:, 0]  # (the 32-bit sum is the row that is normalised)
    size = total.double().abs()
    off = DEPTH * ref.U32 * size  # of a mean from one sum of the row
    y = nm.nm_layer_norm(X, eps=eps, residual=R, train=True)
    # a mean that is corrected by the mean difference to it is off by as small a part of that difference
    assert bool((y[0].double().abs() <= (1.01 * DEPTH * ref.U32 * off / eps ** 0.5)[:, None]).all()), y[0].abs().amax(1)
    assert torch.equal(y[-1][:, 0], total)
    least = 1 / (eps + 4 * DEPTH * ref.U32 * off ** 2).sqrt()
    rstd = y[-1][:, 1].double()
    assert bool((rstd >= least * (1 - 8 * ref.U32)).all()) and bool((rstd <= eps ** -0.5 * (1 + 8 * ref.U32)).all())


def test_nothing_of_them_reaches_the_gradients():
    import paper_2409_09708_amd as nm
    X = torch.tensor(VALUES, dtype=torch.float32, device="cuda")[:, None].expand(-1, 768).contiguous()
    stats = nm.nm_layer_norm(X, eps=1e-6, train=True)[1]
    dX, dw, db = nm.nm_layer_norm_backward(torch.ones_like(X), X, stats)
    # (the mean of ones is rounded twice: the width's inverse, and its product with their sum)
    assert float(dw.abs().max()) == 0 and float(dX.abs().max()) <= 1.01e3 * 2 * ref.U32
    assert torch.equal(db, torch.full_like(db, len(VALUES)))
