"""Layer norm and its gradients at the ends of the range that the header states."""
import pytest
import torch

from paper_2302_02390_amd import binding as qb
from train_util import DEV, matrix, near, norm, norm_grad

pytestmark = pytest.mark.gpu


def _both(x, dy, eps):
    rows, n = x.shape
    y, dx, stats = torch.empty_like(x, device=DEV), torch.empty_like(x, device=DEV), torch.empty((rows, 2), device=DEV)
    dw, db = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    qb.qsdp_layer_norm(x.to(DEV), None, None, eps, y, stats)
    qb.qsdp_layer_norm_backward(x.to(DEV), None, stats, dy.to(DEV), dx, dw, db)
    return y, dx, dw, db


@pytest.mark.parametrize("n", [1001, 1024, 5000, 20000, 40000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("std,eps", [(2.0 ** 55, 1e-5), (2.0 ** -62, 0.0), (2.0 ** 55, 0.0), (1.0, 2.0 ** 40)])
def test_large_and_small_rows(n, dtype, std, eps):
    """40000 squares of 2^110 are below 2^126; the mean square of 2^-124 is a normal number."""
    x, dy = matrix(6, n, dtype, seed=n, std=std), matrix(6, n, dtype, seed=n + 1)
    want, _, _, off, _, _ = norm(x, None, None, eps)
    grads, offs = norm_grad(x, None, dy, eps)
    y, dx, dw, db = _both(x, dy, eps)
    assert near(y, want, off)
    for name, t in (("dx", dx), ("dw", dw), ("db", db)):
        assert near(t, grads[name], offs[name]), name


@pytest.mark.parametrize("n", [5, 1001, 1024, 5001, 20001])
def test_constant_rows_far_from_zero(n):
    """Sums of up to 2^15 times a power of two are exact, so h is 0: the gradients are those of a row of zeros, also where a team's last
    lanes have no elements and |mean| rstd = 2^108."""
    x, dy = torch.full((3, n), 2.0 ** 100), matrix(3, n, torch.float32, seed=n)
    x[1] = -2.0 ** 100
    x[2] = 0.0
    grads, offs = norm_grad(torch.zeros_like(x), None, dy, 2.0 ** -16)
    y, dx, dw, db = _both(x, dy, 2.0 ** -16)
    assert bool((y == 0).all()) and bool((dw == 0).all())
    assert near(dx, grads["dx"], offs["dx"]) and near(db, grads["db"], offs["db"])
