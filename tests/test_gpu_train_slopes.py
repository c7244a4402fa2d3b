"""Gradients of layer norm and of products in blocks against differences along the gradients themselves, where a slope is a norm and
its bound a small part of it: a gradient that is missing, halved, of the wrong sign or wrong in one part fails."""
import pytest
import torch

from paper_2302_02390_amd import binding as qb
from train_util import DEV, DTYPES, blocks, held, matrix, norm, norm_grad, product

pytestmark = pytest.mark.gpu

U64 = 2.0 ** -53


def _directions(gradient, parts):
    """The gradient in 64 bits over its norm, whole and cut to each of `parts` runs of its columns."""
    yield gradient / gradient.norm()
    for columns in torch.arange(gradient.shape[-1]).chunk(parts):
        d = torch.zeros_like(gradient)
        d[..., columns] = gradient[..., columns]
        yield d / d.norm()


def check(value, at, got, gradient, off, step, size, bend, parts=3):
    """`value` is a function in 64 bits whose sums have terms of `size` in all, `off` what each element of `got` may be off and `bend`
    what a step may change of the slope, relative to it. A value is off by at most 256 roundings of its size: additions in pairs and the
    operations of a term."""
    for d in _directions(gradient, parts):
        slope = (value(at + step * d) - value(at - step * d)) / (2 * step)
        bound = float((off * d.abs()).sum()) + 256 * U64 * size / step + bend * abs(slope)
        assert bound < 0.02 * abs(slope)
        along = float((got.detach().cpu().double() * d).sum())
        assert abs(along - slope) <= bound, (along, slope, bound)


@pytest.mark.parametrize("rows,n,x,y,w", [(12, 96, "f32", "f32", "f32"), (12, 2048, "f32", "f32", "f32"), (7, 1001, "f32", "bf16", "f32"),
                                          (40, 4100, "bf16", "bf16", "bf16"), (5, 9000, "f16", "f16", "f16"), (3, 20000, "bf16", "bf16", "f32")])
def test_layer_norm(rows, n, x, y, w):
    xs, dy = matrix(rows, n, DTYPES[x], seed=21, std=1.5, mean=0.7), matrix(rows, n, DTYPES[y], seed=24, std=0.5)
    weight, bias = matrix(1, n, DTYPES[w], seed=22, std=0.2, mean=1.0)[0], matrix(1, n, DTYPES[w], seed=23, std=0.3)[0]
    xg, wg, stats = xs.to(DEV), weight.to(DEV), torch.empty((rows, 2), device=DEV)
    qb.qsdp_layer_norm(xg, wg, bias.to(DEV), 1e-5, torch.empty((rows, n), dtype=DTYPES[y], device=DEV), stats)
    dx, dw, db = torch.empty_like(xg), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    qb.qsdp_layer_norm_backward(xg, wg, stats, dy.to(DEV), dx, dw, db)
    grads, offs = norm_grad(xs, weight, dy, 1e-5)
    offs["dx"] = offs["dx"] + grads["dx"].abs() * torch.finfo(xs.dtype).eps / 2 + torch.finfo(xs.dtype).smallest_normal * torch.finfo(xs.dtype).eps
    dyd, f = dy.double(), lambda *args: float((norm(*args, 1e-5)[0] * dyd).sum())
    size = float(((norm(xs, weight, bias, 1e-5)[0].abs() + 2 * weight.double().abs()) * dyd.abs()).sum())
    # a step of 1e-4 turns a row, of norm sqrt(n) at least, by 1e-5 at most: the slope changes by its square, a few times over
    check(lambda v: f(v, weight, bias), xs.double(), dx, grads["dx"], offs["dx"], 1e-4, size, 1e-8)
    check(lambda v: f(xs, v, bias), weight.double(), dw, grads["dw"], offs["dw"], 1e-2, size, 0.0)
    check(lambda v: f(xs, weight, v), bias.double(), db, grads["db"], offs["db"], 1e-2, size, 0.0)


@pytest.mark.parametrize("m,n,k,dtype", [(200, 260, 300, "bf16"), (333, 1000, 520, "f16"), (130, 500, 1100, "bf16")])
def test_product(m, n, k, dtype):
    """The product of what the codes stand for is linear in either side."""
    x, w, dy = (matrix(r, c, DTYPES[dtype], seed=i, std=s) for i, (r, c, s) in enumerate(((m, k, 1.0), (n, k, 0.05), (m, n, 0.01))))
    xq, dq, wq = qb.alloc_blocks(m, k, False, DEV), qb.alloc_blocks(m, n, False, DEV), qb.alloc_blocks(n, k, True, DEV)
    for t, square, to in ((x, False, xq), (dy, False, dq), (w, True, wq)):
        qb.qsdp_quantize_blocks(t.to(DEV), square, *to)
    dx, dw = torch.empty((m, k), dtype=DTYPES[dtype], device=DEV), torch.empty((n, k), device=DEV)
    qb.qsdp_matmul_blocks(*dq[:2], *wq[2:], n, None, dx)
    qb.qsdp_matmul_blocks(*dq[2:], *xq[2:], m, None, dw)
    hx, hw, hd = held(*blocks(x, 1, 128), 1, 128), held(*blocks(w, 128, 128), 128, 128), held(*blocks(dy, 1, 128), 1, 128)
    want, off = product(hd, hw.t().contiguous(), False)
    off = off + want.abs() * torch.finfo(dx.dtype).eps / 2 + torch.finfo(dx.dtype).smallest_normal * torch.finfo(dx.dtype).eps
    size = float((hx.abs() @ hw.abs().t() * hd.abs()).sum())
    check(lambda v: float((v @ hw.t() * hd).sum()), hx, dx, want, off, 1.0, size, 0.0)
    # the weight's gradient rounds dy and x along their columns: its own held values
    ht, hdt = held(*blocks(x.t(), 1, 128), 1, 128), held(*blocks(dy.t(), 1, 128), 1, 128)
    want, off = product(hdt, ht, True)
    size = float((ht.t().abs() @ hw.abs().t() * hdt.t().abs()).sum())
    check(lambda v: float((ht.t() @ v.t() * hdt.t()).sum()), hw, dw, want, off, 1.0, size, 0.0)
