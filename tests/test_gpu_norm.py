"""Layer norm and its gradients against 64 bits."""
import pytest
import torch

from paper_2302_02390_amd import binding as qb
from train_util import DEV, DTYPES, matrix, near, norm, norm_grad, to_gpu

pytestmark = pytest.mark.gpu

# rows, n, pad of rows, elements behind an aligned address
SHAPES = [(1, 1, 0, 0), (3, 1, 2, 1), (1, 7, 0, 0), (5, 8, 0, 3), (17, 511, 3, 1), (9, 512, 0, 0), (70, 513, 1, 0), (33, 1024, 8, 5),
          (40, 1025, 0, 0), (1, 2048, 0, 0), (2049, 768, 0, 0), (1025, 2048, 0, 0), (1030, 1500, 4, 2), (21, 2049, 7, 1),
          (600, 4096, 0, 0), (13, 8192, 0, 0), (11, 8193, 1, 1), (6, 16384, 0, 0), (5, 16385, 3, 0), (7, 32768, 0, 0),
          (40, 32769, 5, 3), (3, 70000, 0, 0)]
FORMATS = [("f32", "f32", "f32"), ("f32", "bf16", "f32"), ("f32", "f16", "f16"), ("bf16", "bf16", "f32"), ("bf16", "bf16", "bf16"),
           ("f16", "f16", "f16")]


def _inputs(rows, n, pad, offset, x, y, w, seed=0):
    xs = matrix(rows, n, DTYPES[x], pad, offset, seed, 1.5, 0.7)
    weight = matrix(1, n, DTYPES[w], 0, 0, seed + 1, 0.2, 1.0)[0]
    bias = matrix(1, n, DTYPES[w], 0, 0, seed + 2, 0.3)[0]
    dy = matrix(rows, n, DTYPES[y], pad, offset, seed + 3, 0.5)
    return xs, weight, bias, dy


def _forward(x, w, b, eps, out, pad=3):
    rows, n = x.shape
    y = torch.full((rows, n + pad), 7.0, dtype=out, device=DEV)
    stats = torch.empty((rows, 2), device=DEV)
    qb.qsdp_layer_norm(x, w, b, eps, y[:, :n], stats)
    assert bool((y[:, n:] == 7.0).all())
    return y[:, :n], stats


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("formats", FORMATS)
def test_forward_and_gradients(shape, formats):
    if shape[1] > 16384 and formats not in (FORMATS[1], FORMATS[3]):
        pytest.skip("long rows: two formats")
    rows, n, pad, offset = shape
    x, w, b, dy = _inputs(*shape, *formats)
    xg, wg, bg, dyg = to_gpu(x), w.to(DEV), b.to(DEV), to_gpu(dy)
    eps = 1e-5
    want, stats, _, off, stats_off, _ = norm(x, w, b, eps)
    y, got = _forward(xg, wg, bg, eps, DTYPES[formats[1]])
    assert near(y, want, off)
    assert near(got, stats, stats_off)
    grads, offs = norm_grad(x, w, dy, eps)
    dx = torch.full((rows, n + pad), 5.0, dtype=x.dtype, device=DEV)
    dw, db = torch.full((n,), 3.0, device=DEV), torch.full((n,), 3.0, device=DEV)
    qb.qsdp_layer_norm_backward(xg, wg, got, dyg, dx[:, :n], dw, db)
    assert bool((dx[:, n:] == 5.0).all())
    for name, t in (("dx", dx[:, :n]), ("dw", dw), ("db", db)):
        assert near(t, grads[name], offs[name]), name
    again = [torch.empty_like(t) for t in (dw, db)]
    qb.qsdp_layer_norm_backward(xg, wg, got, dyg, None, *again)
    assert all(torch.equal(a, t) for a, t in zip(again, (dw, db)))  # the same bits, without dx
    before = dw.clone()
    qb.qsdp_layer_norm_backward(xg, wg, got, dyg, None, dw, None, accumulate=True)
    assert torch.equal(dw, before + before)


@pytest.mark.parametrize("n", [5, 768, 2048, 5000, 20000])
def test_without_weight_and_bias_and_in_place(n):
    x, w, b, dy = _inputs(30, n, 0, 0, "bf16", "bf16", "f32", 9)
    for weight, bias in ((None, None), (w, None), (None, b)):
        want, _, _, off, _, _ = norm(x, weight, bias, 1e-3)
        xg = x.to(DEV)
        qb.qsdp_layer_norm(xg, None if weight is None else w.to(DEV), None if bias is None else b.to(DEV), 1e-3, xg)
        assert near(xg, want, off)
    xg, dyg, wg = x.to(DEV), dy.to(DEV), w.to(DEV)
    stats = torch.empty((30, 2), device=DEV)
    qb.qsdp_layer_norm(xg, wg, None, 1e-5, torch.empty_like(xg), stats)
    plain = torch.empty_like(xg), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    qb.qsdp_layer_norm_backward(xg, wg, stats, dyg, *plain)
    for over in ("dy", "x"):
        a, d = xg.clone(), dyg.clone()
        to = d if over == "dy" else a
        dw, db = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        qb.qsdp_layer_norm_backward(a, wg, stats, d, to, dw, db)
        assert all(torch.equal(p, q) for p, q in zip(plain, (to, dw, db)))
    grads, offs = norm_grad(x, None, dy, 1e-5)
    dx = torch.empty_like(xg)
    qb.qsdp_layer_norm_backward(xg, None, stats, dyg, dx)
    assert near(dx, grads["dx"], offs["dx"])


def test_rows_far_from_zero_constant_rows_and_what_is_no_number():
    n = 1000
    x = matrix(8, n, torch.float32, seed=4)
    x[0] += 3e4
    x[1] = 2.5
    x[2] = 0.0
    x[3, 17] = float("nan")
    x[4, 999] = float("inf")
    want, stats, _, off, stats_off, _ = norm(x, None, None, 1e-5)
    y, got = _forward(x.to(DEV), None, None, 1e-5, torch.float32)
    fine = [0, 1, 2, 5, 6, 7]
    assert near(y[fine], want[fine], off[fine]) and near(got[fine], stats[fine], stats_off[fine])
    assert bool(y[[3, 4]].isnan().all())
    dy = matrix(8, n, torch.float32, seed=5)
    dx, dw, db = torch.empty((8, n), device=DEV), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    qb.qsdp_layer_norm_backward(x.to(DEV), None, got, dy.to(DEV), dx, dw, db)
    grads, offs = norm_grad(x, None, dy, 1e-5)
    assert near(dx[fine], grads["dx"][fine], offs["dx"][fine]) and bool(dx[[3, 4]].isnan().all()) and bool(dw.isnan().all())
    assert near(db, grads["db"], offs["db"])
    y, _ = _forward(torch.full((2, 64), 3.0, device=DEV), None, None, 0.0, torch.float32)
    assert bool(y.isnan().all())


def test_no_rows():
    x = torch.empty((0, 100), device=DEV)
    stats, dw, db = torch.empty((0, 2), device=DEV), torch.full((100,), 4.0, device=DEV), torch.full((100,), 4.0, device=DEV)
    qb.qsdp_layer_norm(x, None, None, 1e-5, torch.empty_like(x), stats)
    qb.qsdp_layer_norm_backward(x, None, stats, x, x, dw, db, accumulate=True)
    assert bool((dw == 4.0).all()) and bool((db == 4.0).all())
    qb.qsdp_layer_norm_backward(x, None, stats, x, x, dw, None)
    assert bool((dw == 0.0).all()) and bool((db == 4.0).all())


@pytest.mark.parametrize("n", [96, 2048])
def test_gradients_against_differences(n):
    """Of sum(y dy) along random directions, the function in 64 bits, steps of 1e-4."""
    x, w, b, dy = _inputs(12, n, 0, 0, "f32", "f32", "f32", 21)
    _, stats = _forward(x.to(DEV), w.to(DEV), b.to(DEV), 1e-5, torch.float32)
    dx, dw, db = torch.empty((12, n), device=DEV), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    qb.qsdp_layer_norm_backward(x.to(DEV), w.to(DEV), stats, dy.to(DEV), dx, dw, db)
    grads, offs = norm_grad(x, w, dy, 1e-5)
    for name, at, got in (("dx", x, dx), ("dw", w, dw), ("db", b, db)):
        d = torch.randn(at.shape, generator=torch.Generator().manual_seed(3), dtype=torch.float64)
        d /= d.norm()
        step, values = 1e-4, []
        for sign in (1, -1):
            moved = at.double() + sign * step * d
            args = {"dx": (moved, w, b), "dw": (x, moved, b), "db": (x, w, moved)}[name]
            values.append(float((norm(*args, 1e-5)[0] * dy.double()).sum()))
        slope = (values[0] - values[1]) / (2 * step)
        along = float((got.cpu().double() * d).sum())
        # third derivatives are of the order of the gradient itself: 1e-8 of it by the steps; and rounding of the sums
        size = float(grads[name].abs().sum())
        bound = float((offs[name] * d.abs()).sum()) + 1e-6 * size + 1e-11 * float((dy.double().abs()).sum()) * n / step
        assert abs(along - slope) <= bound, (name, along, slope, bound)
