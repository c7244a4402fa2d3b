"""Distillation from a teacher's top logits, loss and gradient, against the 64-bit definitions."""
import math

import pytest
import torch

import lm_util as lu
from paper_2302_02390_amd import binding as qb

pytestmark = pytest.mark.gpu


def lists(rows, vocab, top, seed, spread=3.0):
    gen = torch.Generator().manual_seed(seed)
    index = torch.stack([torch.randperm(vocab, generator=gen)[:top] for _ in range(rows)]).int()
    return index, torch.randn((rows, top), generator=gen) * spread + 5.0


def run(z, index, logit, labels, tau, alpha, scale=None, grad=True, pad=0, two=False):
    """(loss, gradient, the padded buffer it lies in); two: loss first, then the gradient from its stats."""
    rows, vocab = z.shape
    gpu = lambda t: None if t is None else t.to(lu.DEV)  # noqa: E731
    index, logit, labels, scale = gpu(index), gpu(logit), gpu(labels), gpu(scale)
    loss = torch.full((rows,), 7.0, device=lu.DEV)
    full = torch.full((rows, vocab + pad), 3.0, dtype=z.dtype, device=lu.DEV)
    d = full[:, :vocab]
    if two:
        stats = torch.full((rows, 3), 7.0, device=lu.DEV)
        qb.qsdp_distill_loss(z, index, logit, labels, tau, alpha, None, loss, stats)
        g = torch.ones(rows, device=lu.DEV) if scale is None else scale
        qb.qsdp_distill_loss_backward(z, index, logit, labels, tau, alpha, stats, g, d)
    else:
        qb.qsdp_distill_loss(z, index, logit, labels, tau, alpha, scale, loss, None, d if grad else None)
    return loss, d, full


def check(z_cpu, index, logit, labels, tau, alpha, scale=None):
    want, want_d, loss_off, off = lu.distill(z_cpu, index, logit, labels, tau, alpha)
    s = torch.ones(len(want), dtype=torch.float64) if scale is None else scale.double()
    for two, pad in ((False, 0), (False, 3), (True, 0)):
        loss, d, full = run(lu.to_gpu(z_cpu), index, logit, labels, tau, alpha, scale, True, pad, two)
        assert lu.near(loss, want, loss_off), (two, pad)
        assert lu.near(d, want_d * s[:, None], off * s.abs()[:, None]), (two, pad)
        assert bool((full[:, z_cpu.shape[1]:] == 3.0).all())
    alone, _, _ = run(lu.to_gpu(z_cpu), index, logit, labels, tau, alpha, scale, grad=False)
    assert torch.equal(alone.nan_to_num(-1), loss.nan_to_num(-1))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [1, 2, 9, 64, 255, 1000, 8191, 50257, 131073])
def test_sizes(vocab, dtype):
    z = lu.make_rows(3, vocab, lu.DTYPES[dtype], vocab % 3, seed=vocab, offset=vocab % 4)
    top = min(vocab, {"f32": 128, "bf16": 20, "f16": 64}[dtype])
    index, logit = lists(3, vocab, top, vocab)
    labels = torch.tensor([0, -100, vocab - 1])
    for tau, alpha in ((1.0, 1.0), (2.0, 0.5), (1.0, 0.3)):
        check(z, index, logit, labels, tau, alpha, torch.tensor([0.5, -2.0, 1.0]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [1, 3, 64, 65, 128])
def test_lists(top, dtype):
    z = lu.make_rows(6, 3001, lu.DTYPES[dtype], 0, seed=top)
    index, logit = lists(6, 3001, top, top)
    index[1, top // 2:] = -1                       # a shorter list
    index[2] = -1                                  # none
    index[3] = index[3, :1]                        # one index throughout
    logit[4] = -math.inf                           # no mass
    logit[5, top // 2:] = -math.inf
    index[0, 0] = 3001                             # past the vocabulary: absent
    labels = torch.tensor([3, int(index[1, 0]), 5, int(index[3, 0]), 3000, -1])
    check(z, index, logit, labels, 2.0, 0.7)
    check(z, index, logit, None, 0.5, 1.0)


def test_labels_alone():
    z = lu.make_rows(4, 777, torch.float32, 0, seed=3)
    check(z, None, None, torch.tensor([0, 776, -1, 5]), 1.0, 0.0)
    loss, _, _ = run(lu.to_gpu(z), None, None, torch.tensor([0, 777, -1, 5]), 1.0, 0.0)
    assert loss.isnan().tolist() == [False, True, False, False]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_masks(dtype):
    dt = lu.DTYPES[dtype]
    z = lu.make_rows(6, 5003, dt, 0, seed=8)
    index, logit = lists(6, 5003, 10, 8)
    z[0, 100:] = -math.inf
    index[0] = torch.arange(10)
    z[1] = -math.inf                                # nothing left: infinite loss, no gradient
    z[2, 50:] = torch.finfo(dt).min
    index[2] = torch.arange(10)
    z[3] = torch.finfo(dt).min
    z[4, int(index[4, 3])] = -math.inf              # the student cannot say what the teacher does
    logit[4, 3] = -math.inf                         # ... nor the teacher: no part in the loss
    z[5, int(index[5, 0])] = -math.inf              # the loss is infinite, its gradient is not
    labels = torch.tensor([5, 6, 7, 8, 9, 10])
    check(z, index, logit, labels, 1.0, 0.5)
    check(z, index, logit, None, 3.0, 1.0)
    assert run(lu.to_gpu(z), index, logit, None, 1.0, 1.0)[0].isinf().tolist() == [False, True, False, False, False, True]


def test_nan_and_infinity():
    z = lu.make_rows(4, 1001, torch.float32, 0, seed=2)
    index, logit = lists(4, 1001, 8, 2)
    z[0, 500] = math.nan
    z[1, 501] = math.inf
    logit[2, 3] = math.nan
    loss, d, _ = run(lu.to_gpu(z), index, logit, None, 1.0, 1.0)
    assert loss.isnan().tolist() == [True, True, True, False]
    assert d[0].isnan().all() and d[1].isnan().all() and d[2].isnan().any() and d[3].isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1001, 50257, 131073])
def test_in_place(vocab, dtype):
    z = lu.to_gpu(lu.make_rows(5, vocab, lu.DTYPES[dtype], 0, seed=1))
    index, logit = lists(5, vocab, 50, 1)
    labels = torch.tensor([1, 2, 3, 4, int(index[4, 0])])
    loss, d, _ = run(z, index, logit, labels, 2.0, 0.5)
    again = torch.empty_like(loss)
    qb.qsdp_distill_loss(z, index.to(lu.DEV), logit.to(lu.DEV), labels.to(lu.DEV), 2.0, 0.5, None, again, None, z)
    assert torch.equal(z, d) and torch.equal(again, loss)


def test_gradient_against_differences():
    """Central differences of the loss along random directions of +-1: the loss's error (see lm_util.spread) over the step
    2^-6, and its third derivative (below 8 tau^2 / tau^3 + 8) times its square."""
    gen = torch.Generator().manual_seed(4)
    rows, vocab, eps, tau, alpha = 5, 41, 2.0 ** -6, 1.5, 0.6
    z = torch.randn((rows, vocab), generator=gen)
    index, logit = lists(rows, vocab, 9, 4, 1.0)
    labels = torch.randint(0, vocab, (rows,), generator=gen)
    _, d, _ = run(z.to(lu.DEV), index, logit, labels, tau, alpha)
    for _ in range(5):
        v = torch.randint(0, 2, z.shape, generator=gen).float() * 2 - 1
        up, down = (run((z + s * eps * v).to(lu.DEV), index, logit, labels, tau, alpha, grad=False)[0].cpu().double()
                    for s in (1, -1))
        along = (d.cpu().double() * v.double()).sum(1)
        assert bool((((up - down) / (2 * eps) - along).abs() <= 16 * eps ** 2 + 2.0 ** -17 / eps).all())


def test_many_rows_and_a_graph():
    rows = (1 << 20) + 5
    z = torch.randn((rows, 2), device=lu.DEV)
    labels = torch.randint(0, 2, (rows,), device=lu.DEV)
    loss, d = torch.empty(rows, device=lu.DEV), torch.empty_like(z)
    qb.qsdp_distill_loss(z, None, None, labels, 1.0, 0.0, None, loss, None, d)
    want = -torch.log_softmax(z.double(), 1).gather(1, labels[:, None])[:, 0]
    assert float((loss - want).abs().max()) < 1e-6
    z = lu.to_gpu(lu.make_rows(3, 50257, torch.bfloat16, 0, seed=4))
    index, logit = (t.to(lu.DEV) for t in lists(3, 50257, 64, 4))
    labels = torch.tensor([4, 5, 6], device=lu.DEV)
    loss, d = torch.empty(3, device=lu.DEV), torch.empty_like(z)
    step = lambda: qb.qsdp_distill_loss(z, index, logit, labels, 2.0, 0.5, None, loss, None, d)  # noqa: E731
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (5, 6, 7):
        z.copy_(lu.make_rows(3, 50257, torch.bfloat16, 0, seed=seed))
        step()
        torch.cuda.synchronize()
        want = loss.clone(), d.clone()
        loss.zero_(), d.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want[0], loss) and torch.equal(want[1], d)


def test_refusals_of_the_binding():
    z = torch.zeros((3, 50), device=lu.DEV)
    index, logit = torch.zeros((3, 4), dtype=torch.int32, device=lu.DEV), torch.zeros((3, 4), device=lu.DEV)
    labels, loss = torch.zeros(3, dtype=torch.int64, device=lu.DEV), torch.zeros(3, device=lu.DEV)
    with pytest.raises(ValueError):
        qb.qsdp_distill_loss(z, index[:2], logit[:2], labels, 1.0, 0.5, None, loss)
    with pytest.raises(ValueError):
        qb.qsdp_distill_loss(z, index, logit, labels[:1], 1.0, 0.5, None, loss)
    with pytest.raises(TypeError):
        qb.qsdp_distill_loss(z, index.long(), logit, labels, 1.0, 0.5, None, loss)
    with pytest.raises(ValueError):
        qb.qsdp_distill_loss(z, index, logit, labels, 1.0, 0.5, None, loss, None, z[:, :49])
    for tau, alpha in ((0.0, 0.5), (1.0, -0.1), (1.0, 1.1), (1.0, math.nan), (math.nan, 0.5)):
        with pytest.raises(qb.QsdpError):
            qb.qsdp_distill_loss(z, index, logit, labels, tau, alpha, None, loss)
    with pytest.raises(qb.QsdpError):
        qb.qsdp_distill_loss(z, index, logit, None, 1.0, 0.5, None, loss)      # labels are needed
    with pytest.raises(qb.QsdpError):
        qb.qsdp_distill_loss(z, None, None, labels, 1.0, 0.5, None, loss)      # and the list
    wide = torch.zeros((3, 129), dtype=torch.int32, device=lu.DEV), torch.zeros((3, 129), device=lu.DEV)
    with pytest.raises(qb.QsdpError):
        qb.qsdp_distill_loss(z, *wide, labels, 1.0, 0.5, None, loss)
