"""Log probabilities, entropy and top alternatives of rows of logits, and their gradient, against the 64-bit definitions."""
import math

import pytest
import torch

import lm_util as lu
from paper_2302_02390_amd import binding as qb

pytestmark = pytest.mark.gpu
SIZES = [1, 2, 7, 63, 64, 65, 255, 1000, 4097, 12345, 50257, 131073]


def run_score(z, tokens, tau, top=0, workspace=None, entropy=True):
    rows = z.shape[0]
    f = dict(dtype=torch.float32, device=z.device)
    logprob, ent = torch.full((rows,), 7.0, **f), torch.full((rows,), 7.0, **f) if entropy else None
    stats = torch.full((rows, 2), 7.0, **f)
    tl = torch.full((rows, top), 7.0, **f) if top else None
    ti = torch.full((rows, top), -7, dtype=torch.int32, device=z.device) if top else None
    qb.qsdp_token_logprobs(z, tokens, tau, logprob, ent, stats, tl, ti, workspace)
    return logprob, ent, stats, tl, ti


def full_workspace(z, top):
    n = qb.token_logprobs_bytes(z.shape[0], z.shape[1], top)
    return torch.full((max(n, 16),), 0xA5, dtype=torch.uint8, device=z.device)


def check(z_cpu, tokens, tau, top, workspace=False):
    z = lu.to_gpu(z_cpu)
    logprob, entropy, stats, tl, ti = run_score(z, tokens.to(lu.DEV), tau, top, full_workspace(z, top) if workspace else None)
    want = lu.score(z_cpu, tokens, tau)
    rel = lu.spread(want[3], want[2])
    at = tokens.clamp(0, z.shape[1] - 1)[:, None]
    assert lu.near(logprob, want[0], rel.gather(1, at)[:, 0])
    assert lu.near(stats, want[2], rel.amin(1, keepdim=True))
    # entropy: the log of the sum and a weighted mean of t, whose terms carry the error of their probability
    p = want[3].exp()
    terms = torch.where(p == 0, 0.0, p * (want[3].abs() + want[2][:, 1:].abs().nan_to_num(0, 0, 0) + 1) * rel)
    assert lu.near(entropy, want[1], 2 * terms.sum(1).nan_to_num(0))
    if top:
        index = lu.order(z_cpu, top)
        assert torch.equal(ti.cpu().long(), index)
        bad = want[1].isnan()[:, None]
        assert lu.near(tl, torch.where(bad, math.nan, want[3].gather(1, index)), rel.gather(1, index))
    return logprob, entropy, stats, tl, ti


@pytest.mark.parametrize("workspace", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", SIZES)
def test_sizes(vocab, dtype, workspace):
    pad, offset = {"f32": (0, 1), "bf16": (3, 5), "f16": (vocab % 2, 0)}[dtype]
    z = lu.make_rows(3, vocab, lu.DTYPES[dtype], pad, seed=vocab, offset=offset)
    tokens = torch.tensor([0, vocab - 1, -100])
    check(z, tokens, 1.0, min(vocab, {"f32": 128, "bf16": 20, "f16": 1}[dtype]), workspace)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("top", [2, 63, 64, 65, 127, 128])
@pytest.mark.parametrize("tau", [0.25, 1.7])
def test_tops(top, tau, dtype):
    z = lu.make_rows(9, 5001, lu.DTYPES[dtype], 0, seed=top)
    check(z, torch.arange(9) * 555, tau, top)


@pytest.mark.parametrize("workspace", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_masks_and_ties(dtype, workspace):
    """Rows by name: mostly masked, masked whole, masked with the lowest value, one value throughout, two zeros of opposite
    sign, descending and ascending runs, the large ones all in one place, one entry left."""
    dt, vocab = lu.DTYPES[dtype], 40001
    z = lu.make_rows(12, vocab, dt, 0, seed=5)
    low = torch.finfo(dt).min
    keep = torch.rand(vocab, generator=torch.Generator().manual_seed(1)) < 0.001
    z[0, ~keep] = -math.inf
    z[1] = -math.inf
    z[2, ~keep] = low
    z[3] = low
    z[4] = 2.5
    z[5] = 0.0
    z[5, ::3] = -0.0
    z[6] = torch.linspace(20, -20, vocab).to(dt)
    z[7] = torch.linspace(-20, 20, vocab).to(dt)
    z[8, 17 * 64:17 * 64 + 600] = 30.0
    z[9] = -math.inf
    z[9, 33333] = -1.0
    z[10, ::256] = 25.0   # one lane's elements in every strided layout
    z[11] = torch.finfo(dt).max
    tokens = torch.tensor([int(keep.nonzero()[0]), 3, 5, 7, 11, 13, 17, 19, 23, 33333, 256, 31])
    check(z, tokens, 1.0, 100, workspace)
    check(z, torch.where(torch.arange(12) == 9, 0, tokens), 2.0, 7, workspace)


@pytest.mark.parametrize("workspace", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_nan_and_infinity(dtype, workspace):
    z = lu.make_rows(5, 3001, lu.DTYPES[dtype], 0, seed=6)
    z[0, 77] = math.nan
    z[1, 78] = math.inf
    z[2, 5:9] = math.nan
    z[2, 100] = math.inf
    z[3] = math.nan
    zg = lu.to_gpu(z)
    tokens = torch.tensor([4, 78, 6, 0, 3001])
    logprob, entropy, stats, tl, ti = run_score(zg, tokens.to(lu.DEV), 1.0, 12, full_workspace(zg, 12) if workspace else None)
    assert logprob.isnan().all() and entropy[:4].isnan().all() and not entropy[4].isnan()
    assert stats[:4, 1].isnan().all() and tl[:4].isnan().all() and not tl[4].isnan().any()
    assert torch.equal(ti.cpu().long(), lu.order(z, 12))
    d = torch.empty_like(zg)
    ones = torch.ones(5, device=lu.DEV)
    qb.qsdp_token_logprobs_backward(zg, tokens.to(lu.DEV), 1.0, stats, entropy, ones, ones, d)
    assert d[:4].isnan().all() and d[4].isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", SIZES)
def test_gradient(vocab, dtype):
    dt = lu.DTYPES[dtype]
    z = lu.make_rows(5, vocab, dt, vocab % 5, seed=vocab + 1, offset=3)
    if vocab > 100:
        z[3] = -math.inf
        z[4, 3:-7] = -math.inf
    tokens = torch.tensor([0, vocab - 1, -1, vocab // 2, vocab - 1])
    gen = torch.Generator().manual_seed(vocab)
    for g, h in ((torch.randn(5, generator=gen), None), (None, torch.randn(5, generator=gen)),
                 (torch.randn(5, generator=gen), torch.randn(5, generator=gen))):
        zg = lu.to_gpu(z)
        logprob, entropy, stats, _, _ = run_score(zg, tokens.to(lu.DEV), 0.7)
        want, off = lu.score_grad(z, tokens, 0.7, g, h)
        gg, hg = (None if v is None else v.to(lu.DEV) for v in (g, h))
        outs = []
        for pad in (0, 1, 8):  # other rows than the logits' among them
            full = torch.full((5, vocab + pad), 3.0, dtype=dt, device=lu.DEV)
            d = full[:, :vocab]
            qb.qsdp_token_logprobs_backward(zg, tokens.to(lu.DEV), 0.7, stats, entropy if h is not None else None, gg, hg, d)
            assert lu.near(d, want, off), (pad, g is None, h is None)
            assert bool((full[:, vocab:] == 3.0).all())
            outs.append(d.clone())
        qb.qsdp_token_logprobs_backward(zg, tokens.to(lu.DEV), 0.7, stats, entropy if h is not None else None, gg, hg, zg)
        assert all(torch.equal(o, zg) for o in outs)  # and in place


def test_gradient_against_differences():
    """Central differences of sum g logprob + h entropy along random directions. The step is 2^-6: the outputs' error (see
    spread) over it and the third derivative (below 8 (|g| + 3 |h|) for a direction of entries +-1) times its square."""
    vocab, rows, eps = 37, 6, 2.0 ** -6
    gen = torch.Generator().manual_seed(3)
    z = torch.randn((rows, vocab), generator=gen)
    tokens = torch.randint(0, vocab, (rows,), generator=gen)
    g, h = torch.randn(rows, generator=gen), torch.randn(rows, generator=gen)
    zg, tg = z.to(lu.DEV), tokens.to(lu.DEV)
    _, entropy, stats, _, _ = run_score(zg, tg, 1.0)
    d = torch.empty_like(zg)
    qb.qsdp_token_logprobs_backward(zg, tg, 1.0, stats, entropy, g.to(lu.DEV), h.to(lu.DEV), d)
    for _ in range(5):
        v = torch.randint(0, 2, z.shape, generator=gen).float() * 2 - 1

        def value(sign):
            lp, en, _, _, _ = run_score((z + sign * eps * v).to(lu.DEV), tg, 1.0)
            return g.double() * lp.cpu().double() + h.double() * en.cpu().double()
        slope = (value(1) - value(-1)) / (2 * eps)
        along = (d.cpu().double() * v.double()).sum(1)
        size = g.abs().double() + 3 * h.abs().double()
        assert bool(((slope - along).abs() <= size * (8 * eps ** 2 + 2.0 ** -18 / eps)).all())


def test_outputs_left_out():
    z = lu.to_gpu(lu.make_rows(3, 1001, torch.float32, 0, seed=1))
    tokens = torch.tensor([1, 2, 3], device=lu.DEV)
    logprob, entropy, stats, tl, ti = run_score(z, tokens, 1.0, 5)
    only = torch.empty(3, device=lu.DEV)
    qb.qsdp_token_logprobs(z, None, 1.0, None, only)
    assert torch.equal(only, entropy)
    qb.qsdp_token_logprobs(z, tokens, 1.0, only)
    assert torch.equal(only, logprob)
    t2, i2 = torch.empty_like(tl), torch.empty_like(ti)
    qb.qsdp_token_logprobs(z, None, 1.0, None, None, None, t2, i2)
    assert torch.equal(t2, tl) and torch.equal(i2, ti)
    qb.qsdp_token_logprobs(z[:0], tokens[:0], 1.0, only[:0])
    qb.qsdp_token_logprobs_backward(z[:0], tokens[:0], 1.0, stats[:0], None, only[:0], None, z[:0])


def test_many_rows():
    """More rows than a launch has workgroups."""
    rows = (1 << 20) + 77
    z = torch.randn((rows, 3), device=lu.DEV)
    tokens = torch.randint(0, 3, (rows,), device=lu.DEV)
    logprob, entropy, stats, tl, ti = run_score(z, tokens, 1.0, 1)
    want = torch.log_softmax(z.double(), 1)
    assert float((logprob - want.gather(1, tokens[:, None])[:, 0]).abs().max()) < 1e-6
    assert torch.equal(ti[:, 0].long(), z.argmax(1))
    d = torch.empty_like(z)
    qb.qsdp_token_logprobs_backward(z, tokens, 1.0, stats, None, torch.ones(rows, device=lu.DEV), None, d)
    assert float((d + want.exp() - torch.nn.functional.one_hot(tokens, 3)).abs().max()) < 1e-6


def test_rows_far_apart():
    """Offsets beyond 2^32 elements."""
    vocab, stride = 999, (1 << 31) + 8
    flat = torch.empty(2 * stride + vocab, dtype=torch.bfloat16, device=lu.DEV)
    z = flat.as_strided((3, vocab), (stride, 1))
    cpu = lu.make_rows(3, vocab, torch.bfloat16, 0, seed=9)
    z.copy_(cpu.to(lu.DEV))
    tokens = torch.tensor([5, 6, 7])
    logprob, entropy, stats, tl, ti = run_score(z, tokens.to(lu.DEV), 1.0, 9)
    want = lu.score(cpu, tokens, 1.0)
    assert lu.near(logprob, want[0], torch.full((3,), 1e-5)) and torch.equal(ti.cpu().long(), lu.order(cpu, 9))
    g = torch.ones(3)
    qb.qsdp_token_logprobs_backward(z, tokens.to(lu.DEV), 1.0, stats, None, g.to(lu.DEV), None, z)
    assert lu.near(z.contiguous(), *lu.score_grad(cpu, tokens, 1.0, g, None))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_same_again_and_on_another_stream(dtype):
    z = lu.to_gpu(lu.make_rows(4, 50257, lu.DTYPES[dtype], 0, seed=2))
    tokens = torch.tensor([1, 2, 3, 4], device=lu.DEV)
    first = [t.clone() for t in run_score(z, tokens, 1.0, 64, full_workspace(z, 64))]
    assert all(torch.equal(a, b) for a, b in zip(first, run_score(z, tokens, 1.0, 64, full_workspace(z, 64))))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        z2 = z * 1.0
        out = run_score(z2, tokens, 1.0, 64, full_workspace(z2, 64))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, out))


def test_in_a_graph():
    z = lu.to_gpu(lu.make_rows(2, 50257, torch.float32, 0, seed=4))
    tokens = torch.tensor([1, 2], device=lu.DEV)
    ws = full_workspace(z, 20)
    f = dict(dtype=torch.float32, device=lu.DEV)
    lp, en, st, tl = torch.empty(2, **f), torch.empty(2, **f), torch.empty((2, 2), **f), torch.empty((2, 20), **f)
    ti = torch.empty((2, 20), dtype=torch.int32, device=lu.DEV)
    d = torch.empty_like(z)
    one = torch.ones(2, **f)

    def step():
        qb.qsdp_token_logprobs(z, tokens, 1.0, lp, en, st, tl, ti, ws)
        qb.qsdp_token_logprobs_backward(z, tokens, 1.0, st, en, one, one, d)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (10, 11, 12):
        z.copy_(lu.make_rows(2, 50257, torch.float32, 0, seed=seed))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (lp, en, st, tl, ti, d)]
        for t in (lp, en, st, tl, d):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (lp, en, st, tl, ti, d)))


def test_refusals_of_the_binding():
    z = torch.zeros((3, 50), device=lu.DEV)
    t = torch.zeros(3, dtype=torch.int64, device=lu.DEV)
    out = torch.zeros(3, device=lu.DEV)
    ti = torch.zeros((3, 51), dtype=torch.int32, device=lu.DEV)
    with pytest.raises(TypeError):
        qb.qsdp_token_logprobs(z.double(), t, 1.0, out)
    with pytest.raises(TypeError):
        qb.qsdp_token_logprobs(z.t(), t, 1.0, out)
    with pytest.raises(TypeError):
        qb.qsdp_token_logprobs(z, t.int(), 1.0, out)
    with pytest.raises(ValueError):
        qb.qsdp_token_logprobs(z, t[:2], 1.0, out)
    with pytest.raises(ValueError):
        qb.qsdp_token_logprobs(z, t, 1.0, out, None, None, None, ti)
    for tau in (0.0, -1.0, math.inf, math.nan):
        with pytest.raises(qb.QsdpError):
            qb.qsdp_token_logprobs(z, t, tau, out)
    with pytest.raises(qb.QsdpError):  # more alternatives than entries
        qb.qsdp_token_logprobs(z, t, 1.0, out, None, None, torch.zeros((3, 51), device=lu.DEV), ti)
    with pytest.raises(qb.QsdpError):  # rows on top of each other
        qb.qsdp_token_logprobs(z[:1].expand(3, 50), t, 1.0, out)
    with pytest.raises(ValueError):
        qb.qsdp_token_logprobs_backward(z, t, 1.0, torch.zeros((3, 2), device=lu.DEV), None, out, None, z.half())
    with pytest.raises(qb.QsdpError):  # nothing to differentiate
        qb.qsdp_token_logprobs_backward(z, t, 1.0, torch.zeros((3, 2), device=lu.DEV), None, None, None, z)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [65536, 70001, 150003])
def test_rows_cut_into_parts(vocab, dtype):
    """Long rows shared among workgroups, parts without anything, equal values across parts: the results of whole rows."""
    dt = lu.DTYPES[dtype]
    assert qb.token_logprobs_bytes(9, vocab, 100) > 0
    z = lu.make_rows(9, vocab, dt, 3, seed=vocab, offset=1)
    z[1] = -math.inf
    z[2] = -math.inf
    z[2, vocab - 2] = 1.0                       # all but the last part empty
    z[3] = 0.25                                 # equal throughout
    z[4, ::1000] = 20.0                         # equal ones in every part
    z[5] = torch.finfo(dt).min
    z[6, 5000:60000] = torch.finfo(dt).min
    z[7, :vocab // 2] = -math.inf
    tokens = torch.tensor([vocab - 1, 4, vocab - 2, 7, 1000, 9, -5, vocab - 9, vocab // 2])
    check(z, tokens, 1.0, 100, True)
    check(z, tokens, 0.7, 1, True)
    zg = lu.to_gpu(z)
    zg[8, 66] = math.nan
    out = run_score(zg, tokens.to(lu.DEV), 1.0, 20, full_workspace(zg, 20))
    whole = run_score(zg, tokens.to(lu.DEV), 1.0, 20)
    assert torch.equal(out[4], whole[4]) and out[0][8].isnan() and out[1][8].isnan() and out[3][8].isnan().all()
    short = torch.empty(qb.token_logprobs_bytes(9, vocab, 20) - 1, dtype=torch.uint8, device=lu.DEV)
    assert all(torch.equal(a.nan_to_num(9), b.nan_to_num(9)) for a, b in zip(run_score(zg, tokens.to(lu.DEV), 1.0, 20, short), whole))
