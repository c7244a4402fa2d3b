"""The operators of a training step in few bits as a step uses them together: every result against its definition from what went in,
the step captured and replayed, on other streams, and at offsets that 32 bits do not hold."""
import pytest
import torch

from paper_2302_02390_amd import binding as qb
from train_util import DEV, DTYPES, adamw, blocks, held, matrix, near, norm, norm_grad, product

pytestmark = pytest.mark.gpu

EPS, HYPER = 1e-5, dict(beta1=0.9, beta2=0.95, eps=1e-8)


class Layer:
    """Layer norm and a linear layer on it, with a gradient that comes from behind, and their AdamW; `rows` tokens of `k` features."""

    def __init__(self, rows, k, n, dtype, seed=0):
        dt = DTYPES[dtype]
        self.rows, self.k, self.n = rows, k, n
        dev = lambda r, c, t, s, std, mean=0.0: matrix(r, c, t, seed=seed + s, std=std, mean=mean).to(DEV)
        self.x, self.dy = dev(rows, k, dt, 1, 1.0), dev(rows, n, dt, 2, 1e-2)
        self.w, self.gain, self.shift = dev(n, k, torch.float32, 3, 0.02), dev(1, k, torch.float32, 4, 0.1, 1.0)[0], dev(1, k, torch.float32, 5, 0.1)[0]
        self.w16 = self.w.to(dt)
        like = lambda *size: torch.zeros(size, dtype=dt, device=DEV)
        self.h, self.y, self.dh, self.dx, self.answer = like(rows, k), like(rows, n), like(rows, k), like(rows, k), like(1, n)
        self.stats = torch.zeros((rows, 2), device=DEV)
        self.dw, self.dgain, self.dshift = (torch.zeros_like(t) for t in (self.w, self.gain, self.shift))
        self.hq, self.dyq, self.wq = qb.alloc_blocks(rows, k, False, DEV), qb.alloc_blocks(rows, n, False, DEV), qb.alloc_blocks(n, k, True, DEV)
        bytes_ = max(qb.matmul_blocks_bytes(rows, n, k), qb.matmul_blocks_bytes(rows, k, n), qb.matmul_blocks_bytes(n, k, rows),
                     qb.layer_norm_backward_bytes(rows, k), qb.linear_blocks_bytes(1, n, k), 16)
        self.room = torch.empty(bytes_, dtype=torch.uint8, device=DEV)  # one after another on one stream: they can share it
        params = [self.w, self.gain, self.shift]
        state = [qb.alloc_moments(p, 8 if p.dim() == 2 else 32) for p in params]
        self.m, self.v, self.s = (list(t) for t in zip(*state))
        self.table = qb.AdamWTensors(params, [self.dw, self.dgain, self.dshift], self.m, self.v, self.s, [self.w16 if dtype != "f32" else None, None, None],
                                     [0.1, 0.0, 0.0])
        self.schedule, self.more = torch.tensor([1e-2, 0.1, 0.05], device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)

    def forward(self):
        qb.qsdp_layer_norm(self.x, self.gain, self.shift, EPS, self.h, self.stats)
        qb.qsdp_quantize_blocks(self.h, False, *self.hq)
        qb.qsdp_quantize_blocks(self.w16, True, *self.wq)
        qb.qsdp_matmul_blocks(*self.hq[:2], *self.wq[:2], self.k, None, self.y, False, self.room)
        qb.qsdp_linear_blocks(self.h[:1], *self.wq[:2], None, self.answer, self.room)

    def backward(self):
        qb.qsdp_quantize_blocks(self.dy, False, *self.dyq)
        qb.qsdp_matmul_blocks(*self.dyq[:2], *self.wq[2:], self.n, None, self.dh, False, self.room)
        qb.qsdp_matmul_blocks(*self.dyq[2:], *self.hq[2:], self.rows, None, self.dw, False, self.room)
        qb.qsdp_layer_norm_backward(self.x, self.gain, self.stats, self.dh, self.dx, self.dgain, self.dshift, False, self.room)

    def step(self):
        qb.qsdp_adamw_tensors(self.table, 1.0, bias1=1.0, bias2=1.0, seed=5, seed_increment=self.more, schedule=self.schedule, **HYPER)

    def all(self):
        self.forward()
        self.backward()
        self.step()

    def state(self):
        return [t.clone() for t in (self.h, self.y, self.answer, self.dh, self.dx, self.dw, self.dgain, self.dshift, self.w, self.gain,
                                    self.shift, self.w16, *self.m, *self.v, self.s[0])]


SHAPES = [(333, 200, 500, "bf16"), (65, 1000, 130, "f16"), (2100, 260, 384, "f32")]


@pytest.mark.parametrize("rows,k,n,dtype", SHAPES)
def test_a_step(rows, k, n, dtype):
    l = Layer(rows, k, n, dtype)
    w, gain, shift = (t.cpu() for t in (l.w, l.gain, l.shift))
    m, v, s = ([None if t is None else t.cpu() for t in a] for a in (l.m, l.v, l.s))
    l.forward()
    want, stats, _, off, stats_off, _ = norm(l.x.cpu(), gain, shift, EPS)
    assert near(l.h, want, off) and near(l.stats, stats, stats_off)
    h, exact = l.h.cpu(), dtype == "f32"
    hh, hw = held(*blocks(h, 1, 128), 1, 128), held(*blocks(l.w16.cpu(), 128, 128), 128, 128)
    assert near(l.y, *product(hh, hw, exact)) and near(l.answer, *product(hh[:1], hw, exact))
    l.backward()
    dy = l.dy.cpu()
    hd, hdt = held(*blocks(dy, 1, 128), 1, 128), held(*blocks(dy.t(), 1, 128), 1, 128)
    assert near(l.dh, *product(hd, hw.t().contiguous(), exact))
    assert near(l.dw, *product(hdt, held(*blocks(h.t(), 1, 128), 1, 128), True))
    grads, offs = norm_grad(l.x.cpu(), gain, l.dh.cpu(), EPS)
    for got, name in ((l.dx, "dx"), (l.dgain, "dw"), (l.dshift, "db")):
        assert near(got, grads[name], offs[name]), name
    l.step()
    first = 0
    h = dict(HYPER, bias1=0.1, bias2=0.05, lr=1e-2)
    for i, (p, old, g) in enumerate(((l.w, w, l.dw), (l.gain, gain, l.dgain), (l.shift, shift, l.dshift))):
        x, off, m1, v1, s1 = adamw(old.reshape(-1), g.cpu().reshape(-1), m[i].reshape(-1), v[i].reshape(-1), s[i], first, 5,
                                   decay=0.0 if i else 0.1, **h)
        first += -(-old.numel() // 2048)
        assert near(p.reshape(-1), x, off) and torch.equal(l.m[i].cpu().reshape(-1), m1) and torch.equal(l.v[i].cpu().reshape(-1), v1)
        assert s1 is None or torch.equal(l.s[i].cpu(), s1)
    if dtype != "f32":
        assert torch.equal(l.w16, l.w.to(l.w16.dtype))


def test_gradients_of_the_held_values_against_differences():
    """The product of what the codes stand for is linear in either side: a difference along any direction is its slope but for
    roundings."""
    l = Layer(200, 300, 260, "bf16")
    l.forward()
    l.backward()
    hh, hw = held(*blocks(l.h.cpu(), 1, 128), 1, 128), held(*blocks(l.w16.cpu(), 128, 128), 128, 128)
    hd = held(*blocks(l.dy.cpu(), 1, 128), 1, 128)
    value = lambda a, b: float(((a @ b.t()) * hd).sum())
    d = torch.randn(hh.shape, generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    slope = (value(hh + 0.5 * d, hw) - value(hh - 0.5 * d, hw))
    _, off = product(hd, hw.t().contiguous(), False)
    got = l.dh.double().cpu()
    bound = float(((off + got.abs() * 2.0 ** -8) * d.abs()).sum()) + 1e-9 * float((hh.abs() @ hw.abs().t() * hd.abs()).sum())
    assert abs(float((got * d).sum()) - slope) <= bound
    # the weight's gradient rounds dy and x along the rows: its own held values
    ht, hdt = held(*blocks(l.h.cpu().t(), 1, 128), 1, 128), held(*blocks(l.dy.cpu().t(), 1, 128), 1, 128)
    value = lambda b: float(((ht.t() @ b.t()) * hdt.t()).sum())
    d = torch.randn(hw.shape, generator=torch.Generator().manual_seed(2), dtype=torch.float64)
    slope = value(hw + 0.5 * d) - value(hw - 0.5 * d)
    _, off = product(hdt, ht, True)
    bound = float((off * d.abs()).sum()) + 1e-9 * float((ht.t().abs() @ hw.abs().t() * hdt.t().abs()).sum())
    assert abs(float((l.dw.double().cpu() * d).sum()) - slope) <= bound


@pytest.mark.parametrize("rows,k,n,dtype", SHAPES + [(40, 6200, 64, "bf16")])
def test_a_captured_step(rows, k, n, dtype):
    """Captured once and replayed five times, eager work and synchronizations between, against eager steps: the same bits."""
    eager, replayed = Layer(rows, k, n, dtype), Layer(rows, k, n, dtype)
    replayed.all()  # before the capture, as a program warms up; then back to the start
    fresh = Layer(rows, k, n, dtype)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed.all()
    for t, s in zip((replayed.w, replayed.gain, replayed.shift, replayed.w16, *replayed.m, *replayed.v, replayed.s[0]),
                    (fresh.w, fresh.gain, fresh.shift, fresh.w16, *fresh.m, *fresh.v, fresh.s[0])):
        t.copy_(s)
    for step in range(5):
        for l in (eager, replayed):
            l.more.fill_(step)
            l.schedule.copy_(torch.tensor([1e-2 / (step + 1), 1 - 0.9 ** (step + 1), 1 - 0.95 ** (step + 1)]))
            l.dy.mul_(-0.75)
        eager.all()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager.state(), replayed.state())), step
        float(torch.randn(1 << 20, device=DEV).sum())


def test_two_streams_at_once():
    layers = [Layer(500, 768, 1000, "bf16", seed=i) for i in range(2)]
    alone = [Layer(500, 768, 1000, "bf16", seed=i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in layers]
    torch.cuda.synchronize()
    for _ in range(4):
        for l, s in zip(layers, streams):
            with torch.cuda.stream(s):
                l.all()
    torch.cuda.synchronize()
    for l in alone:
        for _ in range(4):
            l.all()
    for a, b in zip(layers, alone):
        assert all(torch.equal(p, q) for p, q in zip(a.state(), b.state()))


def test_rows_past_32_bits():
    """Elements and bytes whose numbers pass 2^32: the last rows are those of a call of their own."""
    n = 2048
    rows = (1 << 32) // n + 300
    x = torch.empty((rows, n), dtype=torch.bfloat16, device=DEV).normal_(generator=torch.Generator(DEV).manual_seed(1))
    y, stats = torch.empty_like(x), torch.empty((rows, 2), device=DEV)
    qb.qsdp_layer_norm(x, None, None, EPS, y, stats)
    last = slice(rows - 400, rows)
    y1, stats1 = torch.empty_like(x[last]), torch.empty((400, 2), device=DEV)
    qb.qsdp_layer_norm(x[last], None, None, EPS, y1, stats1)
    want, s, _, off, s_off, _ = norm(x[last].cpu(), None, None, EPS)
    assert near(y[last], want, off) and near(stats[last], s, s_off) and near(y1, want, off)
    dx = y
    qb.qsdp_layer_norm_backward(x, None, stats, x, dx)
    grads, offs = norm_grad(x[last].cpu(), None, x[last].cpu(), EPS)
    assert near(dx[last], grads["dx"], offs["dx"])
    del y, dx
    codes, scales, codes_t, scales_t = qb.alloc_blocks(rows, n, False, DEV)
    qb.qsdp_quantize_blocks(x, False, codes, scales, codes_t, scales_t)
    begin = rows // 128 * 128 - 128  # whole blocks of rows
    part = qb.alloc_blocks(rows - begin, n, False, DEV)
    qb.qsdp_quantize_blocks(x[begin:], False, *part)
    as_bytes = lambda t: t.view(torch.uint8)
    assert torch.equal(as_bytes(codes)[begin:], as_bytes(part[0])) and torch.equal(scales[:, begin:], part[1])
    assert torch.equal(as_bytes(codes_t)[:, begin:], as_bytes(part[2])) and torch.equal(scales_t[begin // 128:], part[3])
    del codes_t, scales_t
    w = qb.alloc_blocks(70, n, True, DEV)
    qb.qsdp_quantize_blocks(matrix(70, n, torch.float32, seed=3, std=0.05).to(DEV), True, *w)
    y = torch.empty((rows, 70), dtype=torch.bfloat16, device=DEV)
    qb.qsdp_matmul_blocks(codes, scales, *w[:2], n, None, y)
    hh = held(codes[last].float().cpu(), scales[:, last].t().cpu(), 1, 128)
    hw = held(w[0].float().cpu(), w[1].t().cpu(), 128, 128)
    assert near(y[last], *product(hh, hw, False))


def test_results_past_32_bits():
    m, n, k = (1 << 17) + 70, 33000, 128
    a, b = matrix(m, k, torch.bfloat16, seed=1), matrix(n, k, torch.bfloat16, seed=2, std=0.05)
    ac, bc = qb.alloc_blocks(m, k, False, DEV), qb.alloc_blocks(n, k, True, DEV)
    qb.qsdp_quantize_blocks(a.to(DEV), False, *ac)
    qb.qsdp_quantize_blocks(b.to(DEV), True, *bc)
    y = torch.empty((m, n), dtype=torch.bfloat16, device=DEV)
    qb.qsdp_matmul_blocks(*ac[:2], *bc[:2], k, None, y)
    ha, hb = held(*blocks(a[-200:], 1, 128), 1, 128), held(*blocks(b, 128, 128), 128, 128)
    assert near(y[-200:], *product(ha, hb, False))


def test_more_workgroups_than_a_grid_has():
    """Products of more than 2^20 tiles, and 2^20 rows that no team holds, go in several launches."""
    m, n, k = (1 << 26) + 300, 130, 100
    codes = torch.zeros((m, 128), dtype=torch.uint8, device=DEV)
    codes[:, :k] = torch.randint(0, 0x70, (1, k), dtype=torch.uint8, device=DEV)
    scales = torch.linspace(0.5, 1.0, m, device=DEV).view(1, m)
    b = matrix(n, k, torch.bfloat16, seed=2, std=0.05)
    bc = qb.alloc_blocks(n, k, True, DEV)
    qb.qsdp_quantize_blocks(b.to(DEV), True, *bc)
    y = torch.empty((m, n), dtype=torch.bfloat16, device=DEV)
    qb.qsdp_matmul_blocks(codes, scales, *bc[:2], k, None, y)
    hb = held(*blocks(b, 128, 128), 128, 128)
    for rows in (slice(0, 200), slice((1 << 26) - 100, (1 << 26) + 300)):
        ha = held(codes[rows, :k].view(torch.float8_e4m3fn).float().cpu(), scales[:, rows].t().cpu(), 1, 128)
        assert near(y[rows], *product(ha, hb, False))
    del codes, scales, y
    rows, n = (1 << 20) + 3, 32769
    x = torch.empty((rows, n), dtype=torch.bfloat16, device=DEV).normal_(generator=torch.Generator(DEV).manual_seed(1))
    stats = torch.empty((rows, 2), device=DEV)
    at = slice(rows - 5, rows)
    before = x[at].cpu()
    want, s, _, off, s_off, _ = norm(before, None, None, EPS)
    dy = torch.empty_like(x)
    qb.qsdp_layer_norm(x, None, None, EPS, dy, stats)
    assert near(dy[at], want, off) and near(stats[at], s, s_off)
    grads, offs = norm_grad(before, None, dy[at].cpu(), EPS)
    qb.qsdp_layer_norm_backward(x, None, stats, dy, dy)
    assert near(dy[at], grads["dx"], offs["dx"])


@pytest.mark.parametrize("bits", [32, 8])
def test_a_tensor_past_32_bits(bits):
    n = (1 << 32) + 5000
    x = torch.empty(n, device=DEV).normal_(0.0, 0.02, generator=torch.Generator(DEV).manual_seed(1))
    g = torch.empty(n, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1e-2, generator=torch.Generator(DEV).manual_seed(2))
    m, v, s = qb.alloc_moments(x, bits)
    begin = (1 << 32) - 4096
    old = [None if t is None else t.cpu() for t in (x[begin:], g[begin:], m[begin:], v[begin:], None if s is None else s[begin // 128:])]
    h = dict(HYPER, lr=1e-2, bias1=0.1, bias2=0.05)
    qb.qsdp_adamw_tensors(qb.AdamWTensors([x], [g], [m], [v], [s], weight_decay=0.1), seed=3, **h)
    want, off, m1, v1, s1 = adamw(*old, begin // 2048, 3, decay=0.1, **h)
    assert near(x[begin:], want, off) and torch.equal(m[begin:].cpu(), m1) and torch.equal(v[begin:].cpu(), v1)
    assert s is None or torch.equal(s[begin // 128:].cpu(), s1)
