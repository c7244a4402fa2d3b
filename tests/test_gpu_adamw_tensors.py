"""AdamW over many tensors: moments in 32 and in 8 bits, bit for bit; weights against 64 bits."""
import pytest
import torch

from paper_2302_02390_amd import binding as qb
from train_util import DEV, DTYPES, adamw, by_256, moments, near

pytestmark = pytest.mark.gpu

HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8, bias1=1 - 0.9 ** 3, bias2=1 - 0.95 ** 3)
SIZES = [1, 2048, 7, 0, 255, 256, 257, 4096, 2049, 5000, 8, 12345, 70001, 0]


class Model:
    """Tensors of given sizes and their states, `offset` elements behind aligned addresses, and the same on the CPU."""

    def __init__(self, sizes, bits, dtype="f32", copy=None, offset=0, seed=0):
        gen = torch.Generator().manual_seed(seed)
        rnd = lambda n, std: torch.randn(n, generator=gen) * std
        self.bits = [bits[i % len(bits)] for i in range(len(sizes))]
        self.x = [rnd(n, 0.02) for n in sizes]
        self.g = [(rnd(n, 1e-2) * torch.rand(n, generator=gen) ** 3).to(DTYPES[dtype]) for n in sizes]
        self.decay = [0.1 if n > 300 else 0.0 for n in sizes]
        self.rate = [1.0 if i % 3 else 0.5 for i in range(len(sizes))]
        state = [qb.alloc_moments(x, b) for x, b in zip(self.x, self.bits)]
        self.m, self.v, self.s = (list(t) for t in zip(*state))

        def put(t):
            if t is None:
                return None
            step = 8 if t.element_size() == 1 else offset
            room = torch.empty(t.numel() + step, dtype=t.dtype, device=DEV)[step:]
            return room.copy_(t)

        self.dx, self.dg, self.dm, self.dv = ([put(t) for t in l] for l in (self.x, self.g, self.m, self.v))
        self.ds = [None if t is None else t.to(DEV) for t in self.s]
        self.copies = [None if copy is None or i % 4 == 3 else torch.empty(n + 1, dtype=DTYPES[copy], device=DEV)[1:]
                       for i, n in enumerate(sizes)]
        self.table = qb.AdamWTensors(self.dx, self.dg, self.dm, self.dv, self.ds, self.copies, self.decay, self.rate)

    def step_and_check(self, seed, scale=None, **hyper):
        h = dict(HYPER, **hyper)
        factor = None if scale is None else torch.tensor([scale], device=DEV)
        qb.qsdp_adamw_tensors(self.table, **h, seed=seed, grad_scale=factor)
        first = 0
        lr = h.pop("lr")
        for i, x in enumerate(self.x):
            g = self.g[i].float() if scale is None else self.g[i].float() * torch.tensor(scale)
            rate = float(torch.tensor(lr) * torch.tensor(self.rate[i]))
            y, off, m, v, s = adamw(x, g, self.m[i], self.v[i], self.s[i], first, seed, rate, decay=self.decay[i], **h)
            first += -(-x.numel() // 2048)
            if x.numel() == 0:
                continue
            assert near(self.dx[i], y, off), i
            assert torch.equal(self.dm[i].cpu(), m) and torch.equal(self.dv[i].cpu(), v), i
            if s is not None:
                assert torch.equal(self.ds[i].cpu(), s), i
            if self.copies[i] is not None:
                assert torch.equal(self.copies[i], self.dx[i].to(self.copies[i].dtype)), i
            self.x[i], self.m[i], self.v[i], self.s[i] = self.dx[i].cpu(), m, v, s


@pytest.mark.parametrize("bits", [(32,), (8,), (8, 32)])
@pytest.mark.parametrize("dtype,copy,offset", [("f32", None, 0), ("bf16", "bf16", 1), ("f16", "f16", 3)])
def test_steps(bits, dtype, copy, offset):
    model = Model(SIZES, bits, dtype, copy, offset)
    for seed in (0, 5, (7 << 32) + 3):
        model.step_and_check(seed)
    model.step_and_check(9, scale=0.25)


@pytest.mark.parametrize("count", [1, 63, 64, 65, 400, 4097])
def test_many_tensors_are_found(count):
    model = Model([(i * 37) % 300 + (2100 if i % 50 == 0 else 0) for i in range(count)] if count > 1 else [3], (8, 32), seed=count)
    model.step_and_check(3)


def test_32_bits_are_the_step_without_quantizers():
    """The order of operations on moments is that of qsdp_fused_adamw_step; there, gradients of one value to a bucket are exact."""
    n, bucket = 4096, 32
    x = torch.randn(n, generator=torch.Generator().manual_seed(1)).to(DEV)
    g = (torch.randn(n // bucket, generator=torch.Generator().manual_seed(2)) * 1e-2).repeat_interleave(bucket).to(DEV)
    m, v, _ = qb.alloc_moments(x, 32)
    m2, v2 = m.clone(), v.clone()
    table = qb.AdamWTensors([x.clone()], [g], [m], [v], weight_decay=0.1)
    qb.qsdp_adamw_tensors(table, **HYPER)
    h = HYPER
    qb.qsdp_fused_adamw_step(x, g, m2, v2, h["lr"], h["beta1"], h["beta2"], h["eps"], 0.1, h["bias1"], h["bias2"], 8, 8, bucket, 0.0,
                             0, 0)
    assert torch.equal(m, m2) and torch.equal(v, v2)


def test_a_positive_second_moment_keeps_a_code_and_zeros_stay():
    n = 512
    g = torch.zeros(n)
    g[0], g[1], g[300] = 1e3, 1e-9, 1e-21
    x = torch.ones(n, device=DEV)
    m, v, s = qb.alloc_moments(x, 8)
    qb.qsdp_adamw_tensors(qb.AdamWTensors([x], [g.to(DEV)], [m], [v], [s]), **HYPER, seed=1)
    assert v[:2].tolist() == [255, 1] and int(v[2:256].sum()) == 0 and int(m[2:].abs().sum()) <= 127 and int(m[0]) == 127
    assert int(v[300]) == 255 and bool((x[301:] == 1).all())  # 0.05 * 1e-42 is a subnormal number, its root a normal one
    g[300] = 1e-38
    m, v, s = qb.alloc_moments(x, 8)
    qb.qsdp_adamw_tensors(qb.AdamWTensors([x], [g.to(DEV)], [m], [v], [s]), **HYPER, seed=1)
    assert int(v[300]) == 0 and int(m[300]) == 0 and s[2:].tolist() == [0.0, 0.0]


@pytest.mark.parametrize("beta2", [0.95, 0.999])
def test_the_mean_over_seeds_is_right(beta2):
    """One step from the same moments under 4096 seeds: codes' values have the mean that the step computes. The rounding's variance is
    at most a quarter of a step squared; six standard errors. (sqrt v is what is rounded, so its mean is.)"""
    gen = torch.Generator().manual_seed(4)
    n = 256
    x, g = torch.zeros(n), torch.randn(n, generator=gen) * 1e-3
    m = torch.randint(-127, 128, (n,), generator=gen).to(torch.int8)
    v = torch.randint(1, 256, (n,), generator=gen).to(torch.uint8)
    s = torch.tensor([1e-3, 2e-3])
    count = 4096
    rep = lambda t: t.repeat(count).to(DEV)  # blocks of one tensor have thresholds of their own
    xs, gs, ms, vs, ss = (rep(t) for t in (x, g, m, v, s))
    qb.qsdp_adamw_tensors(qb.AdamWTensors([xs], [gs], [ms], [vs], [ss]), **dict(HYPER, beta2=beta2), seed=77)
    got_m, got_v = moments(ms.cpu(), vs.cpu(), ss.cpu())
    dm, dv = (t[0] for t in moments(m, v, s))
    want_m = 0.9 * dm.double() + 0.1 * g.double()
    want_r = (beta2 * dv.double() + (1 - beta2) * g.double() ** 2).sqrt()
    for got, want, most in ((got_m, want_m, 127.0), (got_v.sqrt(), want_r, 255.0)):
        top = float(want.abs().max())
        code = (want.abs() / top).sqrt() * most
        step = top / most ** 2 * (2 * code + 1)
        error = (got.double().mean(0) - want).abs()
        assert bool((error <= 6 * 0.5 * step / count ** 0.5 + 1e-6 * top).all())


def test_a_slow_moment_moves():
    """With beta2 = 0.999 a step moves v by less than half a code; it follows its gradients all the same."""
    n, steps = 4096, 1000
    x, g = torch.zeros(n, device=DEV), torch.full((n,), 2e-3, device=DEV)
    m, v, s = qb.alloc_moments(x, 8)
    v.fill_(255)
    s.view(-1, 2)[:, 1] = 1e-3
    table = qb.AdamWTensors([x], [g], [m], [v], [s])
    for t in range(steps):
        qb.qsdp_adamw_tensors(table, 0.0, 0.9, 0.999, 1e-8, 1.0, 1.0, seed=t)
    want = 1e-6 * 0.999 ** steps + 4e-6 * (1 - 0.999 ** steps)
    got = moments(m.cpu(), v.cpu(), s.cpu())
    # the rounding of sqrt v, at most half a step of 2 / 255 each time, averages over 1 / (1 - beta2) steps and 4096 elements; that of
    # its square adds at most 1000 / (4 * 255^2) ... a hundredth
    assert abs(float(got[1].double().mean()) / want - 1) < 0.02
    assert abs(float(got[0].double().mean()) / 2e-3 - 1) < 1e-3


def test_schedule_seed_and_scale_on_the_device():
    a, b = Model(SIZES, (8, 32), seed=3), Model(SIZES, (8, 32), seed=3)
    h = {k: v for k, v in HYPER.items() if k in ("beta1", "beta2", "eps")}
    schedule = torch.tensor([HYPER["lr"], HYPER["bias1"], HYPER["bias2"]], device=DEV)
    qb.qsdp_adamw_tensors(a.table, **HYPER, seed=12)
    qb.qsdp_adamw_tensors(b.table, lr=1.0, bias1=1.0, bias2=1.0, **h, seed=5, seed_increment=torch.tensor([7], device=DEV),
                          schedule=schedule)
    for name in ("dx", "dm", "dv"):
        assert all(torch.equal(p, q) for p, q in zip(getattr(a, name), getattr(b, name)))
    before = [[t.clone() for t in l] for l in (b.dx, b.dm, b.dv)]
    for bad in (float("inf"), float("nan"), float("-inf")):
        qb.qsdp_adamw_tensors(b.table, **HYPER, grad_scale=torch.tensor([bad], device=DEV))
    assert all(torch.equal(p, q) for old, new in zip(before, (b.dx, b.dm, b.dv)) for p, q in zip(old, new))


@pytest.mark.parametrize("bits", [32, 8])
def test_infinite_gradients_stay_in_their_block(bits):
    n = 1024
    g = torch.full((n,), 1e-3)
    g[5], g[700] = float("inf"), float("nan")
    x = torch.ones(n, device=DEV)
    m, v, s = qb.alloc_moments(x, bits)
    qb.qsdp_adamw_tensors(qb.AdamWTensors([x], [g.to(DEV)], [m], [v], [s]), **HYPER)
    fine = torch.isfinite(x.cpu())
    assert not bool(fine[5]) and not bool(fine[700]) and int((~fine).sum()) == 2
