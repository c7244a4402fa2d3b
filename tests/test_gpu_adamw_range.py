"""AdamW over many tensors where a finite gradient's square passes the largest number: weights stay finite, as the formula has it."""
import numpy as np
import pytest
import torch

from paper_2302_02390_amd import binding as qb
from train_util import DEV, DTYPES, adamw, by_256, codes_of, fma, moments, near, philox

pytestmark = pytest.mark.gpu

HYPER = dict(beta1=0.9, beta2=0.95, eps=1e-8, bias1=1 - 0.9 ** 3, bias2=1 - 0.95 ** 3)


def _second(v32, numbers, seed):
    """Codes and R of a second moment, an infinite root being 2^64."""
    counter = np.zeros((len(numbers), 4), dtype=np.uint64)
    counter[:, 0], counter[:, 2] = numbers, 3
    root = by_256(v32.double().sqrt().float().clamp(max=2.0 ** 64))
    d, top = codes_of(root, philox(counter, seed)[:, 1], 255)
    return torch.where((root > 0) & (top > 0), d.clamp(min=1.0), d).reshape(-1)[:v32.numel()].to(torch.uint8), top[:, 0]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("large", [9e19, 1e25, -3e38])
@pytest.mark.parametrize("tiny", [False, True])
def test_a_square_that_overflows(bits, dtype, large, tiny):
    """In one element of the first block and one of the last of 900; `tiny` leaves zeros beside them. Three steps, ordinary gradients
    after the first."""
    n = 900
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(n, generator=gen) * 0.02
    m, v, s = qb.alloc_moments(x, bits)
    dx, dm, dv, ds = (None if t is None else t.to(DEV) for t in (x, m, v, s))
    dg = torch.empty(n, dtype=DTYPES[dtype], device=DEV)
    table = qb.AdamWTensors([dx], [dg], [dm], [dv], [ds], weight_decay=0.1)
    for step in range(3):
        g = torch.randn(n, generator=gen) * 1e-2
        if tiny:
            g[10:20] = g[800:805] = 0.0
        if step == 0:
            g[5] = g[880] = large
        dg.copy_(g)
        g = dg.cpu()
        qb.qsdp_adamw_tensors(table, 1e-2, **HYPER, seed=step)
        v32 = (v if s is None else moments(m, v, s)[1].reshape(-1)[:n])
        want, off, m1, v1, s1 = adamw(x, g, m, v, s, 0, step, 1e-2, decay=0.1, **HYPER)
        assert bool(torch.isfinite(want).all()) and bool(torch.isfinite(dx).all())
        assert near(dx, want, off), step
        assert torch.equal(dm.cpu(), m1)
        if s is not None:
            b2 = torch.tensor(HYPER["beta2"])
            v1, top = _second(fma(b2, v32, ((1 - b2) * g.float()) * g.float()), np.arange(4), step)
            s1 = s1.view(4, 2).clone()
            s1[:, 1] = top
            s1 = s1.reshape(-1)
            assert torch.equal(ds.cpu(), s1) and s1.view(4, 2)[[0, 3], 1].tolist() == [2.0 ** 64] * 2 and v1[[5, 880]].tolist() == [255, 255]
        assert torch.equal(dv.cpu(), v1)
        x, m, v, s = dx.cpu(), m1, v1, s1
