"""What products in blocks keep of their operands' digits: nothing lost that binary32 sums would hold where the products are exact, and
cuts towards zero, which signed terms take out, where the codes go into the matrix instruction as they are."""
import pytest
import torch

from paper_2302_02390_amd import binding as qb
from train_util import DEV, DTYPES, F8

pytestmark = pytest.mark.gpu


# m, n, k of few rows that reach every one of their kernels: one group of columns, two, parts of a long sum, many columns in one run and two
FEW = [(1, 2048, 2048), (16, 300, 700), (1, 8192, 2048), (16, 8200, 260), (1, 1024, 16384), (7, 700, 3000), (16, 32769, 2048), (5, 33000, 2200)]


@pytest.mark.parametrize("m,n,k", FEW)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_few_rows_keep_what_large_terms_leave(m, n, k, dtype):
    """Every block of 128 has the terms 448 * 448, -448 * 448 and 13 next to each other and no other ones, so that all sums of its
    products are whole numbers below 2^18, which binary32 holds: 13 is left of every block, times scales of 1. The last block of a
    row is as the others or too short for them. Sums of up to 128 thirteens are below 2^11: bf16 rounds them, binary16 does not."""
    x, w = torch.zeros((m, -(-k // 128), 128)), torch.zeros((n, -(-k // 128), 128))
    x[:, :, :3] = torch.tensor([448.0, -448.0, 1.0])
    w[:, :, :3] = torch.tensor([448.0, 448.0, 13.0])
    x, w = x.view(m, -1)[:, :k], w.view(n, -1)[:, :k]
    codes = qb.alloc_blocks(n, k, True, DEV)[:2]
    qb.qsdp_quantize_blocks(w.to(DEV), True, *codes)
    assert bool((codes[1] == 1.0).all())
    y = torch.empty((m, n), dtype=DTYPES[dtype], device=DEV)
    qb.qsdp_linear_blocks(x.to(DTYPES[dtype]).to(DEV), *codes, None, y)
    want = torch.tensor(13.0 * -(-k // 128)).to(y.dtype).float()
    assert bool((y.float().cpu() == want).all()), (y.float().unique().tolist()[:8], float(want))
