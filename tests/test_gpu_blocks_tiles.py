"""Products whose tiles are wider than the matrix in one direction or both: rows and columns behind it are copies that nobody stores."""
import pytest
import torch

from paper_2302_02390_amd import binding as qb
from train_util import DEV, DTYPES, held, matrix, near, product

pytestmark = pytest.mark.gpu

# m, n, k, the tile of results in 16 bits and of those in binary32 (test_train_tiles asks the plan)
CASES = [(17, 28700, 300, "T128", "T128"), (64, 50257, 260, "T128", "T128"), (28700, 17, 300, "T128", "T128"),
         (150, 57200, 1030, "T256", "T128"), (57200, 130, 1100, "T256", "T128"), (17, 3, 129, "T64_4", "T64"), (17, 20000, 200, "T64_4", "T64"),
         (33, 28500, 140, "T64_4", "T64"), (2, 28700, 300, "T128", "T128")]


@pytest.mark.parametrize("m,n,k", [c[:3] for c in CASES])
@pytest.mark.parametrize("square", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_products(m, n, k, square, dtype):
    a, b = matrix(m, k, torch.bfloat16, seed=m), matrix(n, k, torch.bfloat16, seed=n, std=0.05)
    ac, bc = qb.alloc_blocks(m, k, False, DEV)[:2], qb.alloc_blocks(n, k, square, DEV)[:2]
    qb.qsdp_quantize_blocks(a.to(DEV), False, *ac)
    qb.qsdp_quantize_blocks(b.to(DEV), square, *bc)
    ha, hb = held(ac[0].float()[:, :k], ac[1].t(), 1, 128), held(bc[0].float()[:, :k], bc[1].t(), 128 if square else 1, 128)
    want, off = (t.cpu() for t in product(ha, hb, dtype == "f32"))
    flat = torch.full((m + 1, n + 3), 2.0, dtype=DTYPES[dtype], device=DEV)
    y = flat[:m, :n]
    qb.qsdp_matmul_blocks(*ac, *bc, k, None, y)
    assert near(y, want, off)
    first = y.clone()
    qb.qsdp_matmul_blocks(*ac, *bc, k, None, y, True)
    assert near(y, want + first.cpu().double(), off)
    if square and m > 16:
        qb.qsdp_linear_blocks(a.to(DEV), *bc, None, y)
        assert torch.equal(y, first) or qb.matmul_blocks_bytes(m, n, k) and near(y, want, off)
    assert bool((flat[m:] == 2.0).all()) and bool((flat[:, n:] == 2.0).all())
