"""Rounding to 8-bit floating point in blocks, and products in it, against the definitions."""
import math

import pytest
import torch

from paper_2302_02390_amd import binding as qb
from train_util import DEV, DTYPES, F8, blocks, held, matrix, near, product, to_gpu

pytestmark = pytest.mark.gpu


def _quantized(x, square, dtype=F8):
    """All four outputs for a matrix on the GPU, codes as float32 on the CPU."""
    out = qb.alloc_blocks(*x.shape, square, DEV)
    out = [t.view(dtype) if t.dtype == F8 else t for t in out]
    for t in out:
        t.view(torch.uint8 if t.element_size() == 1 else t.dtype).fill_(85)
    qb.qsdp_quantize_blocks(x, square, *out)
    return [t.view(F8).float().cpu() if t.element_size() == 1 else t.cpu() for t in out]


@pytest.mark.parametrize("rows,cols,pad,offset", [(1, 1, 0, 0), (1, 128, 0, 0), (3, 129, 2, 1), (128, 128, 0, 0), (129, 7, 1, 3),
                                                  (200, 300, 0, 0), (257, 1000, 5, 1), (16, 4096, 0, 0), (1030, 136, 8, 0)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("square", [False, True])
def test_codes_and_scales(rows, cols, pad, offset, dtype, square):
    x = matrix(rows, cols, DTYPES[dtype], pad, offset, rows + cols, 2.0)
    x *= torch.exp(torch.randn((rows, 1), generator=torch.Generator().manual_seed(1)) * 2).to(x.dtype)
    codes, scales, codes_t, scales_t = _quantized(to_gpu(x), square)
    want, of = blocks(x, 128 if square else 1, 128)
    assert torch.equal(codes[:, :cols], want) and bool((codes[:, cols:] == 0).all()) and torch.equal(scales, of.t())
    want, of = blocks(x.t(), 128 if square else 1, 128)
    assert torch.equal(codes_t[:, :rows], want) and bool((codes_t[:, rows:] == 0).all()) and torch.equal(scales_t, of.t())


def test_one_of_both_outputs():
    x = matrix(300, 200, torch.bfloat16, seed=5).to(DEV)
    for square in (False, True):
        whole = _quantized(x, square, torch.uint8)
        codes, scales, codes_t, scales_t = qb.alloc_blocks(300, 200, square, DEV)
        qb.qsdp_quantize_blocks(x, square, codes, scales)
        qb.qsdp_quantize_blocks(x, square, None, None, codes_t, scales_t)
        for got, want in zip((codes, scales, codes_t, scales_t), whole):
            assert torch.equal(got.float().cpu(), want)


def test_every_value_of_the_formats_rounds_as_defined():
    """All bf16 and binary16 numbers in blocks whose largest is a power of two times 448, so that codes are ties and neighbours."""
    for dtype in (torch.bfloat16, torch.float16):
        every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype)
        every = every[torch.isfinite(every)]
        for top in (448.0, 1.0, 300.0):
            here = every[every.abs() <= top]
            x = torch.zeros((-(-here.numel() // 127), 128), dtype=dtype)
            x[:, 0] = top
            x[:, 1:].reshape(-1)
            x[:, 1:] = torch.nn.functional.pad(here, (0, x.shape[0] * 127 - here.numel())).view(-1, 127)
            codes, scales, _, _ = _quantized(x.to(DEV), False)
            want, of = blocks(x, 1, 128)
            assert torch.equal(codes, want) and torch.equal(scales, of.t())


def test_tiny_blocks_and_what_is_no_number():
    x = matrix(6, 256, torch.float32, seed=2)
    x[0, :128] *= 1e-38
    x[1, :128] = 0.0
    x[2, 5] = math.nan
    x[3, 130] = math.inf
    x[4, 131] = -math.inf
    codes, scales, codes_t, scales_t = _quantized(x.to(DEV), False)
    want, of = blocks(x, 1, 128)
    assert torch.equal(codes.nan_to_num(9e3), want.nan_to_num(9e3)) and torch.equal(scales, of.t())
    assert bool(codes[2, 5].isnan()) and bool(codes[3, 130].isnan()) and math.isinf(float(scales[1, 3]))
    # products: NaN in the rows that hold one, the others as without
    b = matrix(70, 256, torch.float32, seed=3, std=0.1)
    bc = qb.alloc_blocks(70, 256, True, DEV)
    qb.qsdp_quantize_blocks(b.to(DEV), True, *bc)
    for dtype in (torch.float32, torch.bfloat16):
        y = torch.empty((6, 70), dtype=dtype, device=DEV)
        qb.qsdp_linear_blocks(x.to(DEV), bc[0], bc[1], None, y)
        assert bool(y[[2, 3, 4]].isnan().all())
        fine = [0, 1, 5]
        hb = held(bc[0].float().cpu(), bc[1].cpu().t(), 128, 128)
        w, off = product(held(want, of, 1, 128)[fine], hb, dtype == torch.float32)
        assert near(y[fine], w, off)


def _operands(m, n, k, square, seed=0):
    a, b = matrix(m, k, torch.bfloat16, seed=seed), matrix(n, k, torch.bfloat16, seed=seed + 1, std=0.05)
    a *= torch.exp(torch.randn((m, 1), generator=torch.Generator().manual_seed(seed))).to(a.dtype)
    ac, bc = qb.alloc_blocks(m, k, False, DEV)[:2], qb.alloc_blocks(n, k, square, DEV)[:2]
    qb.qsdp_quantize_blocks(a.to(DEV), False, *ac)
    qb.qsdp_quantize_blocks(b.to(DEV), square, *bc)
    ha = held(ac[0].float()[:, :k], ac[1].t(), 1, 128)  # on the GPU, where products in 64 bits are quick
    hb = held(bc[0].float()[:, :k], bc[1].t(), 128 if square else 1, 128)
    return a, ac, bc, ha, hb


# m, n, k of products that reach every kernel
SMALL = [(1, 1, 1), (1, 64, 128), (3, 65, 129), (16, 100, 300), (17, 63, 127), (1, 2048, 2048), (16, 8200, 260), (5, 32805, 130),
         (2, 40, 5000), (3, 8195, 4200), (4, 700, 3000), (16, 32769, 4096), (7, 33000, 2200), (3, 1001, 6300), (16, 300, 16390),
         (33, 4097, 640), (64, 64, 1024), (65, 127, 513), (130, 129, 256), (200, 1000, 2048), (513, 300, 4096), (200, 130, 8200),
         (1000, 1024, 384), (1540, 1490, 650)]
LARGE = [(1930, 1950, 100), (1921, 1921, 200), (1920, 2000, 300), (1930, 1950, 1030), (3850, 3830, 1030), (3850, 3830, 4100), (3841, 3841, 4353)]
PRODUCTS = SMALL + LARGE


@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("square", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_products(m, n, k, square, dtype):
    if (m, n, k) in LARGE and dtype == "f16":
        pytest.skip("the large ones in two formats")
    _, ac, bc, ha, hb = _operands(m, n, k, square, m + n + k)
    bias = matrix(1, n, torch.float32, seed=8)[0]
    want, off = (t.cpu() for t in product(ha, hb, dtype == "f32"))
    y = torch.full((m, n + 3), 2.0, dtype=DTYPES[dtype], device=DEV)
    qb.qsdp_matmul_blocks(*ac, *bc, k, bias.to(DEV), y[:, :n])
    assert bool((y[:, n:] == 2.0).all())
    assert near(y[:, :n], want + bias, off + 1e-7 * (want.abs() + bias.abs()))
    if dtype != "f16":
        old = matrix(m, n, DTYPES[dtype], seed=4)
        y = old.to(DEV)
        room = torch.empty(qb.matmul_blocks_bytes(m, n, k), dtype=torch.uint8, device=DEV)
        qb.qsdp_matmul_blocks(*ac, *bc, k, None, y, True, room)
        assert near(y, want + old, off + 1e-7 * (want.abs() + old.abs()))


@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("bf16", "f16")])
def test_linear(m, n, k, dtype, out):
    x = matrix(m, k, DTYPES[dtype], 3, 1, m + n, 2.0)
    _, _, bc, _, hb = _operands(1, n, k, True, 3)
    bias = matrix(1, n, torch.float32, seed=8)[0]
    if (m, n, k) in LARGE and dtype == "f16":
        pytest.skip("the large ones in three formats")
    want, off = (t.cpu() for t in product(held(*blocks(x, 1, 128), 1, 128).to(DEV), hb, out == "f32"))
    flat = torch.full((m * (n + 5) + 1,), 2.0, dtype=DTYPES[out], device=DEV)
    y = flat[1:].view(m, n + 5)
    qb.qsdp_linear_blocks(to_gpu(x), *bc, bias.to(DEV), y[:, :n])
    assert bool((y[:, n:] == 2.0).all())
    assert near(y[:, :n], want + bias, off + 1e-7 * (want.abs() + bias.abs()))


@pytest.mark.parametrize("m,n,k", [(300, 500, 260), (130, 1000, 700)])
def test_gradients_of_a_product(m, n, k):
    """y, dx and dw of one layer from the codes both ways round, against the held values."""
    x, w, dy = (matrix(r, c, torch.bfloat16, seed=i, std=s) for i, (r, c, s) in enumerate(((m, k, 1), (n, k, .05), (m, n, .01))))
    xq, dq, wq = qb.alloc_blocks(m, k, False, DEV), qb.alloc_blocks(m, n, False, DEV), qb.alloc_blocks(n, k, True, DEV)
    for t, square, to in ((x, False, xq), (dy, False, dq), (w, True, wq)):
        qb.qsdp_quantize_blocks(t.to(DEV), square, *to)
    y, dx = torch.empty((m, n), dtype=torch.bfloat16, device=DEV), torch.empty((m, k), dtype=torch.bfloat16, device=DEV)
    dw = torch.empty((n, k), device=DEV)
    qb.qsdp_matmul_blocks(*xq[:2], *wq[:2], k, None, y)
    qb.qsdp_matmul_blocks(*dq[:2], *wq[2:], n, None, dx)
    qb.qsdp_matmul_blocks(*dq[2:], *xq[2:], m, None, dw)
    hw = held(*blocks(w, 128, 128), 128, 128)
    for got, a, b, exact in ((y, held(*blocks(x, 1, 128), 1, 128), hw, False), (dx, held(*blocks(dy, 1, 128), 1, 128), hw.t(), False),
                             (dw, held(*blocks(dy.t(), 1, 128), 1, 128), held(*blocks(x.t(), 1, 128), 1, 128), True)):
        want, off = product(a, b.contiguous(), exact)
        assert near(got, want, off)


def test_no_rows():
    w = qb.alloc_blocks(50, 130, True, DEV)
    qb.qsdp_quantize_blocks(torch.ones((50, 130), device=DEV), True, *w)
    x, y = torch.empty((0, 130), device=DEV), torch.empty((0, 50), device=DEV)
    q = qb.alloc_blocks(0, 130, False, DEV)
    qb.qsdp_quantize_blocks(x, False, *q)
    qb.qsdp_matmul_blocks(*q[:2], *w[:2], 130, None, y)
    qb.qsdp_linear_blocks(x, *w[:2], None, y)
