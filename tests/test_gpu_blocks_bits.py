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


def _rounded(x, square=False):
    codes = qb.alloc_blocks(*x.shape, square, DEV)[:2]
    qb.qsdp_quantize_blocks(x.to(DEV), square, *codes)
    return codes


# m, n, k of many rows, one of each kind of tile and a sum in parts
MANY = [(200, 300, 520), (1930, 1950, 260), (3850, 3830, 1030), (700, 3000, 128), (64, 70, 8200)]


@pytest.mark.parametrize("m,n,k", MANY)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_what_is_cut_off_is_cut_towards_zero(m, n, k, dtype):
    """448 * 448 has its first bit at 2^17, so 13 beside it and its negative may lose what lies below 2^3: every block keeps 5 to 13
    of it, and -13 keeps the same, negative. Binary32 results keep all."""
    room = torch.empty(max(16, qb.matmul_blocks_bytes(m, n, k)), dtype=torch.uint8, device=DEV)
    x = torch.zeros((m, -(-k // 128), 128))
    x[:, :, :3] = torch.tensor([448.0, -448.0, 1.0])
    a, blocks = _rounded(x.view(m, -1)[:, :k].contiguous()), -(-k // 128)
    got = {}
    for sign in (1.0, -1.0):
        w = torch.zeros((n, blocks, 128))
        w[:, :, :3] = torch.tensor([448.0, 448.0, 13.0 * sign])
        b = _rounded(w.view(n, -1)[:, :k].contiguous())
        for to in (dtype, "f32"):
            y = torch.empty((m, n), dtype=DTYPES[to], device=DEV)
            qb.qsdp_matmul_blocks(*a, *b, k, None, y, False, room)
            got[to, sign] = y.float()
        assert bool((got["f32", sign] == 13.0 * sign * blocks).all())
        size, half = got[dtype, sign] * sign, 13.0 * blocks * torch.finfo(DTYPES[dtype]).eps / 2
        assert bool((size >= 5.0 * blocks - half).all()) and bool((size <= 13.0 * blocks + half).all())
    assert torch.equal(got[dtype, 1.0], -got[dtype, -1.0])


@pytest.mark.parametrize("k", [1024, 65536])
def test_signed_terms_take_the_cuts_out(k):
    """Each product of normal operands is cut by less than 2^-14 of the largest of eight, whose square is (2.6)^2 times a product's in the
    mean, towards zero, so with either sign alike: 2^-14 * 2.6 / sqrt 3 = 9.2e-5 of the norm at most, for any k, beside the rounding's
    2.07e-4: together less than 1.1 times the rounding alone. Cuts to one side would add up, to 3e-4 at 65536."""
    m = n = 512
    gen = torch.Generator(DEV).manual_seed(k)
    a, b = (torch.randn((r, k), device=DEV, generator=gen) for r in (m, n))
    a, b = _rounded(a), _rounded(b)
    held = lambda t: (t[0].double().view(m, -1, 128) * t[1].t().double()[:, :, None]).view(m, k)
    want = held(a) @ held(b).t().contiguous()
    y = torch.empty((m, n), dtype=torch.float16, device=DEV)
    qb.qsdp_matmul_blocks(*a, *b, k, None, y)
    assert float((y.double() - want).norm()) <= 1.1 * float((want.half().double() - want).norm())


@pytest.mark.parametrize("m", [1, 200])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("square", [False, True])
def test_blocks_of_the_least_and_the_largest_scales(m, dtype, square):
    """Largest values whose products are 2^-108 and 2^144, the limits that are stated. A scale is 2^e / 448 rounded, two of them and
    their product: three roundings of 2^-24; codes 448 (first case) or 0.875 (second) are exact."""
    n, k = 130, 256
    for x, w, each in ((torch.full((m, k), 2.0 ** -54), torch.full((n, k), 2.0 ** -54), 128 * 2.0 ** -108),
                       (torch.tensor([2.0 ** 72, 2.0 ** 63, 0.0]), torch.tensor([0.0, 2.0 ** 62, 2.0 ** 72]), 2.0 ** 125)):
        if x.dim() == 1:
            few, (x, w) = (x, w), (torch.zeros((r, 2, 128)) for r in (m, n))
            x[:, :, :3], w[:, :, :3] = few
            x, w = x.view(m, k), w.view(n, k)
        a, b = _rounded(x), _rounded(w, square)
        y = torch.empty((m, n), dtype=DTYPES[dtype], device=DEV)
        qb.qsdp_matmul_blocks(*a, *b, k, None, y)
        ys = [y]
        if square:
            ys.append(torch.empty_like(y))
            qb.qsdp_linear_blocks(x.to(DEV), *b, None, ys[1])
        for y in ys:  # two blocks: their sum and its rounding to the format
            off = (3 + 1) * 2.0 ** -24 + torch.finfo(y.dtype).eps / 2
            assert bool(((y.double() / (2 * each) - 1).abs() <= off).all()), (float(y[0, 0]), 2 * each)
