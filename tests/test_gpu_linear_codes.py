"""Tokens rounded to 8 bits times weights held as packed 8-bit codes: codes, scales and sums exactly, products against the
64-bit definition."""
import math

import pytest
import torch

import lm_util as lu
from paper_2302_02390_amd import binding as qb

pytestmark = pytest.mark.gpu


def weights(n, k, bucket, seed):
    """Codes uint8 [n, whole buckets] (anything past k) and meta [n, buckets, 2] of uneven buckets."""
    gen = torch.Generator().manual_seed(seed)
    buckets = -(-k // bucket)
    codes = torch.randint(0, 256, (n, buckets * bucket), generator=gen, dtype=torch.uint8)
    scale = torch.rand((n, buckets), generator=gen) * 1e-3 + 1e-5
    base = -128.0 * scale * (0.5 + torch.rand((n, buckets), generator=gen))
    return codes, torch.stack([base, scale], 2)


def make_x(m, k, dtype, seed, pad=0, offset=0):
    x = lu.make_rows(m, k, dtype, pad, seed, 1.0, offset)
    return x


def run(x, codes, meta, bucket, bias, out, pad=0, two=False):
    (m, k), n = x.shape, meta.shape[0]
    full = torch.full((m, n + pad), 3.0, dtype=out, device=lu.DEV)
    y = full[:, :n]
    wcodes, wmeta = codes.to(lu.DEV).view(torch.int32), meta.to(lu.DEV)
    bias = None if bias is None else bias.to(lu.DEV)
    if two:
        c = torch.full((m, -(-k // 128) * 128), 99, dtype=torch.int8, device=lu.DEV)
        s = torch.empty(m, device=lu.DEV)
        sums = torch.empty((m, meta.shape[1]), device=lu.DEV)
        qb.qsdp_quantize_tokens(x, bucket, c, s, sums)
        qb.qsdp_matmul_codes(c, s, sums, wcodes, wmeta, n, k, bucket, bias, y)
    else:
        ws = torch.full((qb.tokens_bytes(m, k, bucket),), 0xA5, dtype=torch.uint8, device=lu.DEV)
        qb.qsdp_linear_codes(x, wcodes, wmeta, n, bucket, bias, y, ws)
    assert bool((full[:, n:] == 3.0).all())
    return y


def check(m, n, k, bucket, dtype="bf16", out="bf16", bias=False, pad=0, offset=0, seed=0, x=None):
    x = make_x(m, k, lu.DTYPES[dtype], seed, pad, offset) if x is None else x
    codes, meta = weights(n, k, bucket, seed + 1)
    b = torch.randn(n, generator=torch.Generator().manual_seed(seed + 2)) if bias else None
    scale, q, sums = lu.tokens8(x, bucket)
    want, off = lu.product(scale, q, sums, codes, meta, b, bucket)
    xg = lu.to_gpu(x)
    y = run(xg, codes, meta, bucket, b, lu.DTYPES[out], pad)
    assert lu.near(y, want, off)
    assert torch.equal(run(xg, codes, meta, bucket, b, lu.DTYPES[out], 0, two=True).nan_to_num(5.5), y.nan_to_num(5.5))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("k,bucket", [(1, 32), (31, 32), (33, 64), (127, 128), (128, 128), (129, 160), (768, 256),
                                      (1000, 1024), (1000, 8192), (4096, 1024), (8192, 8192), (9001, 128), (20000, 4096)])
def test_tokens(k, bucket, dtype):
    x = make_x(5, k, lu.DTYPES[dtype], k, 3, 1)
    x[1] = 0.0
    x[2, k // 2] = math.inf
    x[3, 0] = math.nan
    x[4] = torch.linspace(-1, 1, k).to(x.dtype) if k > 1 else x[4]
    buckets = -(-k // bucket)
    pitch = -(-k // 128) * 128
    codes = torch.full((5, pitch), 99, dtype=torch.int8, device=lu.DEV)
    scale, sums = torch.empty(5, device=lu.DEV), torch.empty((5, buckets), device=lu.DEV)
    qb.qsdp_quantize_tokens(lu.to_gpu(x), bucket, codes, scale, sums)
    s, q, total = lu.tokens8(x, bucket)
    assert torch.equal(scale.cpu().nan_to_num(-1), s.nan_to_num(-1))
    assert torch.equal(codes[:, :k].cpu().long(), q) and bool((codes[:, k:] == 0).all())
    assert torch.equal(sums.cpu().long(), total)


@pytest.mark.parametrize("m", [1, 2, 3, 8, 15, 16, 17, 31, 33, 64, 65, 100, 127, 129, 255, 257])
@pytest.mark.parametrize("n,k", [(1, 32), (15, 100), (17, 64), (129, 1000), (300, 512), (513, 2048)])
def test_shapes(m, n, k):
    bucket = -(-k // 32) * 32
    check(m, n, k, bucket, ["bf16", "f16", "f32"][(m + n) % 3], ["f32", "bf16", "f16"][(m + k) % 3], bias=m % 2 == 0,
          pad=m % 4, offset=n % 3, seed=m)


@pytest.mark.parametrize("m", [1, 7, 48, 130, 300])
@pytest.mark.parametrize("n,k,bucket", [(65, 256, 128), (130, 2048, 1024), (40, 2000, 1024), (257, 1152, 384), (70, 8192, 1024),
                                        (33, 4096, 4096), (64, 20000, 8192), (48, 600, 8192)])
def test_buckets(m, n, k, bucket):
    check(m, n, k, bucket, "bf16", "f32", bias=n % 2 == 0, seed=k + m)


@pytest.mark.parametrize("m", [33, 100, 200])
@pytest.mark.parametrize("n,k,bucket", [(130, 2047, 2048), (130, 2049, 2080), (63, 2176, 128), (100, 2177, 128), (66, 3200, 640),
                                        (66, 5000, 1024), (5, 5000, 8192), (2000, 2500, 2560)])
def test_teams_that_share_a_tile(m, n, k, bucket):
    """Few tiles and long sums: teams take runs of steps that are not equally long and end inside a bucket."""
    check(m, n, k, bucket, "bf16", "f32", bias=n % 2 == 0, seed=k + m)


@pytest.mark.parametrize("m", [2, 40, 200])
def test_rows_of_zeros_nan_and_infinity(m):
    x = make_x(m, 500, torch.float32, 3)
    x[0] = 0.0
    x[-1, 499] = math.nan
    if m > 2:
        x[1, 0] = -math.inf
        x[2] = torch.finfo(torch.float32).max
        x[3] *= 1e-38
        x[4] = 1e-45  # its 127th part is zero
    check(m, 100, 500, 512, "f32", "f32", x=x, bias=True)


@pytest.mark.parametrize("m", [1, 64, 512])
def test_extreme_codes(m):
    """Every product at its largest: |D| = 127 * 128 * 8192 needs 28 bits."""
    for k, bucket in ((8192, 8192), (16384, 8192)):
        x = torch.ones((m, k))
        codes = torch.zeros((80, k), dtype=torch.uint8)
        codes[1::2] = 255
        meta = torch.tensor([[-1.0, 2.0 / 255]]).repeat(80, k // bucket, 1)
        scale, q, sums = lu.tokens8(x, bucket)
        want, off = lu.product(scale, q, sums, codes, meta, None, bucket)
        assert lu.near(run(x.to(lu.DEV), codes, meta, bucket, None, torch.float32), want, off)


@pytest.mark.parametrize("m", [1, 24, 96, 260])
def test_with_the_codec(m):
    """Weights encoded by the codec, a bucket per channel, against the product with what it decodes."""
    n, k = 384, 768
    w = 0.02 * torch.randn((n, k), device=lu.DEV, generator=torch.Generator(lu.DEV).manual_seed(1))
    codes, meta = qb.alloc_packed(n * k, 8, k, lu.DEV)
    qb.qsdp_quantize_weight(w.view(-1), 8, k, 0.0, 5, codes, meta.view(-1))
    decoded = torch.empty(n * k, device=lu.DEV)
    qb.qsdp_dequantize(codes, meta.view(-1), n * k, 8, k, decoded)
    x = torch.randn((m, k), device=lu.DEV, generator=torch.Generator(lu.DEV).manual_seed(2))
    y = torch.empty((m, n), device=lu.DEV)
    qb.qsdp_linear_codes(x, codes, meta.view(-1), n, k, None, y)
    scale, q, _ = lu.tokens8(x.cpu(), k)
    want = scale.double()[:, None] * (q.double() @ decoded.cpu().double().view(n, k).t())
    # decoded weights are rounded once more than the product's: 2^-24 of each
    off = scale.double()[:, None] * (q.double().abs() @ decoded.cpu().double().view(n, k).abs().t()) * 4 * lu.EPS
    codes8 = codes.cpu().view(torch.uint8).view(n, k)
    off = off + lu.product(scale, q, lu.tokens8(x.cpu(), k)[2], codes8, meta.cpu().view(n, 1, 2), None, k)[1]
    assert lu.near(y, want, off)
    # 8 bits on both sides: a relative error of about a hundredth against the full-precision product
    full = x.cpu().double() @ w.cpu().double().t()
    assert float((y.cpu() - full).norm() / full.norm()) < 0.02


def test_long_channel_offsets():
    """Codes and outputs beyond 2^32 bytes: 600,000 channels of 8192 codes."""
    n, k, m = 600_000, 8192, 3
    codes = torch.randint(-2 ** 31, 2 ** 31 - 1, (n * k // 4,), dtype=torch.int32, device=lu.DEV)
    meta = torch.tensor([-1.0, 2.0 / 255], device=lu.DEV).repeat(n, 1)
    x = torch.randn((m, k), device=lu.DEV)
    y = torch.empty((m, n), device=lu.DEV)
    qb.qsdp_linear_codes(x, codes, meta, n, k, None, y)
    rows = torch.tensor([0, 1, 17, 300_000, 524_287, 524_288, 524_289, n - 1])
    part = codes.view(n, k // 4)[rows.to(lu.DEV)].cpu().view(torch.uint8)
    scale, q, sums = lu.tokens8(x.cpu(), k)
    want, off = lu.product(scale, q, sums, part, meta.cpu()[rows].view(-1, 1, 2), None, k)
    assert lu.near(y[:, rows.to(lu.DEV)], want, off)


def test_streams_graphs_and_empty_batches():
    codes, meta = weights(200, 512, 512, 3)
    wcodes, wmeta = codes.to(lu.DEV).view(torch.int32), meta.to(lu.DEV)
    for m in (1, 40, 300):
        x = make_x(m, 512, torch.bfloat16, 3).to(lu.DEV)
        y = torch.empty((m, 200), dtype=torch.bfloat16, device=lu.DEV)
        ws = torch.empty(qb.tokens_bytes(m, 512, 512), dtype=torch.uint8, device=lu.DEV)
        step = lambda: qb.qsdp_linear_codes(x, wcodes, wmeta, 200, 512, None, y, ws)  # noqa: E731
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for seed in (1, 2, 3):
            x.copy_(make_x(m, 512, torch.bfloat16, seed))
            step()
            torch.cuda.synchronize()
            want = y.clone()
            y.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            y2 = torch.empty_like(y)
            qb.qsdp_linear_codes(x, wcodes, wmeta, 200, 512, None, y2)
        side.synchronize()
        assert torch.equal(y2, want)
    qb.qsdp_linear_codes(x[:0], wcodes, wmeta, 200, 512, None, y[:0], ws)


def test_refusals_of_the_binding():
    codes, meta = weights(20, 512, 512, 3)
    wcodes, wmeta = codes.to(lu.DEV).view(torch.int32), meta.to(lu.DEV)
    x, y = torch.zeros((3, 512), device=lu.DEV), torch.zeros((3, 20), device=lu.DEV)
    ws = torch.empty(qb.tokens_bytes(3, 512, 512), dtype=torch.uint8, device=lu.DEV)
    call = qb.qsdp_linear_codes
    with pytest.raises(ValueError):
        call(x, wcodes, wmeta, 21, 512, None, torch.zeros((3, 21), device=lu.DEV), ws)   # codes too short
    with pytest.raises(ValueError):
        call(x, wcodes, wmeta[:19], 20, 512, None, y, ws)
    with pytest.raises(ValueError):
        call(x, wcodes, wmeta, 20, 512, torch.zeros(19, device=lu.DEV), y, ws)
    with pytest.raises(ValueError):
        call(x, wcodes, wmeta, 20, 512, None, y[:2], ws)
    with pytest.raises(TypeError):
        call(x.double(), wcodes, wmeta, 20, 512, None, y, ws)
    with pytest.raises(TypeError):
        call(x, wcodes.view(torch.uint8), wmeta, 20, 512, None, y, ws)
    with pytest.raises(qb.QsdpError):
        call(x, wcodes, wmeta, 20, 512, None, y, ws[:-16])                                # workspace too short
    with pytest.raises(qb.QsdpError):
        call(x, wcodes, wmeta, 20, 512, None, y, torch.empty(ws.numel() + 1, dtype=torch.uint8, device=lu.DEV)[1:])
    for bucket in (0, 16, 100, 8224, 96, 160):   # not the codec's, or several to a channel and not of whole steps
        with pytest.raises((qb.QsdpError, ValueError)):
            call(x, wcodes, wmeta, 20, bucket, None, y, ws)
