"""Every kernel that the plan of the operators on logits and on packed weights chooses among (csrc/lm/lm_plan.hpp), at sizes that
reach it with ragged edges, against the 64-bit definitions. tests/test_lm_plan.py holds the choices to those named here."""
import math

import pytest
import torch

import lm_util as lu
from paper_2302_02390_amd import binding as qb
from test_gpu_distill import lists
from test_gpu_linear_codes import make_x, run, weights
from test_gpu_scoring import full_workspace, run_score

pytestmark = pytest.mark.gpu

# kernel, m, n, k, bucket
PRODUCTS = [
    ("FEW_16_8", 7, 8191, 1000, 1024), ("FEW_16_8", 16, 333, 2048, 128),
    ("FEW_16_4", 3, 9001, 1000, 1024), ("FEW_16_4", 16, 8193, 2048, 1024), ("FEW_16_4", 13, 20001, 640, 128),
    ("FEW_16_4", 1, 32768, 300, 320),
    ("FEW_32_8", 31, 4095, 700, 704), ("FEW_32_8", 17, 100, 1280, 128),
    ("FEW_32_4", 20, 5001, 1000, 1024), ("FEW_32_4", 17, 4097, 2048, 1024), ("FEW_32_4", 29, 9999, 768, 256),
    ("TILE_64_TEAMS", 65, 2001, 2048, 1024), ("TILE_64_TEAMS", 130, 999, 2900, 128),
    ("TILE_64_DEEP", 100, 3000, 600, 640), ("TILE_64_DEEP", 700, 1500, 1000, 1024), ("TILE_64_DEEP", 700, 1501, 1024, 512),
    ("TILE_64", 1031, 4099, 1000, 1024), ("TILE_64", 1000, 4099, 384, 128),
    ("TILE_128", 700, 3001, 1000, 1024), ("TILE_128", 1500, 4001, 2048, 1024), ("TILE_128", 1500, 4003, 1152, 384),
    ("TILE_256", 4000, 8191, 100, 128), ("TILE_256", 3000, 5003, 777, 800),
]


@pytest.mark.parametrize("kernel,m,n,k,bucket", PRODUCTS)
def test_products(kernel, m, n, k, bucket):
    x = make_x(m, k, torch.bfloat16, m + k, 1, n % 2)
    codes, meta = weights(n, k, bucket, n)
    bias = torch.randn(n, generator=torch.Generator().manual_seed(n + 1))
    scale, q, sums = lu.tokens8(x, bucket)
    for b in (bias, None):
        want, off = lu.product(scale, q, sums, codes, meta, b, bucket)
        for out in ("f32", "bf16", "f16") if b is not None else ("bf16",):
            assert lu.near(run(lu.to_gpu(x), codes, meta, bucket, b, lu.DTYPES[out], pad=3), want, off), out


def test_more_tiles_than_a_launch_holds():
    """2^19 channel tiles of 128 by three of tokens, in two launches; outputs of 40 GB."""
    n, k, m = 1 << 26, 32, 300
    gen = torch.Generator(lu.DEV).manual_seed(1)
    codes = torch.randint(-2 ** 31, 2 ** 31 - 1, (n * k // 4,), dtype=torch.int32, device=lu.DEV, generator=gen)
    meta = torch.tensor([-1.0, 2.0 / 255], device=lu.DEV).repeat(n, 1)
    x = torch.randn((m, k), device=lu.DEV, generator=gen)
    y = torch.empty((m, n), dtype=torch.bfloat16, device=lu.DEV)
    qb.qsdp_linear_codes(x, codes, meta, n, k, None, y)
    at = torch.tensor([0, 1, 127, 128, 5_000_001, n // 2 - 1, n // 2, n - 129, n - 1])
    part = codes.view(n, k // 4)[at.to(lu.DEV)].cpu().view(torch.uint8)
    scale, q, sums = lu.tokens8(x.cpu(), k)
    want, off = lu.product(scale, q, sums, part, meta[at.to(lu.DEV)].cpu().view(-1, 1, 2), None, k)
    assert lu.near(y[:, at.to(lu.DEV)], want, off)


def test_more_tokens_than_a_launch_holds():
    m, n, k = (1 << 20) + 3, 40, 40
    x = make_x(m, k, torch.bfloat16, 5)
    codes, meta = weights(n, k, 64, 6)
    scale, q, sums = lu.tokens8(x, 64)
    want, off = lu.product(scale, q, sums, codes, meta, None, 64)
    assert lu.near(run(x.to(lu.DEV), codes, meta, 64, None, torch.float32), want, off)


def test_channels_encoded_as_tensors():
    """Channels of 1000 weights, each a tensor of its own to the codec: a bucket of 1024 with slots that are not used."""
    n, k, bucket, m = 70, 1000, 1024, 40
    w = 0.02 * torch.randn((n, k), device=lu.DEV, generator=torch.Generator(lu.DEV).manual_seed(3))
    table = qb.Segments([k] * n, bucket, lu.DEV)
    codes, meta = table.alloc_packed(8)
    codes.fill_(-1)
    qb.qsdp_quantize_weight_segmented(w.view(-1), table, 8, 0.0, 5, codes, meta.view(-1))
    x = make_x(m, k, torch.float32, 4)
    y = torch.empty((m, n), device=lu.DEV)
    qb.qsdp_linear_codes(x.to(lu.DEV), codes, meta.view(-1), n, bucket, None, y)
    scale, q, sums = lu.tokens8(x, bucket)
    want, off = lu.product(scale, q, sums, codes.cpu().view(torch.uint8).view(n, bucket), meta.cpu().view(n, 1, 2), None, bucket)
    assert lu.near(y, want, off)
    full = x.double() @ w.cpu().double().t()
    assert float((y.cpu() - full).norm() / full.norm()) < 0.02


# ---- rows ------------------------------------------------------------------------------------------------------------------
# format -> the longest rows of each team, and the team for rows that are one longer: whether four workgroups share a unit or not
LIMITS = {
    "f32": [(1024, "T128"), (8192, "T256"), (16384, "T512"), (25344, "T512_LDS"), (32768, "T1024"), (51968, "T1024_LDS")],
    "16": [(2047, "T128"), (16383, "T256"), (32767, "T512"), (50687, "T512_LDS"), (65535, "T1024"), (103935, "T1024_LDS")],
}


def limits(dtype):
    return LIMITS["f32" if dtype == "f32" else "16"]


def strange_rows(vocab, dtype):
    """Rows in which thresholds, ties and masks take every way, by name in test_gpu_scoring.test_masks_and_ties; and NaN."""
    dt = lu.DTYPES[dtype]
    z = lu.make_rows(13, vocab, dt, 1, seed=vocab)
    keep = torch.rand(vocab, generator=torch.Generator().manual_seed(1)) < 0.003
    keep[vocab // 2] = True
    z[0, ~keep] = -math.inf
    z[1] = -math.inf
    z[2, ~keep] = torch.finfo(dt).min
    z[3] = torch.finfo(dt).min
    z[4] = 2.5
    z[5] = 0.0
    z[5, ::3] = -0.0
    z[6] = torch.linspace(20, -20, vocab).to(dt)
    z[7] = -math.inf
    z[7, vocab // 2:vocab // 2 + 30] = 1.0       # a few neighbours that are allowed
    z[8, vocab // 3:vocab // 3 + 600] = 30.0
    z[9] = -math.inf
    z[9, vocab - 1] = -1.0
    z[10, ::256] = 25.0
    z[11, 7] = math.nan
    z[11, vocab - 2] = math.inf
    tokens = torch.tensor([int(keep.nonzero()[0]), 3, 5, 7, 11, 13, 17, vocab // 2, 23, vocab - 1, 256, 31, -1])
    return z, tokens


def check_rows(z, tokens, top, repeat=1, workspace=False):
    """As test_gpu_scoring.check, for rows that are given `repeat` times over, and rows with a NaN among them."""
    vocab = z.shape[1]
    want = lu.score(z, tokens, 1.0)
    bad = want[1].isnan()
    again = torch.arange(repeat * len(z)) % len(z)
    pitch = vocab + 1
    flat = torch.empty(repeat * len(z) * pitch + 1, dtype=z.dtype, device=lu.DEV)
    zg = flat[1:].view(-1, pitch)[:, :vocab]
    zg.copy_(z.to(lu.DEV)[again.to(lu.DEV)])
    out = run_score(zg, tokens[again].to(lu.DEV), 1.0, top, full_workspace(zg, top) if workspace else None)
    logprob, entropy, stats, top_logprob, top_index = out
    rel = lu.spread(want[3], want[2])
    rel = torch.where(bad[:, None], 0.0, rel)
    at = tokens.clamp(0, vocab - 1)[:, None]
    assert lu.near(logprob, want[0][again], rel.gather(1, at)[again, 0])
    assert lu.near(stats, torch.where(bad[:, None], math.nan, want[2])[again], rel.amin(1, keepdim=True)[again])
    p = want[3].exp()
    terms = torch.where(p == 0, 0.0, p * (want[3].abs() + want[2][:, 1:].abs().nan_to_num(0, 0, 0) + 1) * rel)
    assert lu.near(entropy, want[1][again], 2 * terms.sum(1).nan_to_num(0)[again])
    if top:
        index = lu.order(z, top)
        assert torch.equal(top_index.cpu().long(), index[again])
        value = torch.where(bad[:, None], math.nan, want[3].gather(1, index))
        assert lu.near(top_logprob, value[again], rel.gather(1, index)[again])


@pytest.mark.parametrize("top", [1, 100, 128])
@pytest.mark.parametrize("vocab,dtype", [(1000, "bf16"), (16000, "f16"), (20001, "f32"), (25344, "f32"), (40001, "bf16"),
                                         (50257, "f16"), (50257, "f32"), (60001, "f32"), (104001, "bf16")])
def test_many_rows_with_alternatives(vocab, dtype, top):
    """As many rows as four workgroups to a compute unit are chosen for."""
    z, tokens = strange_rows(vocab, dtype)
    check_rows(z, tokens, top, repeat=40)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("limit", range(6))
def test_rows_at_the_limits_of_the_teams(limit, dtype):
    """The longest row of each team and one element more, at both starts that 16-bit rows have."""
    for vocab in (limits(dtype)[limit][0], limits(dtype)[limit][0] + 1):
        z = lu.make_rows(4, vocab, lu.DTYPES[dtype], 1 - vocab % 2, seed=vocab)
        z[1, -1] = 50.0
        z[2, 0] = 50.0
        z[3, :-3] = -math.inf
        tokens = torch.tensor([vocab - 1, 5, 0, vocab - 2])
        check_rows(z, tokens, 20)
        check_rows(z, tokens, 0)
        index, logit = lists(4, vocab, 20, vocab)
        index[0, 0], index[3, 0], index[3, 1:] = vocab - 1, vocab - 2, -1
        want, want_d, loss_off, off = lu.distill(z, index, logit, tokens, 2.0, 0.5)
        loss, d = torch.empty(4, device=lu.DEV), torch.empty((4, vocab), dtype=z.dtype, device=lu.DEV)
        qb.qsdp_distill_loss(lu.to_gpu(z), index.to(lu.DEV), logit.to(lu.DEV), tokens.to(lu.DEV), 2.0, 0.5, None, loss, None, d)
        assert lu.near(loss, want, loss_off) and lu.near(d, want_d, off)


PARTS = [("f32", 65536), ("f32", 250001), ("f32", 300001), ("f32", 500001), ("bf16", 300001), ("bf16", 600001), ("f16", 900001)]


@pytest.mark.parametrize("dtype,vocab", PARTS)
def test_parts_of_every_length(dtype, vocab):
    """A row's eighths in registers, with LDS and chunk by chunk."""
    z, tokens = strange_rows(vocab, dtype)
    some = torch.tensor([0, 1, 4, 7, 9, 10, 11, 12])
    check_rows(z[some], tokens[some], 100, workspace=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tau,alpha", [(1.0, 1.0), (2.0, 0.5), (3.0, 0.5)])
def test_gradient_after_the_loss_in_place(tau, alpha, dtype):
    """Segments of a row are overwritten while others still look up the list's places in theirs."""
    rows, vocab = 300, 50257
    z = lu.to_gpu(lu.make_rows(4, vocab, lu.DTYPES[dtype], 0, seed=4))[torch.arange(rows, device=lu.DEV) % 4].contiguous()
    index, logit = (t[torch.arange(rows) % 4].to(lu.DEV).contiguous() for t in lists(4, vocab, 128, 4))
    labels = torch.arange(rows, device=lu.DEV) * 167
    labels[0] = int(index[0, 0])
    loss, stats = torch.empty(rows, device=lu.DEV), torch.empty((rows, 3), device=lu.DEV)
    g = torch.linspace(-2, 2, rows, device=lu.DEV)
    qb.qsdp_distill_loss(z, index, logit, labels, tau, alpha, None, loss, stats)
    d = torch.empty_like(z)
    qb.qsdp_distill_loss_backward(z, index, logit, labels, tau, alpha, stats, g, d)
    qb.qsdp_distill_loss_backward(z, index, logit, labels, tau, alpha, stats, g, z)
    assert torch.equal(z, d)
