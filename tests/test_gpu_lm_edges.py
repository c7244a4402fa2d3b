"""Rows of logits with what is no number, no token or no teacher in them, and masks of the format's lowest value."""
import math

import pytest
import torch

import lm_util as lu
from paper_2302_02390_amd import binding as qb
from test_gpu_distill import lists
from test_gpu_scoring import full_workspace, run_score

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [5, 3001, 50257, 70001, 131073])
def test_statistics_of_rows_with_a_nan_or_infinity(vocab, dtype):
    """Neither the maximum nor the sum of such a row is a number, whole or in parts."""
    z = lu.make_rows(4, vocab, lu.DTYPES[dtype], 1, seed=vocab)
    z[0, vocab // 2] = math.nan
    z[1, vocab - 1] = math.inf
    z[2] = math.nan
    zg = lu.to_gpu(z)
    tokens = torch.tensor([0, vocab - 1, -1, 2], device=lu.DEV)
    for workspace in (None, full_workspace(zg, 3)):
        logprob, entropy, stats, _, _ = run_score(zg, tokens, 1.0, 3, workspace)
        assert stats.isnan().tolist() == [[True, True]] * 3 + [[False, False]]
        # a row without a token has no log probability to be wrong
        assert logprob[:2].isnan().all() and float(logprob[2]) == 0.0 and entropy[:3].isnan().all()
        d = torch.empty_like(zg)
        one = torch.ones(4, device=lu.DEV)
        qb.qsdp_token_logprobs_backward(zg, tokens, 1.0, stats, entropy, one, one, d)
        assert d[:3].isnan().all() and d[3].isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [7, 3001, 70001])
def test_tokens_past_the_vocabulary_of_a_masked_row(vocab, dtype):
    """A token that does not exist is NaN in every row, one that is not asked for 0."""
    z = lu.to_gpu(torch.full((4, vocab), -math.inf, dtype=lu.DTYPES[dtype]))
    tokens = torch.tensor([vocab, vocab - 1, -1, 1 << 40], device=lu.DEV)
    for workspace in (None, full_workspace(z, 0)):
        logprob, entropy, stats, _, _ = run_score(z, tokens, 1.0, 0, workspace)
        assert logprob[0].isnan() and float(logprob[1]) == -math.inf and float(logprob[2]) == 0.0 and logprob[3].isnan()
        assert bool((entropy == 0).all()) and bool((stats == -math.inf).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [9, 5003, 50257])
def test_a_list_of_weight_zero_is_not_looked_at(vocab, dtype):
    """alpha = 0: whatever the list holds, loss and gradient are the labels' alone."""
    z = lu.to_gpu(lu.make_rows(3, vocab, lu.DTYPES[dtype], 0, seed=vocab))
    index, logit = (t.to(lu.DEV) for t in lists(3, vocab, 5, vocab))
    logit[0, 2], logit[1, 1], logit[2] = math.nan, math.inf, -math.inf
    labels = torch.tensor([3, -1, 0], device=lu.DEV)
    found = []
    for i, t in ((None, None), (index, logit)):
        loss, stats = torch.empty(3, device=lu.DEV), torch.empty((3, 3), device=lu.DEV)
        d, after = torch.empty_like(z), torch.empty_like(z)
        qb.qsdp_distill_loss(z, i, t, labels, 2.0, 0.0, None, loss, stats, d)
        qb.qsdp_distill_loss_backward(z, i, t, labels, 2.0, 0.0, stats, torch.ones(3, device=lu.DEV), after)
        assert loss.isfinite().all() and d.isfinite().all() and after.isfinite().all()
        found.append((loss, stats, d, after))
    assert all(torch.equal(a, b) for a, b in zip(*found))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tau", [1.0, 2.0, 0.75, 3.0])
def test_lists_on_tokens_masked_with_the_lowest_value(tau, dtype):
    """The student's logit at places of the list is the format's lowest: its log probability there is a large number and not
    -inf, and so is the loss as far as binary32 holds it. Error: a probability of the list has an exponent of a magnitude below
    16 with four roundings, an exponential, a sum of eight and a division, below 100 roundings; the terms and their sum have
    twenty."""
    dt, vocab = lu.DTYPES[dtype], 3001
    z = lu.make_rows(3, vocab, dt, 0, seed=7)
    index, logit = lists(3, vocab, 8, 7, 1.0)
    z[0, int(index[0, 3])] = torch.finfo(dt).min
    z[1, 100:] = torch.finfo(dt).min
    index[1] = torch.arange(96, 104)
    z[2] = torch.finfo(dt).min
    z[2, 5] = 1.0
    index[2] = torch.arange(3, 11)
    labels = torch.tensor([1, 2, 5])
    limit = torch.finfo(torch.float32).max
    for alpha in (1.0, 0.5, 0.25):
        want, want_d, _, off = lu.distill(z, index, logit, labels, tau, alpha)
        zg, d, loss = lu.to_gpu(z), torch.empty((3, vocab), dtype=dt, device=lu.DEV), torch.empty(3, device=lu.DEV)
        qb.qsdp_distill_loss(zg, index.to(lu.DEV), logit.to(lu.DEV), labels.to(lu.DEV), tau, alpha, None, loss, None, d)
        got = loss.cpu().double()
        assert bool(((got - want).abs() <= 128 * lu.EPS * want.abs())[want < 0.99 * limit].all())
        assert bool((got == math.inf)[want > 1.01 * limit].all())
        assert bool((want < 0.99 * limit)[0]) and lu.near(d, want_d, off)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [301, 50257, 131073])
def test_what_is_no_number_in_distillation(vocab, dtype):
    """A NaN or +inf among the logits makes loss and gradient NaN where anything is asked of the row; among the teacher's, the loss
    and the gradient at the list's places; a label past the vocabulary the loss alone. No row_scale, no gradient."""
    z = lu.make_rows(9, vocab, lu.DTYPES[dtype], 1, seed=vocab)
    index, logit = lists(9, vocab, 6, vocab)
    z[0, vocab // 2] = math.nan
    z[1, vocab - 1] = math.inf
    z[2, 0], index[2] = math.nan, -1              # neither list nor label
    z[3, 5] = math.nan                            # row_scale 0
    logit[4, 2] = math.nan
    logit[5, 3] = math.inf
    logit[6, 1], index[6, 1] = math.nan, -1       # an absent slot's
    labels = torch.tensor([1, -1, -1, 4, 5, -1, 7, vocab, 1 << 33])
    scale = torch.tensor([1.0, 1.0, 1.0, 0.0, 1.0, 1.0, 1.0, 1.0, 1.0])
    zg, ig, tg, lg, sg = lu.to_gpu(z), index.to(lu.DEV), logit.to(lu.DEV), labels.to(lu.DEV), scale.to(lu.DEV)
    for tau in (1.0, 2.0, 3.0):
        loss, stats = torch.empty(9, device=lu.DEV), torch.empty((9, 3), device=lu.DEV)
        d, after = (torch.empty((9, vocab), dtype=z.dtype, device=lu.DEV) for _ in range(2))
        qb.qsdp_distill_loss(zg, ig, tg, lg, tau, 0.5, sg, loss, stats, d)
        qb.qsdp_distill_loss_backward(zg, ig, tg, lg, tau, 0.5, stats, sg, after)
        assert loss.isnan().tolist() == [True, True, False, True, True, True, False, True, True] and float(loss[2]) == 0.0
        listed = torch.zeros((9, vocab), dtype=torch.bool)
        listed[4, index[4].long()] = listed[5, index[5].long()] = True
        listed[:2] = True
        for g in (d, after):
            assert torch.equal(g.isnan().cpu(), listed)
            assert bool((g[2:4] == 0).all())
        _, want, _, off = lu.distill(z[6:], index[6:], logit[6:], labels[6:], tau, 0.5)
        assert lu.near(d[6:], want, off) and lu.near(after[6:], want, off)
