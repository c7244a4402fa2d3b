"""Plain 64-bit forms of the operators on logits and on packed weights, and how far 32-bit arithmetic may be from them."""
import math

import torch

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 2.0 ** -24                                             # half an ulp of 1 in binary32
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -9, torch.float16: 2.0 ** -12}  # ... with an implicit 2x slack
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}


def make_rows(rows, vocab, dtype, pad=0, seed=0, std=3.0, offset=0):
    """Logits [rows, vocab] as a view of padded rows, `offset` elements behind an aligned address."""
    gen = torch.Generator().manual_seed(seed)
    pitch = vocab + pad
    flat = (torch.randn(rows * pitch + offset, generator=gen) * std).to(dtype)
    return flat[offset:].view(rows, pitch)[:, :vocab]


def to_gpu(view):
    """The same view (storage, offset, strides) of a copy on the GPU."""
    base = view._base if view._base is not None else view
    flat = base.reshape(-1).to(DEV)
    return flat.as_strided(view.shape, view.stride(), view.storage_offset())


def shifted(z, tau):
    """m, t = (z - m) / tau, log sum exp t; rows of -inf: m = -inf, t = -inf, log sum = -inf."""
    m = z.max(1, keepdim=True).values
    t = (z - torch.where(m == -math.inf, 0.0, m)) / tau
    return m, t, t.exp().sum(1, keepdim=True).log()


def score(z, tokens, tau):
    """(logprob, entropy, stats, log p) in 64 bits."""
    z = z.double()
    vocab = z.shape[1]
    m, t, ls = shifted(z, tau)
    empty = ls == -math.inf
    log_p = torch.where(empty, -math.inf, t - ls)
    p = log_p.exp()
    entropy = -torch.where(p == 0, 0.0, p * log_p).sum(1)
    entropy = torch.where(empty[:, 0], 0.0, entropy)
    at = tokens.clamp(0, vocab - 1)
    logprob = log_p.gather(1, at[:, None])[:, 0]
    logprob = torch.where(tokens < 0, 0.0, torch.where((tokens >= vocab) & ~empty[:, 0], math.nan, logprob))
    bad = (z.isnan() | (z == math.inf)).any(1)
    nan = torch.tensor(math.nan, dtype=torch.float64)
    stats = torch.cat([m, ls], 1)
    return (torch.where(bad & (tokens >= 0), nan, logprob), torch.where(bad, nan, entropy), stats, log_p)


def score_grad(z, tokens, tau, g, h, of_score=None):
    """d logits in 64 bits, and how far each may be off in 32-bit arithmetic before it is rounded to the logits' format."""
    _, entropy, stats, log_p = of_score or score(z, tokens, tau)
    vocab = z.shape[1]
    given = (tokens >= 0) & (tokens < vocab)
    g = (g.double() if g is not None else torch.zeros(len(tokens), dtype=torch.float64)) * given
    h = h.double() if h is not None else torch.zeros(len(tokens), dtype=torch.float64)
    p = log_p.exp()
    info = torch.where(p == 0, 0.0, log_p) + entropy[:, None]
    d = -p * (g[:, None] + h[:, None] * info)
    onehot = torch.zeros_like(p)
    onehot[torch.arange(len(tokens)), tokens.clamp(0, vocab - 1)] = 1.0
    d += onehot * g[:, None]
    rel = spread(log_p, stats)
    size = p * (g.abs()[:, None] + h.abs()[:, None] * (torch.where(p == 0, 0.0, log_p).abs() + entropy[:, None] + 1))
    off = (rel * size + 4 * EPS * onehot * g.abs()[:, None]) / tau
    empty = stats[:, 1:] == -math.inf
    return torch.where(empty, 0.0, d / tau), torch.where(empty, 0.0, off)


def spread(log_p, stats):
    """Relative error of a probability: four roundings on the way to the exponent (difference, constant, product, the log of
    the sum taken off), the exponential's own few, and the sum's: additions in parts, 8 log2(n) roundings for a random walk
    of hundreds of them."""
    n = log_p.shape[1]
    reach = torch.where(torch.isfinite(log_p), log_p.abs(), torch.tensor(110.0, dtype=torch.float64))
    ls = torch.where(torch.isfinite(stats[:, 1:]), stats[:, 1:].abs(), torch.tensor(0.0, dtype=torch.float64))
    return EPS * (4 * (reach + ls + math.log(n)) + 16 + 8 * math.log2(n + 1))


def near(got, want, off):
    """Whether got (in its format) is want within `off`, one rounding to the format and its smallest steps; infinities and
    NaN at the same places, a value beyond the format being its infinity."""
    got64, want = got.detach().cpu().double(), want.double()
    beyond = want.to(got.dtype).isinf()
    want = torch.where(beyond, torch.sign(want) * math.inf, want)
    same = (got64 == want) | (got64.isnan() & want.isnan())
    bound = off + want.abs() * 2 * ROUND[got.dtype] + TINY[got.dtype]
    ok = same | ((got64 - want).abs() <= bound)
    if not bool(ok.all()):
        worst = torch.where(ok, 0.0, (got64 - want).abs() / bound).nan_to_num(math.inf, math.inf)
        i = int(worst.reshape(-1).argmax())
        print(f"{int((~ok).sum())} of {ok.numel()} off, worst {float(worst.reshape(-1)[i])} bounds at {i}: "
              f"{float(got64.reshape(-1)[i])} for {float(want.reshape(-1)[i])}")
    return bool(ok.all())


def order(z, top):
    """The `top` largest of each row downwards, equal ones by index upwards, a NaN above all."""
    import numpy as np
    v = z.double().numpy()
    key = np.where(np.isnan(v), np.inf, v)
    rank = np.lexsort((np.broadcast_to(np.arange(v.shape[1]), v.shape), -key, ~np.isnan(v)), axis=1)
    return torch.from_numpy(rank[:, :top].copy())


def distill(z, index, logit, labels, tau, alpha):
    """(loss, d loss / d logits, how far either may be off) per row, in 64 bits."""
    z = z.double()
    rows, vocab = z.shape
    m, t, ls = shifted(z, tau)
    _, t1, ls1 = shifted(z, 1.0)
    empty = (ls == -math.inf)
    log_q = torch.where(empty, -math.inf, t - ls)
    log_1 = torch.where(empty, -math.inf, t1 - ls1)
    loss, d = torch.zeros(rows, dtype=torch.float64), torch.zeros_like(z)
    loss_off, off = torch.zeros_like(loss), torch.zeros_like(z)
    stats, stats1 = torch.cat([m, ls], 1), torch.cat([m, ls1], 1)
    if index is not None and alpha > 0:
        here = (index >= 0) & (index < vocab)
        at = torch.where(here, index, 0).long()
        u = torch.where(here, logit.double() / tau, -math.inf)
        mass = torch.logsumexp(u, 1, keepdim=True)
        taught = mass != -math.inf
        log_p = torch.where(taught, u - mass, -math.inf)
        p = log_p.exp()
        terms = torch.where(p == 0, 0.0, p * (log_p - log_q.gather(1, at)))
        loss += alpha * tau ** 2 * terms.sum(1)
        rel = spread(log_q, stats)
        size = p * (torch.where(p == 0, 0.0, log_p).abs() + torch.where(p == 0, 0.0, log_q.gather(1, at)).abs().nan_to_num(0, 0, 0) + 1)
        loss_off += alpha * tau ** 2 * (size * (rel.gather(1, at) + EPS * 16)).sum(1) * 2
        target = torch.zeros_like(z).scatter_add_(1, at, p)
        d += alpha * tau * taught * (log_q.exp() - target)
        off += alpha * tau * (log_q.exp() * rel + target * EPS * (32 + 4 * torch.where(p > 0, log_p.abs(), 0.0).amax(1, keepdim=True)))
    if labels is not None and alpha < 1:
        given = (labels >= 0) & (labels < vocab)
        lab = labels.clamp(0, vocab - 1)[:, None]
        loss -= torch.where(given, (1 - alpha) * log_1.gather(1, lab)[:, 0], 0.0)
        rel = spread(log_1, stats1)
        picked = log_1.gather(1, lab)[:, 0].abs().nan_to_num(0, 0, 0) + 1
        loss_off += (1 - alpha) * rel.gather(1, lab)[:, 0] * picked
        hard = log_1.exp()
        off += (1 - alpha) * given[:, None] * hard * rel
        hard = hard.scatter_add(1, lab, torch.full((rows, 1), -1.0, dtype=torch.float64))
        d += (1 - alpha) * given[:, None] * hard
        off += (1 - alpha) * given[:, None] * (hard < 0) * 4 * EPS
        loss = torch.where(labels >= vocab, math.nan, loss)
    return loss, torch.where(empty, 0.0, d), loss_off, torch.where(empty, 0.0, off)


def tokens8(x, bucket):
    """(scale, codes, sums) of the rounding of tokens: a binary32 product and a binary32 division by definition, whole numbers
    after them."""
    x = x.float()
    scale = x.abs().amax(1) * torch.tensor(1.0 / 127.0, dtype=torch.float32)
    scale = torch.where(torch.isfinite(x).all(1), scale, math.nan)
    q = torch.where(scale[:, None] > 0, (x / scale[:, None]).round(), 0.0).clamp(-127, 127).nan_to_num(0).to(torch.int64)
    k = x.shape[1]
    buckets = -(-k // bucket)
    padded = torch.zeros((x.shape[0], buckets * bucket), dtype=torch.int64)
    padded[:, :k] = q
    return scale, q, padded.view(x.shape[0], buckets, bucket).sum(2)


def product(scale, q, sums, codes, meta, bias, bucket):
    """(y, how far it may be off) of the product in 64 bits; codes uint8 [n, buckets * bucket], meta float32 [n, buckets, 2]."""
    n, buckets = meta.shape[:2]
    k = q.shape[1]
    y = torch.zeros((q.shape[0], n), dtype=torch.float64)
    off = torch.zeros_like(y)
    for b in range(buckets):
        lo, hi = b * bucket, min((b + 1) * bucket, k)
        c = codes[:, lo:hi].double()
        qb = q[:, lo:hi].double()
        base, step = meta[:, b, 0].double(), meta[:, b, 1].double()
        y += qb @ (base[:, None] + step[:, None] * c).t()
        whole = (qb @ (c - 128.0).t()).abs() * step.abs()
        centre = (base.abs() + 128 * step.abs())[None, :] * sums[:, b, None].double().abs()
        off += (whole + centre) * EPS * (6 + buckets)
    s = scale.double()[:, None]
    y, off = y * s, off * s.abs() + (y * s).abs() * 2 * EPS
    if bias is not None:
        y = y + bias.double()
        off = off + 2 * EPS * (y.abs() + bias.double().abs())
    return y, off
