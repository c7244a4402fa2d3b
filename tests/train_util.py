"""Plain 64-bit forms of the operators of a training step in few bits, and how far 32-bit arithmetic may be from them."""
import numpy as np
import torch

from lm_util import DEV, DTYPES, EPS, near, to_gpu  # noqa: F401

DEPTH = 96  # additions that one term of a row's sum goes through at most: 32 in its lane, the wave's and the team's


def matrix(rows, n, dtype, pad=0, offset=0, seed=0, std=1.0, mean=0.0):
    """[rows, n] as a view of padded rows, `offset` elements behind an aligned address."""
    gen = torch.Generator().manual_seed(seed)
    pitch = n + pad
    flat = (torch.randn(rows * pitch + offset, generator=gen) * std + mean).to(dtype)
    return flat[offset:].view(rows, pitch)[:, :n]


# ---- layer norm ----------------------------------------------------------------------------------------------------------
def norm(x, w, b, eps):
    """(y, stats, h) in 64 bits and how far y, the mean and h may be off (the latter's relative part by the statistics)."""
    x = x.double()
    n = x.shape[1]
    w = torch.ones(n, dtype=torch.float64) if w is None else w.double()
    b = torch.zeros(n, dtype=torch.float64) if b is None else b.double()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    var = c.square().mean(1, keepdim=True)
    rstd = 1.0 / (var + eps).sqrt()
    h = c * rstd
    mean_off = DEPTH * EPS * x.abs().mean(1, keepdim=True)
    # the variance: its sum, and that the mean taken off is another one; half of that in the root
    rel = (DEPTH + 8) * EPS + mean_off.square() * rstd.square()
    h_off = rstd * (mean_off + EPS * c.abs()) + h.abs() * rel
    y = h * w + b
    y_off = w.abs() * (h_off + 2 * EPS * h.abs()) + 2 * EPS * (y.abs() + b.abs())
    return y, torch.cat([mean, rstd], 1), h, y_off, torch.cat([mean_off, rstd * rel], 1), h_off


def norm_grad(x, w, dy, eps):
    """{dx, dw, db} in 64 bits, and how far each may be off."""
    _, stats, h, _, _, h_off = norm(x, w, None, eps)
    rows, n = x.shape
    dy = dy.double()
    w = torch.ones(n, dtype=torch.float64) if w is None else w.double()
    rstd = stats[:, 1:]
    g = dy * w
    c0, c1 = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    dx = rstd * (g - c0 - h * c1)
    c0_off = (DEPTH + 2) * EPS * g.abs().mean(1, keepdim=True)
    c1_off = (DEPTH + 4) * EPS * (g * h).abs().mean(1, keepdim=True) + (g.abs() * h_off).mean(1, keepdim=True)
    dx_off = rstd * (4 * EPS * (g.abs() + c0.abs() + (h * c1).abs()) + c0_off + h.abs() * c1_off + h_off * c1.abs())
    dx_off = dx_off + dx.abs() * (DEPTH + 16) * EPS
    down = rows / 32 + 64  # additions on the way of a row's term into a column's sum
    dw_off = (dy.abs() * h_off).sum(0) + down * EPS * (dy * h).abs().sum(0)
    return {"dx": dx, "dw": (dy * h).sum(0), "db": dy.sum(0)}, {"dx": dx_off, "dw": dw_off, "db": down * EPS * dy.abs().sum(0)}


# ---- blocks --------------------------------------------------------------------------------------------------------------
F8 = torch.float8_e4m3fn


def blocks(x, high, wide):
    """(codes as float32, scales [blocks down, blocks across]) of blocks high x wide of x on the CPU, by the definition in
    binary32; codes of x's own shape."""
    x = x.float()
    rows, cols = x.shape
    whole = torch.nn.functional.pad(x, (0, -cols % wide, 0, -rows % high))
    parts = whole.reshape(whole.shape[0] // high, high, -1, wide)
    most = torch.maximum(parts.abs().nan_to_num(0.0, posinf=float("inf")).amax((1, 3)), torch.tensor(2.0 ** -100))
    up = torch.tensor(448.0) / most
    codes = (parts * up[:, None, :, None]).to(F8).float().reshape(whole.shape)[:rows, :cols]
    return codes, most / torch.tensor(448.0)


def held(codes, scales, high, wide):
    """The values in 64 bits."""
    rows, cols = codes.shape
    s = scales.double().repeat_interleave(high, 0)[:rows].repeat_interleave(wide, 1)[:, :cols]
    return codes.double() * s


def product(a, b, exact):
    """a [m, k], b [n, k] as held in 64 bits: (a b^T, how far it may be off). Every addition may be off by an ulp of the sum of
    magnitudes so far. Where codes go into the matrix instruction as they are, the products of eight neighbours are aligned to
    the largest and keep at least 14 bits below its first: eight of them lose 2^-11 of it."""
    k = a.shape[1]
    y = a @ b.t()
    off = (a.abs() @ b.abs().t()) * (128 + -(-k // 128) + 16) * 2 * EPS
    if not exact:
        eights = lambda t: torch.nn.functional.pad(t.abs(), (0, -k % 128)).reshape(t.shape[0], -1, 8).amax(2)
        # which eight meet is the kernel's choice: within a block of 128 by pieces of 16 codes, so by 8 in order
        off = off + (eights(a) @ eights(b).t()) * 2.0 ** -11
    return y, off


# ---- AdamW ---------------------------------------------------------------------------------------------------------------
def philox(counter, key):
    """Philox4x32-10 of counters uint64[n, 4] (words) with a 64-bit key: uint64[n, 4]."""
    c = [counter[:, i].astype(np.uint64) for i in range(4)]
    k0, k1 = np.uint64(key & 0xFFFFFFFF), np.uint64(key >> 32)
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ k0, p1 & low, (p0 >> np.uint64(32)) ^ c[3] ^ k1, p0 & low]
        k0, k1 = (k0 + np.uint64(0x9E3779B9)) & low, (k1 + np.uint64(0xBB67AE85)) & low
    return np.stack(c, 1)


def by_256(v):
    return torch.nn.functional.pad(v, (0, -v.numel() % 256)).view(-1, 256)


def moments(m, v, scale):
    """What 8-bit codes stand for, float32 [blocks, 256] as the step decodes them: (m, v)."""
    scale = scale.view(-1, 2)
    c, d = by_256(m.float()), by_256(v.float())
    root = (scale[:, 1:] * torch.tensor(1.0 / 255 ** 2)) * (d * d)
    return (scale[:, :1] * torch.tensor(1.0 / 127 ** 2)) * (c * c.abs()), root * root


def fma(a, b, c):
    return (torch.as_tensor(a).double() * b.double() + c.double()).float()


def codes_of(value, word, most):
    """(codes, largest of each block) of float32 [blocks, 256] that are not negative, with the thresholds of `word` [blocks]."""
    largest = value.amax(1, keepdim=True)
    kept = largest >= 2.0 ** -96
    w = value * torch.where(kept, torch.tensor(float(most * most)) / largest, 0.0)
    c = w.double().sqrt().floor().float()
    t = (torch.from_numpy(word.astype(np.int64))[:, None] + torch.arange(256) * 0x9E3779B9) & 0xFFFFFFFF
    t = ((t >> 20).float() + 0.5) * 2.0 ** -12
    c = torch.where(w - c * c > (2 * c + 1) * t, c + 1, c).clamp(max=float(most))
    return c, torch.where(kept, largest, 0.0)


def adamw(x, g, m, v, scale, first, seed, lr, beta1, beta2, eps, decay, bias1, bias2):
    """One step of one tensor on the CPU: (x in 64 bits, how far it may be off, m, v, scale), the moments as they are held."""
    b1, b2 = torch.tensor(beta1), torch.tensor(beta2)
    n = x.numel()
    m32, v32 = (m, v) if scale is None else (t.reshape(-1)[:n] for t in moments(m, v, scale))
    g = g.float()
    m32 = fma(b1, m32, (1 - b1) * g)
    v32 = fma(b2, v32, ((1 - b2) * g) * g)
    md, vd, xd = m32.double(), v32.double(), x.double()
    lr, decay, eps, bias1, bias2 = (float(torch.tensor(a)) for a in (lr, decay, eps, bias1, bias2))
    u = (md / bias1) / ((vd / bias2).sqrt() + eps)
    y = xd - lr * (u + decay * xd)
    off = 16 * EPS * lr * (u.abs() + (decay * xd).abs()) + 2 * EPS * (y.abs() + xd.abs())
    if scale is None:
        return y, off, m32, v32, None
    blocks_ = -(-n // 256)
    counter = np.zeros((blocks_, 4), dtype=np.uint64)
    numbers = 8 * first + np.arange(blocks_, dtype=np.uint64)
    counter[:, 0], counter[:, 1], counter[:, 2] = numbers & np.uint64(0xFFFFFFFF), numbers >> np.uint64(32), 3
    words = philox(counter, seed)
    root = v32.double().sqrt().float()
    c, top = codes_of(by_256(m32.abs()), words[:, 0], 127)
    d, top_root = codes_of(by_256(root), words[:, 1], 255)
    d = torch.where((by_256(root) > 0) & (top_root > 0), d.clamp(min=1.0), d)
    c = (c * by_256(m32).sign()).reshape(-1)[:n].to(torch.int8)
    return y, off, c, d.reshape(-1)[:n].to(torch.uint8), torch.cat([top, top_root], 1).reshape(-1)
