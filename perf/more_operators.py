"""The operators of a training step in few bits, in plain form and through the binding's entry points.

``listed()`` names twelve uses, ``draw(rng)`` gives more of the same ranges; ``prepare(case, seed)`` makes what a program
holds before the call, ``run(state)`` is one pass, ``exact(case, seed)`` the same outputs in 64 bits from the definitions,
``work(case)`` the bytes and operations that a pass cannot do without.

Uses (``kind``):
  norm    layer norm of rows; with ``grad`` also the gradients of the rows, the weight and the bias
  linear  rows, rounded to 8-bit floating point with a scale per 128 elements, times weights held so in blocks of 128 x 128
  train   the same with everything rounded in the pass: output, gradient of the rows and gradient of the weights
  adamw   an AdamW step over many tensors at once, moments in 32 or in 8 bits

Definitions. Norm of a row x of n: mu = sum x / n, r = 1 / sqrt(sum (x - mu)^2 / n + eps), h = (x - mu) r, y = h w + b;
  with g = dy w: dx = r (g - mean g - h mean (g h)), dw = sum over rows of dy h, db = sum over rows of dy
Blocks: a = max(max |x|, 2^-100) over the block in 32 bits, codes = e4m3(x (448 / a)) to nearest even, scale = a / 448;
  y = sum over blocks of the scales' product times the sum of the codes' products, + bias. Blocks lie along the summed axis:
  128 elements of a row of the first operand (of dy and x for the weights' gradient: 128 tokens of a column), 128 x 128 weights
AdamW: m' = beta1 m + (1 - beta1) g, v' = beta2 v + (1 - beta2) g^2,
  x' = x - lr ((m' / bias1) / (sqrt(v' / bias2) + eps) + decay x)
  Moments in 8 bits, by blocks of 256 elements of a tensor: m = M c |c| / 127^2, sqrt v = R c^2 / 255^2, M and R the block's
  largest |m| and sqrt v. With w the value over M / 127^2 (or R / 255^2) and c = floor sqrt w the new code is c + 1 where
  w - c^2 > (2 c + 1) t, else c; at most 127 (255), and at least 1 where v' > 0. The threshold t of element i of the block is
  (h + 1/2) / 2^12, h the upper 12 bits of (word + i 0x9E3779B9) mod 2^32, word the first (for m) or second (for v) of the
  Philox4x32-10 block with the seed as key and counter (block, 0, 3, 0). Tensors' blocks are numbered in order, each
  tensor's from the next multiple of 8 on.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
VOCAB = 50257  # the framework's GPT shapes
NORM_CELLS = 16384 * 2048  # elements of the largest norm
PRODUCT = 8192 * 2048 * 8192  # products of the largest case's operands
EPS = 1e-5
LR, BETA1, BETA2, ADAM_EPS, DECAY, STEP = 1e-3, 0.9, 0.95, 1e-8, 0.1, 100
PIECE = 2048  # elements of a tensor that its eight blocks of states hold


def listed():
    return [
        # one decoded token through a norm of the 1.3B model: latency
        dict(name="norm-one-token", kind="norm", rows=1, n=2048, pad=0, dtype="bf16", out="bf16", weight="f32", grad=False),
        # odd rows of a float residual stream, padded, outputs for a product in 16 bits
        dict(name="norm-odd", kind="norm", rows=333, n=1023, pad=5, dtype="f32", out="bf16", weight="f32", grad=True),
        # a micro-batch of the 125M model at context 2048, both directions
        dict(name="norm-step", kind="norm", rows=4096, n=768, pad=0, dtype="bf16", out="bf16", weight="bf16", grad=True),
        # eight contexts of the 1.3B model, both directions
        dict(name="norm-long", kind="norm", rows=16384, n=2048, pad=0, dtype="bf16", out="bf16", weight="f32", grad=True),
        # one token through the up-projection of the 1.3B model
        dict(name="linear-one-token", kind="linear", m=1, n=8192, k=2048, dtype="bf16", out="bf16", bias=True),
        # sixteen users' tokens onto the vocabulary
        dict(name="linear-head", kind="linear", m=16, n=VOCAB, k=2048, dtype="bf16", out="f32", bias=False),
        # odd sizes everywhere, blocks that end inside rows and columns
        dict(name="linear-odd", kind="linear", m=333, n=4093, k=1000, dtype="f16", out="f16", bias=True),
        # a layer of the 350M model on a short batch: output and both gradients, loss scaled
        dict(name="train-small", kind="train", m=1000, n=4096, k=1024, dtype="f16", grad="f16"),
        # the up-projection of the 1.3B model over four contexts, the weights' gradient in 32 bits
        dict(name="train-step", kind="train", m=8192, n=8192, k=2048, dtype="bf16", grad="f32"),
        # the vectors of the 350M model (norms, biases), which the codec leaves in full precision
        dict(name="adamw-vectors", kind="adamw", d=1024, layers=24, matrices=False, tensors=0, numel=0, bits=32, dtype="f32",
             copy="none"),
        # the 350M model with moments in 32 bits
        dict(name="adamw-350m-32", kind="adamw", d=1024, layers=24, matrices=True, tensors=0, numel=0, bits=32, dtype="f32",
             copy="none"),
        # the 350M model in mixed precision with moments in 8 bits, short tensors' in 32
        dict(name="adamw-350m-8", kind="adamw", d=1024, layers=24, matrices=True, tensors=0, numel=0, bits=8, dtype="bf16",
             copy="bf16"),
    ]


def draw(rng):
    def size(lo, hi):  # any integer, spread over its logarithm
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["norm", "norm", "linear", "linear", "train", "adamw", "adamw"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    if kind == "norm":
        n = rng.choice([768, 1024, 2048, 4096, 8192, size(1, 16384), size(64, 16384)])
        out = rng.choice(["f32", "bf16", "f16"]) if dtype == "f32" else dtype
        most = NORM_CELLS // n // (2 if dtype == "f32" else 1)
        return dict(kind=kind, rows=size(1, min(65536, most)), n=n, pad=rng.choice([0, 0, -n % 64, rng.randrange(1, 100)]),
                    dtype=dtype, out=out, weight=rng.choice(["f32", out]), grad=rng.random() < 0.7)
    if kind == "adamw":
        bits, copy = rng.choice([8, 8, 32]), rng.choice(["none", "bf16", "f16"])
        if rng.random() < 0.5:
            return dict(kind=kind, d=8 * size(16, 128), layers=size(1, 16), matrices=rng.random() < 0.7, tensors=0, numel=0,
                        bits=bits, dtype=dtype, copy=copy)
        return dict(kind=kind, d=0, layers=0, matrices=False, tensors=size(1, 400), numel=size(1000, 200_000_000), bits=bits,
                    dtype=dtype, copy=copy)
    while True:
        m, n = size(1, 16384), rng.choice([768, 1024, 2048, 4096, 8192, VOCAB, size(64, 16384)])
        k = rng.choice([768, 1024, 2048, 4096, 8192, size(64, 8192)])
        if m * n * k <= PRODUCT and (kind == "linear" or n != VOCAB):
            break
    if kind == "linear":
        return dict(kind=kind, m=m, n=n, k=k, dtype=dtype, out=rng.choice([dtype, dtype, "f32"]), bias=rng.random() < 0.5)
    return dict(kind=kind, m=m, n=n, k=k, dtype=dtype, grad=rng.choice([dtype, "f32"]))


def _tensor_sizes(case):
    """Elements of every tensor, in order: a GPT model's, or odd ones of a given sum."""
    if case["tensors"]:
        count, total = case["tensors"], case["numel"]
        share = [1.0 + 50.0 * ((i * 0.6180339887498949 + total * 0.3819660112501051) % 1.0) ** 4 for i in range(count)]
        return [max(1, int(total * s / sum(share))) for s in share]
    d = case["d"]
    vectors, matrices = [d, d, 3 * d, d, d, d, 4 * d, d], [3 * d * d, d * d, 4 * d * d, 4 * d * d]
    block = vectors + matrices if case["matrices"] else vectors
    return ([VOCAB * d, 2048 * d] if case["matrices"] else []) + block * case["layers"] + [d, d]


def _state_bits(case, n):
    return 8 if case["bits"] == 8 and n >= 4096 else 32  # short tensors' moments stay in 32 bits


def work(case):
    if case["kind"] == "norm":
        cells = case["rows"] * case["n"]
        a, b, w = SIZE[case["dtype"]], SIZE[case["out"]], SIZE[case["weight"]]
        small = case["n"] * (2 * w + (8 if case["grad"] else 0)) + 8 * case["rows"]
        return {"bytes": cells * ((a + b) + (a + b if case["grad"] else 0)) + small, "flops": (24.0 if case["grad"] else 8.0) * cells}
    if case["kind"] == "adamw":
        total = 0
        for n in _tensor_sizes(case):
            states = 16 * n if _state_bits(case, n) == 32 else 4 * n + 16 * -(-n // 256)
            total += n * (8 + SIZE[case["dtype"]] + (0 if case["copy"] == "none" else 2)) + states
        return {"bytes": total, "flops": 20.0 * sum(_tensor_sizes(case))}
    m, n, k = case["m"], case["n"], case["k"]
    if case["kind"] == "linear":
        return {"bytes": m * k * SIZE[case["dtype"]] + n * k + 4 * -(-n // 128) * -(-k // 128) + (4 * n if case["bias"] else 0)
                + m * n * SIZE[case["out"]], "flops": 2.0 * m * n * k}
    return {"bytes": 2 * SIZE[case["dtype"]] * (m * k + m * n) + n * k * (SIZE[case["dtype"]] + SIZE[case["grad"]]),
            "flops": 6.0 * m * n * k}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    return {"norm": _prepare_norm, "linear": _prepare_linear, "train": _prepare_train, "adamw": _prepare_adamw}[case["kind"]](
        case, gen, {"case": dict(case)}, int(seed))


def _normal(gen, shape, std, dtype=torch.float32, mean=0.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=gen).to(dtype)


def _prepare_norm(case, gen, s, seed):
    rows, n = case["rows"], case["n"]
    x = _normal(gen, (rows, n + case["pad"]), 1.0)
    x *= torch.empty((rows, 1), device="cuda").uniform_(0.2, 3.0, generator=gen)
    x += torch.empty((rows, 1), device="cuda").uniform_(-1.0, 1.0, generator=gen)
    s["x"] = x.to(DTYPES[case["dtype"]])[:, :n]
    s["w"] = _normal(gen, n, 0.1, DTYPES[case["weight"]], 1.0)
    s["b"] = _normal(gen, n, 0.1, DTYPES[case["weight"]])
    s["y"] = torch.empty((rows, n), dtype=DTYPES[case["out"]], device="cuda")
    s["stats"] = torch.empty((rows, 2), dtype=torch.float32, device="cuda")
    if case["grad"]:
        s["dy"] = _normal(gen, (rows, n), 1.0 / 64, DTYPES[case["out"]])
        s["dx"] = torch.empty((rows, n), dtype=DTYPES[case["dtype"]], device="cuda")
        s["dw"], s["db"] = (torch.empty(n, dtype=torch.float32, device="cuda") for _ in range(2))
        s["workspace"] = torch.empty(512 * 8 * n + 4096, dtype=torch.uint8, device="cuda")
    return s


def _rounded(x, high, wide):
    """e4m3 codes and scales of blocks high x wide of x, which is whole blocks: {codes, scale per block}."""
    blocks = x.view(x.shape[0] // high, high, x.shape[1] // wide, wide)
    most = blocks.abs().amax((1, 3), keepdim=True).clamp(min=2.0 ** -100)
    codes = (blocks * (torch.full_like(most, 448.0) / most)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return codes.view(x.shape), (most / torch.full_like(most, 448.0))[:, 0, :, 0]


def _whole(x, high, wide):
    return torch.nn.functional.pad(x, (0, -x.shape[1] % wide, 0, -x.shape[0] % high))


def _prepare_linear(case, gen, s, seed):
    m, n, k = case["m"], case["n"], case["k"]
    x = _normal(gen, (m, k), 1.0) * torch.empty((m, 1), device="cuda").uniform_(0.1, 4.0, generator=gen)
    s["x"] = x.to(DTYPES[case["dtype"]])
    codes, scale = _rounded(_whole(_normal(gen, (n, k), 0.02), 128, 128), 128, 128)
    s["w"] = codes[:n].contiguous()
    s["w_scale"] = scale.t().contiguous()  # a row of scales for each 128 of k
    s["bias"] = _normal(gen, n, 0.1) if case["bias"] else None
    s["y"] = torch.empty((m, n), dtype=DTYPES[case["out"]], device="cuda")
    s["workspace"] = torch.empty(m * (k + 128) * 2 + (64 << 20), dtype=torch.uint8, device="cuda")
    return s


def _prepare_train(case, gen, s, seed):
    m, n, k = case["m"], case["n"], case["k"]
    half = case["dtype"] == "f16"  # its gradients come with the loss scaled
    s["x"] = _normal(gen, (m, k), 1.0, DTYPES[case["dtype"]])
    s["w"] = _normal(gen, (n, k), 0.02, DTYPES[case["dtype"]])
    s["dy"] = _normal(gen, (m, n), (1.0 if half else 1e-3) / 64, DTYPES[case["dtype"]])
    s["y"] = torch.empty((m, n), dtype=DTYPES[case["dtype"]], device="cuda")
    s["dx"] = torch.empty((m, k), dtype=DTYPES[case["dtype"]], device="cuda")
    s["dw"] = torch.empty((n, k), dtype=DTYPES[case["grad"]], device="cuda")
    f8, up = torch.float8_e4m3fn, lambda v: -(-v // 128)
    for name, (r, c), square in (("x", (m, k), False), ("w", (n, k), True), ("dy", (m, n), False)):
        # the codes along rows and along columns (transposed), and a row of scales for each 128 of the summed axis
        s[name + "8"] = torch.empty((r, 128 * up(c)), dtype=f8, device="cuda")
        s[name + "8_t"] = torch.empty((c, 128 * up(r)), dtype=f8, device="cuda")
        s[name + "_scale"] = torch.empty((up(c), up(r) if square else r), device="cuda")
        s[name + "_scale_t"] = torch.empty((up(r), up(c) if square else c), device="cuda")
    s["workspace"] = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    return s


def _prepare_adamw(case, gen, s, seed):
    """Tensors are views of flat buffers in which each starts at a multiple of 256 elements; those with moments in 8 bits lie in
    a buffer of their own. Blocks' numbers for the thresholds stand beside them."""
    sizes = _tensor_sizes(case)
    s["seed"] = seed % 1000003
    s["decay"] = [DECAY if n >= 4096 else 0.0 for n in sizes]
    first, piece = [], 0
    for n in sizes:
        first.append(piece)
        piece += -(-n // PIECE)
    s["views"] = [None] * len(sizes)
    for bits in (32, 8):
        mine = [i for i, n in enumerate(sizes) if _state_bits(case, n) == bits]
        if not mine:
            continue
        blocks = torch.tensor([-(-sizes[i] // 256) for i in mine], device="cuda")
        start = (blocks.cumsum(0) - blocks).tolist()
        total = 256 * int(blocks.sum())
        tensor_of = torch.repeat_interleave(torch.arange(len(mine), device="cuda"), blocks)
        local = torch.arange(total // 256, device="cuda") - torch.tensor(start, device="cuda")[tensor_of]
        left = torch.tensor([sizes[i] for i in mine], device="cuda")[tensor_of] - 256 * local
        there = torch.arange(256, device="cuda") < left[:, None]  # the places that hold elements
        x = _normal(gen, (total // 256, 256), 0.02)
        g = _normal(gen, (total // 256, 256), 1e-3)
        g *= torch.empty((1, 256), device="cuda").uniform_(0.05, 2.0, generator=gen)
        m = _normal(gen, (total // 256, 256), 3e-4)
        v = torch.empty((total // 256, 256), device="cuda").uniform_(0.2, 2.0, generator=gen).square_().mul_(1e-6)
        for t in (x, g, m, v):
            t.masked_fill_(~there, 0.0)
        p = {"x": x.view(-1), "g": g.to(DTYPES[case["dtype"]]).view(-1)}
        p["copy"] = None if case["copy"] == "none" else x.to(DTYPES[case["copy"]]).view(-1)
        p["decay"] = torch.tensor([s["decay"][i] for i in mine], device="cuda")[tensor_of][:, None]
        if bits == 32:
            p["m"], p["v"] = m.view(-1), v.view(-1)
        else:
            most, root = m.abs().amax(1, keepdim=True), v.amax(1, keepdim=True).sqrt()
            c = (m.abs() / most * 127.0 ** 2).sqrt().round().clamp(max=127.0) * m.sign()
            p["m"] = c.to(torch.int8).view(-1)
            c = (v.sqrt() / root * 255.0 ** 2).sqrt().round().clamp(min=1.0, max=255.0)
            p["v"] = torch.where(there, c, 0.0).to(torch.uint8).view(-1)
            p["scale"] = torch.cat([most, root], 1).view(-1)
            p["block"] = 8 * torch.tensor([first[i] for i in mine], device="cuda")[tensor_of] + local
        s[bits] = p
        for i, at in zip(mine, start):
            lo, n = 256 * at, sizes[i]
            cut = {name: None if p[name] is None else p[name][lo:lo + n] for name in ("x", "g", "m", "v", "copy")}
            cut["scale"] = p["scale"][2 * at:2 * at + 2 * -(-n // 256)] if bits == 8 else None
            s["views"][i] = cut
    return s


def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"norm": _own_norm, "linear": _own_linear, "train": _own_train, "adamw": _own_adamw}[kind](s)
    return {"norm": _plain_norm, "linear": _plain_linear, "train": _plain_train, "adamw": _plain_adamw}[kind](s)


# ---- through the framework ------------------------------------------------------------------------------------------
def _own_norm(s):
    from paper_2302_02390_amd import binding as qb
    qb.qsdp_layer_norm(s["x"], s["w"], s["b"], EPS, s["y"], s["stats"])
    out = {"y": s["y"], "stats": s["stats"]}
    if s["case"]["grad"]:
        qb.qsdp_layer_norm_backward(s["x"], s["w"], s["stats"], s["dy"], s["dx"], s["dw"], s["db"], False, s["workspace"])
        out.update(dx=s["dx"], dw=s["dw"], db=s["db"])
    return out


def _own_linear(s):
    from paper_2302_02390_amd import binding as qb
    qb.qsdp_linear_blocks(s["x"], s["w"], s["w_scale"], s["bias"], s["y"], s["workspace"])
    return {"y": s["y"]}


def _own_train(s):
    from paper_2302_02390_amd import binding as qb
    m, n, k = (s["case"][i] for i in "mnk")
    qb.qsdp_quantize_blocks(s["x"], False, s["x8"], s["x_scale"], s["x8_t"], s["x_scale_t"])
    qb.qsdp_quantize_blocks(s["w"], True, s["w8"], s["w_scale"], s["w8_t"], s["w_scale_t"])
    qb.qsdp_quantize_blocks(s["dy"], False, s["dy8"], s["dy_scale"], s["dy8_t"], s["dy_scale_t"])
    qb.qsdp_matmul_blocks(s["x8"], s["x_scale"], s["w8"], s["w_scale"], k, None, s["y"], False, s["workspace"])
    qb.qsdp_matmul_blocks(s["dy8"], s["dy_scale"], s["w8_t"], s["w_scale_t"], n, None, s["dx"], False, s["workspace"])
    qb.qsdp_matmul_blocks(s["dy8_t"], s["dy_scale_t"], s["x8_t"], s["x_scale_t"], m, None, s["dw"], False, s["workspace"])
    return {"y": s["y"], "dx": s["dx"], "dw": s["dw"]}


def _own_adamw(s):
    from paper_2302_02390_amd import binding as qb
    if "table" not in s:  # a program makes it once for its parameters
        v = s["views"]
        s["table"] = qb.AdamWTensors([t["x"] for t in v], [t["g"] for t in v], [t["m"] for t in v], [t["v"] for t in v],
                                     [t["scale"] for t in v], [t["copy"] for t in v], weight_decay=s["decay"])
    qb.qsdp_adamw_tensors(s["table"], LR, BETA1, BETA2, ADAM_EPS, 1 - BETA1 ** STEP, 1 - BETA2 ** STEP, s["seed"])
    return _adamw_outputs(s)


def _adamw_outputs(s):
    """The state's own buffers; moments in 8 bits as their codes, whole numbers that are the same where the values are, with
    the blocks' scales."""
    return {f"{bits}.{name}": s[bits][name] for bits in (32, 8) if bits in s for name in ("x", "copy", "m", "v", "scale")
            if s[bits].get(name) is not None}


# ---- plain forms ------------------------------------------------------------------------------------------------------
def _plain_norm(s):
    x, w, b = s["x"].float(), s["w"].float(), s["b"].float()
    mean = x.mean(1, keepdim=True)
    centred = x - mean
    rstd = 1.0 / (centred.square().mean(1, keepdim=True) + EPS).sqrt()
    h = centred * rstd
    out = {"y": (h * w + b).to(s["y"].dtype), "stats": torch.cat([mean, rstd], 1)}
    if s["case"]["grad"]:
        dy = s["dy"].float()
        g = dy * w
        dx = rstd * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
        out.update(dx=dx.to(s["dx"].dtype), dw=(dy * h).sum(0), db=dy.sum(0))
    return out


def _held(x, high, wide):
    """The values that stand for x once it is rounded in blocks."""
    rows, cols = x.shape
    whole = _whole(x, high, wide)
    codes, scale = _rounded(whole, high, wide)
    blocks = codes.float().view(whole.shape[0] // high, high, -1, wide) * scale[:, None, :, None]
    return blocks.view(whole.shape)[:rows, :cols]


def _plain_linear(s):
    n, k = s["case"]["n"], s["case"]["k"]
    x = _held(s["x"].float(), 1, 128)
    scale = s["w_scale"].t().repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]
    y = x @ (s["w"].float()[:, :k] * scale).t()
    if s["bias"] is not None:
        y = y + s["bias"]
    return {"y": y.to(s["y"].dtype)}


def _plain_train(s):
    x, w, dy = s["x"].float(), s["w"].float(), s["dy"].float()
    held = _held(w, 128, 128)
    return {"y": (_held(x, 1, 128) @ held.t()).to(s["y"].dtype), "dx": (_held(dy, 1, 128) @ held).to(s["dx"].dtype),
            "dw": (_held(dy, 128, 1).t() @ _held(x, 128, 1)).to(s["dw"].dtype)}


def _moments(p):
    """m and v that the codes stand for."""
    scale = p["scale"].view(-1, 2)
    c = p["m"].view(-1, 256).float()
    m = (scale[:, :1] * (1.0 / 127 ** 2)) * (c * c.abs())
    c = p["v"].view(-1, 256).float()
    root = (scale[:, 1:] * (1.0 / 255 ** 2)) * (c * c)
    return m, root * root


def _moved(p, m, v):
    """x, m and v after the step, [blocks, 256]; sums as one rounding of the exact product and addend."""
    g = p["g"].view(-1, 256).float()
    b1, b2 = (torch.tensor(b, device=g.device) for b in (BETA1, BETA2))
    m = (b1.double() * m.double() + (g * (1 - b1)).double()).float()
    v = (b2.double() * v.double() + ((g * (1 - b2)) * g).double()).float()
    x = p["x"].view(-1, 256)
    u = (m / (1 - BETA1 ** STEP)) / (v.sqrt() / math.sqrt(1 - BETA2 ** STEP) + ADAM_EPS)
    return x - LR * (u + p["decay"] * x), m, v


def _words(block, seed):
    """The first two words of the Philox4x32-10 blocks with key `seed` and counters (block, 0, 3, 0)."""
    low = 0xFFFFFFFF

    def product(a, c):  # upper and lower half, out of two that fit 64 bits
        top, bottom = (c >> 16) * a, (c & 0xFFFF) * a
        whole = top + (bottom >> 16)
        return whole >> 16, ((whole & 0xFFFF) << 16) | (bottom & 0xFFFF)

    c = [block & low, block >> 32, torch.full_like(block, 3), torch.zeros_like(block)]
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        (h0, l0), (h1, l1) = product(0xD2511F53, c[0]), product(0xCD9E8D57, c[2])
        c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c[0], c[1]


def _codes(value, word, most):
    """{codes, largest} of rows of 256 values that are not negative; codes up to `most`."""
    largest = value.amax(1, keepdim=True)
    some = largest >= 2.0 ** -96
    w = value * torch.where(some, torch.full_like(largest, most * most) / largest, 0.0)
    c = w.sqrt().floor()
    t = (word[:, None] + torch.arange(256, device=word.device) * 0x9E3779B9) & 0xFFFFFFFF
    t = ((t >> 20).float() + 0.5) * 2.0 ** -12
    c = torch.where(w - c * c > (2.0 * c + 1.0) * t, c + 1.0, c)
    return c.clamp(max=float(most)), torch.where(some, largest, 0.0)


def _plain_adamw(s):
    if 32 in s:
        p = s[32]
        x, m, v = _moved(p, p["m"].view(-1, 256), p["v"].view(-1, 256))
        _store(p, x, m, v)
    if 8 in s:
        p = s[8]
        x, m, v = _moved(p, *_moments(p))
        word_m, word_v = _words(p["block"], s["seed"])
        c, most = _codes(m.abs(), word_m, 127)
        root = v.double().sqrt().float()
        r, most_root = _codes(root, word_v, 255)
        r = torch.where((root > 0) & (most_root > 0), r.clamp(min=1.0), r)
        _store(p, x, (c * m.sign()).to(torch.int8), r.to(torch.uint8))
        p["scale"].copy_(torch.cat([most, most_root], 1).view(-1))
    return _adamw_outputs(s)


def _store(p, x, m, v):
    p["x"].copy_(x.view(-1))
    p["m"].copy_(m.view(-1))
    p["v"].copy_(v.view(-1))
    if p["copy"] is not None:
        p["copy"].copy_(p["x"])


# ---- in 64 bits -------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "linear": _exact_linear, "train": _exact_train, "adamw": _exact_adamw}[case["kind"]](case, s)


def _exact_norm(case, s):
    x, w, b = s["x"].double(), s["w"].double(), s["b"].double()
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    sigma = torch.sqrt(var + EPS)
    h = (x - mean) / sigma
    out = {"y": torch.addcmul(b, h, w), "stats": torch.cat([mean, 1.0 / sigma], 1)}
    if case["grad"]:
        dy = s["dy"].double()
        n = case["n"]
        a = (dy * w).sum(1, keepdim=True)
        c = (dy * w * h).sum(1, keepdim=True)
        out.update(dx=(n * dy * w - a - h * c) / (n * sigma), dw=torch.einsum("rn,rn->n", dy, h), db=dy.sum(0))
    return out


def _exact_held(x, axis, square=False):
    """x in 64 bits as its blocks hold it; what is held in 32 bits (largest, quotient, scale) and in 8 is so by definition."""
    x = x.to(torch.float32)
    if axis == 0:
        return _exact_held(x.t().contiguous(), 1, square).t()
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for lo in range(0, x.shape[1], 128):
        part = x[:, lo:lo + 128]
        most = part.abs().max(1).values
        if square:
            tall = torch.zeros(-(-len(most) // 128) * 128, device=x.device)
            tall[:len(most)] = most
            most = tall.view(-1, 128).max(1).values.repeat_interleave(128)[:len(most)]
        most = torch.maximum(most, torch.tensor(2.0 ** -100, device=x.device)).double()
        up, scale = (448.0 / most).float(), (most / 448.0).float()
        codes = torch.clamp(part * up[:, None], -448.0, 448.0).to(torch.float8_e4m3fn)
        out[:, lo:lo + 128] = codes.double() * scale.double()[:, None]
    return out


def _exact_linear(case, s):
    x = _exact_held(s["x"], 1)
    y = torch.zeros((case["m"], case["n"]), dtype=torch.float64, device="cuda")
    rows = torch.arange(case["n"], device="cuda") // 128
    for block, lo in enumerate(range(0, case["k"], 128)):
        hi = min(lo + 128, case["k"])
        w = s["w"].double()[:, lo:hi] * s["w_scale"][block].double()[rows][:, None]
        y.addmm_(x[:, lo:hi].contiguous(), w.t().contiguous())
    return {"y": y if s["bias"] is None else y + s["bias"].double()}


def _exact_train(case, s):
    w = _exact_held(s["w"], 1, True)
    y = _exact_held(s["x"], 1) @ w.t().contiguous()
    dx = _exact_held(s["dy"], 1) @ w
    dw = _exact_held(s["dy"], 0).t().contiguous() @ _exact_held(s["x"], 0).contiguous()
    return {"y": y, "dx": dx, "dw": dw}


def _exact_adamw(case, s):
    out = {}
    for bits in (32, 8):
        if bits not in s:
            continue
        p = s[bits]
        if bits == 32:
            m, v = p["m"].double(), p["v"].double()
        else:
            of = p["scale"].double().view(-1, 2).repeat_interleave(256, 0)
            m = of[:, 0] * p["m"].double() * p["m"].double().abs() / 16129.0
            v = (of[:, 1] * p["v"].double().square() / 65025.0).square()
        g, x = p["g"].double(), p["x"].double()
        m = BETA1 * m + (1.0 - BETA1) * g
        v = BETA2 * v + (1.0 - BETA2) * g * g
        u = m / (1.0 - BETA1 ** STEP) / (torch.sqrt(v / (1.0 - BETA2 ** STEP)) + ADAM_EPS)
        decay = p["decay"].double().expand(-1, 256).reshape(-1)
        x = x * (1.0 - LR * decay) - LR * u
        out[f"{bits}.x"] = x
        if p["copy"] is not None:
            out[f"{bits}.copy"] = x
        if bits == 32:
            out["32.m"], out["32.v"] = m, v
        else:
            out["8.scale"] = torch.stack([m.view(-1, 256).abs().amax(1), v.view(-1, 256).amax(1).sqrt()], 1).view(-1)
    return out
