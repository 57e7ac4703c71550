"""What is timed when the speed of the operators on messages and logits is looked at.

Four operators, which a program that learns from its neighbours' answers runs one after the other:

  product    y[t, r] = sum over c of x[t, c] * M[r, c]: tokens through a matrix that is held as a message (4-bit codes, a
             scale per block; row r of the matrix is laid out as worker r's message of DS_COMP_QUANT_MAXABS, bits = 4)
  gradient   dx[t, c] = sum over r of dy[t, r] * M[r, c]: the gradient of that product with respect to x
  top        the k largest logits of every row as (index, value) pairs, and the row's log-sum-exp: what a teacher sends
  distill    the loss of a student's logits against such pairs, and its gradient with respect to the logits

`own` = False computes them in plain torch operations, True calls the library.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ---- cases --------------------------------------------------------------------------------------

def _matrix(name, op, tokens, rows, cols, block, dtype):
    c = {"op": op, "tokens": tokens, "rows": rows, "cols": cols, "block": block, "dtype": dtype}
    if name:
        c["name"] = name
    return c


def _logits(name, op, rows, vocab, k, dtype, temperature=1.0, lse=False):
    c = {"op": op, "rows": rows, "vocab": vocab, "k": k, "dtype": dtype, "temperature": temperature, "lse": lse}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One token through a small square layer, in the type of the framework's own state: latency is all there is.
        _matrix("product_1_2048x2048_f32", "product", 1, 2048, 2048, 512, "f32"),
        # One token through an output layer: the logits of a neighbour's model, straight from its message.
        _matrix("product_1_65536x4096_bf16", "product", 1, 65536, 4096, 128, "bf16"),
        # A decoding batch through a wide layer.
        _matrix("product_16_4096x16384_f16", "product", 16, 4096, 16384, 256, "f16"),
        # A short prompt, nothing a multiple of anything, the smallest block.
        _matrix("product_61_16001x4099_bf16", "product", 61, 16001, 4099, 64, "bf16"),
        # A few tokens' gradient through a small layer.
        _matrix("gradient_7_2048x2000_bf16", "gradient", 7, 2048, 2000, 128, "bf16"),
        # A training batch's gradient through an output layer.
        _matrix("gradient_64_32768x4096_bf16", "gradient", 64, 32768, 4096, 512, "bf16"),
        # The same in the framework's own type, with a ragged last block.
        _matrix("gradient_16_8192x5000_f32", "gradient", 16, 8192, 5000, 1024, "f32"),
        # A teacher that answers one token.
        _logits("top64_1x131072_bf16", "top", 1, 131072, 64, "bf16"),
        # A teacher that answers a training batch.
        _logits("top128_2048x65536_f32", "top", 2048, 65536, 128, "f32", 2.0),
        # A handful of tokens, odd vocabulary; also the case with the least work of its operator.
        _logits("distill16_8x32003_f32", "distill", 8, 32003, 16, "f32", 2.0),
        # A training batch with a middling vocabulary and odd sizes; the teacher's own log-sum-exp is given.
        _logits("distill100_1023x50001_f16", "distill", 1023, 50001, 100, "f16", 1.0, True),
        # The largest: a long training batch with a large vocabulary.
        _logits("distill64_4096x131072_bf16", "distill", 4096, 131072, 64, "bf16"),
    ]


def draw(rng):
    """1 .. 64 tokens through 16 .. 65536 rows by 64 .. 16384 columns, or 1 .. 4096 rows of 16 .. 262144 logits."""
    def log(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    op = rng.choice(["product", "product", "gradient", "top", "distill"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    if op in ("product", "gradient"):
        tokens = 1 if op == "product" and rng.random() < 0.4 else log(1, 64)
        cols = log(64, 16384)
        rows = max(16, min(log(16, 65536), 2 ** 28 // cols, 2 ** 32 // (cols * tokens)))
        if rng.random() < 0.3:                                  # powers of two, too
            cols, rows = 2 ** int(math.log2(cols)), 2 ** int(math.log2(rows))
        return _matrix("", op, tokens, rows, cols, rng.choice([64, 128, 256, 512, 1024, 2048]), dtype)
    vocab = log(16, 262144)
    rows = max(1, min(log(1, 4096), 2 ** (28 if op == "top" or dtype == "f32" else 29) // vocab))
    if rng.random() < 0.3:
        vocab = 2 ** int(math.log2(vocab))
    return _logits("", op, rows, vocab, min(vocab, log(1, 256)), dtype, rng.choice([1.0, 2.0]), rng.random() < 0.5)


# ---- what a program has in hand before the call ---------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _pack(w, block):
    """The rows of w as messages: per block [f32 scale][one u32 word per eight codes], code to the nearest level."""
    rows, cols = w.shape
    parts = []
    whole = cols // block * block
    for lo, hi, m in ((0, whole, block), (whole, cols, cols - whole)):
        if hi == lo:
            continue
        v = w[:, lo:hi].reshape(rows, (hi - lo) // m, m)
        scale = v.abs().amax(dim=2, keepdim=True)
        codes = torch.clamp(torch.round((v / scale + 1.0) * 7.5), 0, 15).to(torch.int32)
        codes = torch.nn.functional.pad(codes, (0, -m % 8)).reshape(rows, (hi - lo) // m, -1, 8)
        words = torch.zeros(codes.shape[:3], dtype=torch.int32, device=w.device)
        for i in range(8):
            words |= codes[..., i] << (4 * i)
        parts.append(torch.cat([scale.view(torch.int32), words], dim=2).reshape(rows, -1))
    return torch.cat(parts, dim=1).contiguous().view(torch.uint8)


def prepare(case, seed):
    g = _generator(seed)
    dtype = DTYPES[case["dtype"]]
    state = dict(case)
    if case["op"] in ("product", "gradient"):
        w = torch.randn((case["rows"], case["cols"]), generator=g, device="cuda") * 0.02
        state["message"] = _pack(w, case["block"])
        width = case["cols"] if case["op"] == "product" else case["rows"]
        state["in"] = torch.randn((case["tokens"], width), generator=g, device="cuda").to(dtype)
        return state
    rows, vocab, k = case["rows"], case["vocab"], case["k"]
    state["z"] = (torch.randn((rows, vocab), generator=g, device="cuda") * 3.0).to(dtype)
    if case["op"] == "distill":
        # The teacher's largest logits sit where the student's do, more or less: distinct, ascending indices.
        at = torch.randint(0, vocab - k + 1, (rows, k), generator=g, device="cuda").sort(dim=1).values
        at = (at + torch.arange(k, device="cuda")).to(torch.int32)
        value = torch.randn((rows, k), generator=g, device="cuda") * 1.5 + 9.0
        state["pairs"] = torch.stack([at, value.view(torch.int32)], dim=2).contiguous()
        # The mean over the batch; for gradients in half precision the sum, scaled up.  Padding tokens carry no weight.
        each = 1024.0 if case["dtype"] == "f16" else 1.0 / rows
        state["weight"] = (torch.rand(rows, generator=g, device="cuda") > 0.1).float() * each
        state["teacher_lse"] = None
        if case["lse"]:
            state["teacher_lse"] = torch.logsumexp(value.double() / case["temperature"], dim=1).float() + 0.2
    return state


# ---- one pass ---------------------------------------------------------------------------------------

def _decode(message, rows, cols, block):
    """(2 q - 15) * (scale / 15) of every element, fp32."""
    data = message.view(torch.int32).reshape(rows, -1)
    full = cols // block
    shifts = torch.arange(0, 32, 4, device=data.device, dtype=torch.int32)
    parts = []
    for lo, count, m in ((0, full, block), (full * (1 + block // 8), 1 if cols % block else 0, cols % block)):
        if count == 0:
            continue
        words = 1 + (m + 7) // 8
        part = data[:, lo:lo + count * words].reshape(rows, count, words)
        unit = part[:, :, :1].contiguous().view(torch.float32) / 15.0
        codes = ((part[:, :, 1:, None] >> shifts) & 15).reshape(rows, count, -1)[:, :, :m]
        parts.append(((2 * codes - 15).float() * unit).reshape(rows, count * m))
    return parts[0] if len(parts) == 1 else torch.cat(parts, dim=1)


def _lse(a):
    top = a.amax(dim=1, keepdim=True)
    return (a - top).exp().sum(dim=1).log() + top[:, 0]


def _run_plain(s):
    op = s["op"]
    if op in ("product", "gradient"):
        w = _decode(s["message"], s["rows"], s["cols"], s["block"])
        x = s["in"].float()
        return (x @ w.t() if op == "product" else x @ w).to(s["in"].dtype)
    z, tau = s["z"], s["temperature"]
    if op == "top":
        zf = z.float()
        bits = (zf + 0.0).view(torch.int32).long()
        order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)                  # as the numbers are ordered
        at = torch.arange(z.shape[1], device=z.device)
        key = order * 2 ** 32 + (2 ** 32 - 1 - at)                                 # ties: the lower index first
        index = key.topk(s["k"], dim=1).indices.sort(dim=1).values
        return {"index": index.to(torch.int32), "value": zf.gather(1, index), "lse": _lse(zf / tau)}
    index, a = s["pairs"][..., 0].long(), s["pairs"][..., 1].contiguous().view(torch.float32) / tau
    lse = _lse(a) if s["teacher_lse"] is None else s["teacher_lse"]
    log_p = a - lse[:, None]
    p = log_p.exp()
    y = z.float() / tau
    log_q = y - _lse(y)[:, None]
    loss = s["weight"] * (p * (log_p - log_q.gather(1, index))).sum(dim=1)
    grad = p.sum(dim=1, keepdim=True) * log_q.exp()
    grad.scatter_add_(1, index, -p)
    return {"loss": loss, "dz": (grad * (s["weight"] / tau)[:, None]).to(z.dtype)}


def _run_own(s):
    from paper_1907_07346_amd import binding as b
    op = s["op"]
    if op == "product":
        return b.ds_product(s["message"], s["in"], s["rows"], s["block"])
    if op == "gradient":
        return b.ds_product_gradient(s["message"], s["in"], s["cols"], s["block"])
    if op == "top":
        pairs, lse = b.ds_top_logits(s["z"], s["k"], s["temperature"])
        return {"index": pairs[..., 0], "value": pairs.view(torch.float32)[..., 1], "lse": lse}
    loss, dz = b.ds_distill(s["z"], s["pairs"], s["temperature"], teacher_lse=s["teacher_lse"], weight=s["weight"])
    return {"loss": loss, "dz": dz}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without, and what it should give --------------------------------------------

def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] in ("product", "gradient"):
        rows, cols, tokens = case["rows"], case["cols"], case["tokens"]
        full, tail = divmod(cols, case["block"])
        message = rows * (full * (4 + case["block"] // 2) + (4 + 4 * ((tail + 7) // 8) if tail else 0))
        return {"bytes": message + size * tokens * (rows + cols), "flops": 2 * rows * cols * tokens}
    rows, vocab, k = case["rows"], case["vocab"], case["k"]
    if case["op"] == "top":
        return {"bytes": rows * (vocab * size + 8 * k + 4), "flops": 4 * rows * vocab}
    return {"bytes": rows * (2 * vocab * size + 8 * k + 8 + (4 if case["lse"] else 0)), "flops": 8 * rows * vocab}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("product", "gradient"):
        rows, cols, block = s["rows"], s["cols"], s["block"]
        row = s["message"].reshape(rows, -1)
        pitch = 4 + block // 2
        w = torch.empty((rows, cols), dtype=torch.float64, device="cuda")
        for b, lo in enumerate(range(0, cols, block)):
            m = min(block, cols - lo)
            scale = row[:, b * pitch:b * pitch + 4].contiguous().view(torch.float32).double()
            data = row[:, b * pitch + 4:b * pitch + 4 + (m + 1) // 2]
            code = torch.stack([data & 15, data >> 4], dim=2).reshape(rows, -1)[:, :m].double()
            w[:, lo:lo + m] = scale * (2.0 * code - 15.0) / 15.0
        x = s["in"].double()
        if case["op"] == "product":
            return torch.cat([x @ w[lo:lo + 8192].t().contiguous() for lo in range(0, rows, 8192)], dim=1)
        return x @ w
    z, tau = s["z"].double(), case["temperature"]
    if case["op"] == "top":
        out = {"index": [], "value": [], "lse": torch.logsumexp(z / tau, dim=1)}
        for lo in range(0, z.shape[0], 256):
            order = z[lo:lo + 256].sort(dim=1, descending=True, stable=True).indices[:, :case["k"]].sort(dim=1).values
            out["index"].append(order)
            out["value"].append(z[lo:lo + 256].gather(1, order))
        return {"index": torch.cat(out["index"]).to(torch.int32), "value": torch.cat(out["value"]), "lse": out["lse"]}
    at, a = s["pairs"][..., 0].long(), s["pairs"].view(torch.float32)[..., 1].double() / tau
    total = torch.logsumexp(a, dim=1) if s["teacher_lse"] is None else s["teacher_lse"].double()
    p = torch.exp(a - total[:, None])
    z.div_(tau)
    own_total = torch.logsumexp(z, dim=1)
    weight = s["weight"].double()
    loss = weight * (p * (a - total[:, None] - z.gather(1, at) + own_total[:, None])).sum(dim=1)
    z.sub_(own_total[:, None]).exp_().mul_(p.sum(dim=1, keepdim=True)).scatter_add_(1, at, -p)
    return {"loss": loss, "dz": z.mul_((weight / tau)[:, None])}
