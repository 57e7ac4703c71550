"""What is timed when the speed of drawing answers and of clipping gradients is looked at.

Three operators, which a program that learns from what its neighbours say runs beside those on messages and logits:

  sample   a token of every row of logits from a given random number u in [0, 1), and its log-probability.  The row's order is: larger
           logits first, of equal ones the lower index.  With e = exp((z - max z) / temperature), what is kept is a beginning of that
           order: its first top_k; of these the fewest whose e add up to top_p times the sum of them all; of these those with
           e >= min_p.  The token is the first at which the sum of e passes u times the sum of what is kept.
  norm     the Euclidean norm of each worker's gradient, which lies in many tensors
  clip     the gradient of each worker, scaled to a largest norm, as a row of fp32: what ds_step takes

`own` = False computes them in plain torch operations, True calls the library.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ---- cases --------------------------------------------------------------------------------------

def _sample(name, rows, vocab, dtype, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, masked=0.0, each=False):
    c = {"op": "sample", "rows": rows, "vocab": vocab, "dtype": dtype, "temperature": temperature, "top_k": top_k, "top_p": top_p,
         "min_p": min_p, "masked": masked, "each": each}
    if name:
        c["name"] = name
    return c


def _gradient(name, op, workers, total, tensors, dtype):
    c = {"op": op, "workers": workers, "total": total, "tensors": tensors, "dtype": dtype}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One token of one sequence, a middling vocabulary, the filters that decoding is mostly run with: latency is all there is.
        _sample("sample_1x32000_bf16_k50_p95", 1, 32000, "bf16", 0.8, 50, 0.95),
        # One token from a large vocabulary in the type of the framework's own state, by mass alone.
        _sample("sample_1x131072_f32_p90", 1, 131072, "f32", 1.0, 0, 0.9),
        # A serving batch: every sequence with parameters of its own, odd vocabulary, some of it forbidden.
        _sample("sample_24x50001_f16_each", 24, 50001, "f16", 0.9, 40, 0.92, 0.02, 0.3, True),
        # A few hundred sequences, odd vocabulary, kept by their ratio to the largest.
        _sample("sample_256x32003_f32_min5", 256, 32003, "f32", 1.0, 0, 1.0, 0.05),
        # Answers to a training batch, cut by mass.
        _sample("sample_1024x131072_bf16_p95", 1024, 131072, "bf16", 1.0, 0, 0.95),
        # The same with many tokens, cut by rank and by mass.
        _sample("sample_2048x65536_f32_k100_p90", 2048, 65536, "f32", 0.7, 100, 0.9),
        # The largest: a long batch drawn from everything.
        _sample("sample_4096x131072_bf16", 4096, 131072, "bf16"),
        # A small model's gradient in a few tensors: latency.
        _gradient("norm_1x100003_f32", "norm", 1, 100003, 12, "f32"),
        # Eight workers with a gradient in half precision each, as backward passes leave it.
        _gradient("norm_8x25600000_bf16", "norm", 8, 25600000, 161, "bf16"),
        # A small model again, into the row that the step takes.
        _gradient("clip_4x30011_f32", "clip", 4, 30011, 10, "f32"),
        # Sixteen workers with gradients of both kinds of 16 bits and of 32, odd lengths.
        _gradient("clip_16x11173962_mixed", "clip", 16, 11173962, 62, "mixed"),
        # Thirty-two workers of 25.6 million parameters.
        _gradient("clip_32x25600000_f32", "clip", 32, 25600000, 161, "f32"),
    ]


def draw(rng):
    """1 .. 4096 rows of 16 .. 262144 logits, or 1 .. 32 workers' gradients of 1000 .. 25.6 million elements in 1 .. 160 tensors."""
    def log(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    op = rng.choice(["sample", "sample", "sample", "norm", "clip"])
    if op == "sample":
        dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
        vocab = log(16, 262144)
        rows = max(1, min(log(1, 4096), 2 ** (28 if dtype == "f32" else 29) // vocab))
        if rng.random() < 0.3:
            vocab = 2 ** int(math.log2(vocab))
        top_k = 0 if rng.random() < 0.5 else min(vocab, log(1, 1000))
        top_p = 1.0 if rng.random() < 0.4 else rng.uniform(0.3, 0.99)
        min_p = 0.0 if rng.random() < 0.6 else rng.uniform(0.005, 0.3)
        return _sample("", rows, vocab, dtype, rng.uniform(0.5, 1.5), top_k, top_p, min_p, rng.choice([0.0, 0.0, 0.0, 0.6]),
                       rng.random() < 0.2)
    workers, total = log(1, 32), log(1000, 25600000)
    return _gradient("", op, workers, total, min(total, log(1, 160)), rng.choice(["f32", "bf16", "f16", "mixed"]))


# ---- what a program has in hand before the call ---------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _lengths(total, tensors):
    """Lengths of a model's tensors, `total` in all: matrices, and vectors a thousandth of their size among them."""
    rng = random.Random(tensors)
    share = [(1.0 if i % 3 == 0 else 0.001) * 64.0 ** rng.random() for i in range(tensors)]
    spare, scale = total - tensors, sum(share)
    lengths = [1 + int(spare * s / scale) for s in share]
    lengths[0] += total - sum(lengths)
    return lengths


def _tensor_dtypes(case):
    if case["dtype"] != "mixed":
        return [DTYPES[case["dtype"]]] * case["tensors"]
    return [(torch.bfloat16, torch.float32, torch.float16)[i % 3] for i in range(case["tensors"])]


def prepare(case, seed):
    g = _generator(seed)
    state = dict(case)
    if case["op"] == "sample":
        rows, vocab = case["rows"], case["vocab"]
        dtype = DTYPES[case["dtype"]]
        z = torch.empty((rows, vocab), dtype=dtype, device="cuda")
        for lo in range(0, rows, 512):
            part = torch.randn((min(512, rows - lo), vocab), generator=g, device="cuda").mul_(3.0)
            if case["masked"]:
                # Tokens that a grammar forbids; the first stays.
                forbidden = torch.rand(part.shape, generator=g, device="cuda") < case["masked"]
                forbidden[:, 0] = False
                part.masked_fill_(forbidden, -math.inf)
            z[lo:lo + 512] = part
        state["z"] = z
        state["u"] = torch.rand(rows, generator=g, device="cuda")
        if case["each"]:
            def around(value, lo, hi, dtype=torch.float32):
                f = 0.75 + 0.5 * torch.rand(rows, generator=g, device="cuda")
                return (f * value).clamp(lo, hi).to(dtype)
            state["temperature"] = around(case["temperature"], 0.1, 10.0)
            state["top_k"] = around(case["top_k"], 0, vocab, torch.int32)
            state["top_p"] = around(case["top_p"], 0.0, 1.0)
            state["min_p"] = around(case["min_p"], 0.0, 1.0)
        return state
    lengths, dtypes = _lengths(case["total"], case["tensors"]), _tensor_dtypes(case)
    state["grads"] = [[(torch.randn(n, generator=g, device="cuda") * 0.01).to(t) for n, t in zip(lengths, dtypes)]
                      for _ in range(case["workers"])]
    # About two workers of three are above the largest norm.
    for w, tensors in enumerate(state["grads"]):
        if w % 3 == 2:
            for t in tensors:
                t.mul_(0.25)
    state["max_norm"] = 0.005 * math.sqrt(case["total"])
    if case["op"] == "clip":
        # Rows as long as a step's state keeps them: padded to whole tiles.
        pitch = (case["total"] + 4095) // 4096 * 4096
        state["g"] = torch.zeros((case["workers"], pitch), device="cuda")
    if own:
        from paper_1907_07346_amd import binding as b
        state["table"] = b.Gradients(state["grads"])         # a program lays it out once, and keeps it with the tensors
    return state


# ---- one pass ---------------------------------------------------------------------------------------

def _column(value, like, dtype):
    """A parameter as a column, rounded to fp32 as the call takes it."""
    if torch.is_tensor(value):
        return value.to(dtype)[:, None]
    return torch.full((like.shape[0], 1), value, dtype=torch.float32 if dtype == torch.float64 else dtype, device=like.device).to(dtype)


def _run_plain(s):
    op = s["op"]
    if op == "sample":
        z, u = s["z"], s["u"]
        rows, vocab = z.shape
        t, k = _column(s["temperature"], z, torch.float64), _column(s["top_k"], z, torch.int64)
        p, least = _column(s["top_p"], z, torch.float64), _column(s["min_p"], z, torch.float64)
        k = torch.where(k == 0, vocab, k)
        token = torch.empty(rows, dtype=torch.int32, device=z.device)
        logp = torch.empty(rows, device=z.device)
        step = max(1, 2 ** 26 // vocab)
        for lo in range(0, rows, step):
            hi = min(rows, lo + step)
            a, order = (z[lo:hi].float() + 0.0).sort(dim=1, descending=True, stable=True)
            y = (a.double() - a[:, :1].double()) / t[lo:hi]
            e = y.exp()
            e = torch.where(torch.arange(vocab, device=z.device) < k[lo:hi], e, 0.0)
            upto = e.cumsum(dim=1)
            before = torch.cat([torch.zeros_like(upto[:, :1]), upto[:, :-1]], dim=1)
            e = torch.where((before < p[lo:hi] * upto[:, -1:]) & (e >= least[lo:hi]), e, 0.0)
            upto = e.cumsum(dim=1)
            total = upto[:, -1:]
            place = (upto <= u[lo:hi, None].double() * total).sum(dim=1, keepdim=True)
            place = torch.minimum(place, (e > 0).sum(dim=1, keepdim=True) - 1)
            token[lo:hi] = order.gather(1, place)[:, 0].to(torch.int32)
            logp[lo:hi] = (y.gather(1, place) - total.log())[:, 0].float()
        return {"token": token, "logp": logp}
    squares = [sum(x.double().square().sum() for x in tensors) for tensors in s["grads"]]
    norm = torch.stack(squares).sqrt()
    if op == "norm":
        return norm.float()
    factor = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0)
    g = s["g"]
    for w, tensors in enumerate(s["grads"]):
        at = 0
        for x in tensors:
            g[w, at:at + x.numel()] = x.double() * factor[w]
            at += x.numel()
    return {"g": g, "norm": norm.float()}


def _run_own(s):
    from paper_1907_07346_amd import binding as b
    if s["op"] == "sample":
        token, logp = b.ds_sample(s["z"], s["u"], s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
        return {"token": token, "logp": logp}
    if s["op"] == "norm":
        return b.ds_gradient_norm(s["table"])
    return {"g": s["g"], "norm": b.ds_clip(s["table"], s["max_norm"], out=s["g"])}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without, and what it should give --------------------------------------------

def work(case):
    if case["op"] == "sample":
        rows, vocab = case["rows"], case["vocab"]
        size = 4 if case["dtype"] == "f32" else 2
        return {"bytes": rows * (vocab * size + 12 + (16 if case["each"] else 0)), "flops": 4 * rows * vocab}
    lengths, dtypes = _lengths(case["total"], case["tensors"]), _tensor_dtypes(case)
    read = case["workers"] * sum(n * torch.empty(0, dtype=t).element_size() for n, t in zip(lengths, dtypes))
    elements = case["workers"] * case["total"]
    if case["op"] == "norm":
        return {"bytes": read + 4 * case["workers"], "flops": 2 * elements}
    return {"bytes": read + 4 * elements + 4 * case["workers"], "flops": 3 * elements}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "sample":
        z, vocab = s["z"], case["vocab"]

        def of(name, row):
            value = s[name]
            return float(value[row]) if torch.is_tensor(value) else float(torch.tensor(value, dtype=torch.float32))

        token, logp = [], []
        for row in range(case["rows"]):
            y = z[row].double() / of("temperature", row)
            bits = (z[row].float() + 0.0).view(torch.int32).long()
            key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * 2 ** 32 - torch.arange(vocab, device=z.device)
            order = key.argsort(descending=True)
            if of("top_k", row):
                order = order[:int(of("top_k", row))]
            log_p = torch.log_softmax(y[order], dim=0)
            mass = log_p.exp().cumsum(0)
            last = int(torch.searchsorted(mass, mass[-1] * of("top_p", row))) + 1 if of("top_p", row) < 1.0 else len(order)
            if of("min_p", row):
                last = min(last, int((log_p - log_p[0] >= math.log(of("min_p", row))).sum()))
            mass = mass[:last]
            place = min(int(torch.searchsorted(mass, s["u"][row].double() * mass[-1], right=True)), int((log_p[:last] > -math.inf).sum()) - 1)
            token.append(order[place])
            logp.append(log_p[place] - mass[-1].log())
        return {"token": torch.stack(token).to(torch.int32), "logp": torch.stack(logp)}
    rows = torch.stack([torch.cat([x.double() for x in tensors]) for tensors in s["grads"]])
    norm = torch.linalg.vector_norm(rows, dim=1)
    if case["op"] == "norm":
        return norm
    rows *= (s["max_norm"] / norm).clamp(max=1.0)[:, None]
    return {"g": torch.nn.functional.pad(rows, (0, s["g"].shape[1] - rows.shape[1])), "norm": norm}
