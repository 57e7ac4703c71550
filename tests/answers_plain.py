"""Plain implementations, in 64 bits, of the operators on messages and logits: what the tests compare with."""
import numpy as np
import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}       # of a rounding, relative to the value
SMALL = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}   # the smallest numbers above zero


def rounding(y, dtype):
    """How far a rounding of y (float64) to dtype may be off."""
    return HALF[dtype] * y.abs() + SMALL[dtype]


def row_bytes(cols, block):
    full, tail = divmod(cols, block)
    return full * (4 + block // 2) + (4 + 4 * ((tail + 7) // 8) if tail else 0)


def random_message(rows, cols, block, rng, scale=lambda shape, rng: rng.random(shape) + 0.01):
    """A matrix as messages with random codes: (bytes as uint8 tensor, codes, scales per block), made without any packing code."""
    nb = (cols + block - 1) // block
    codes = rng.integers(0, 16, (rows, cols))
    scales = np.asarray(scale((rows, nb), rng), np.float32)
    out = np.zeros((rows, row_bytes(cols, block)), np.uint8)
    for b in range(nb):
        at = b * (4 + block // 2)
        out[:, at:at + 4] = scales[:, b:b + 1].copy().view(np.uint8)
        part = codes[:, b * block:(b + 1) * block]
        part = np.pad(part, ((0, 0), (0, part.shape[1] % 2)))
        out[:, at + 4:at + 4 + part.shape[1] // 2] = part[:, 0::2] | part[:, 1::2] << 4
    return torch.from_numpy(out.reshape(-1)), codes, scales


def dense(codes, scales, block):
    """The matrix, float64."""
    unit = np.repeat(scales.astype(np.float64), block, axis=1)[:, :codes.shape[1]]
    return torch.from_numpy((2.0 * codes - 15.0) * unit / 15.0)


def decode(message, rows, cols, block):
    """The matrix of a message (uint8 numpy array), float64."""
    data = np.asarray(message, np.uint8).reshape(rows, -1)
    out = np.zeros((rows, cols))
    for b, lo in enumerate(range(0, cols, block)):
        at, m = b * (4 + block // 2), min(block, cols - lo)
        unit = data[:, at:at + 4].copy().view(np.float32).astype(np.float64) / 15.0
        part = data[:, at + 4:at + 4 + (m + 1) // 2]
        codes = np.stack([part & 15, part >> 4], axis=2).reshape(rows, -1)[:, :m]
        out[:, lo:lo + m] = (2.0 * codes - 15.0) * unit
    return torch.from_numpy(out)


def top(z, k):
    """Indices (ascending) of the k largest of each row: ties to the lower index, NaN above all."""
    order = np.empty((z.shape[0], k), np.int64)
    for i, row in enumerate(z.double().numpy()):
        key = np.where(np.isnan(row), np.inf, row)
        rank = np.lexsort((np.arange(len(row)), -key, ~np.isnan(row)))
        order[i] = np.sort(rank[:k])
    return torch.from_numpy(order)


def lse(a):
    """ln of the sum of exp over the last dimension, float64; minus infinity where there is nothing, plus infinity where one is."""
    top = a.amax(dim=-1, keepdim=True)
    ref = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    return (a - ref).exp().sum(dim=-1).log() + ref[..., 0]


def log_softmax(a):
    """a - lse(a), without adding what is to be taken off again (logits of -3e38 swallow it, in 64 bits too)."""
    top = a.amax(dim=-1, keepdim=True)
    a = a - torch.where(torch.isinf(top), torch.zeros_like(top), top)
    return a - a.exp().sum(dim=-1, keepdim=True).log()


def distill(z, index, value, temperature, teacher_lse=None, weight=None):
    """(loss, dz) of a row after the other; index int64 (rows, k), value float (rows, k)."""
    z, value = z.double() / temperature, value.double() / temperature
    rows, vocab = z.shape
    weight = torch.ones(rows, dtype=torch.float64) if weight is None else weight.double()
    loss, dz = torch.zeros(rows, dtype=torch.float64), torch.zeros_like(z)
    for i in range(rows):
        here = (index[i] >= 0) & (index[i] < vocab)
        at, a = index[i][here], value[i][here]
        if weight[i] == 0 or not len(at):
            continue
        log_p = log_softmax(a) if teacher_lse is None else a - teacher_lse[i].double()
        p = torch.where(a == -np.inf, torch.zeros_like(a), log_p.exp())
        if not torch.isnan(p).any() and p.sum() == 0:
            continue
        log_q = log_softmax(z[i])
        some = p != 0
        loss[i] = weight[i] * (p[some] * (log_p[some] - log_q[at[some]])).sum()
        dz[i] = weight[i] / temperature * (p.sum() * log_q.exp()).index_add(0, at, -p)
    return loss, dz


def sample_row(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logp) of a row (numpy, any float type), by a sorted list; parameters as the fp32 numbers they are given as."""
    z = np.asarray(z, np.float64)
    temperature, top_p, min_p, u = (float(np.float32(v)) for v in (temperature, top_p, min_p, u))
    if np.isnan(z).any():
        return -1, np.nan
    if z.max() == -np.inf:
        return -1, -np.inf
    order = np.lexsort((np.arange(len(z)), -z))
    greedy = not (2.0 ** -126 <= temperature < np.inf)
    if greedy:
        temperature, top_k = 1.0, 1
    z = z[order]
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        y = np.where(z == z[0], 0.0, (z - z[0]) / temperature)
    e = np.exp(y)
    last = len(z) if top_k <= 0 else min(top_k, len(z))
    mass = np.cumsum(e[:last])
    if top_p < 1.0:
        last = int(np.searchsorted(mass, top_p * mass[-1])) + 1 if top_p > 0 else 1
    if min_p > 0:
        last = min(last, int((e >= min(min_p, 1.0)).sum()))
    mass = mass[:last]
    u = 0.0 if not u > 0 else u
    place = int(np.searchsorted(mass, u * mass[-1], side="right")) if u < 1 else last
    place = min(place, int((e[:last] > 0).sum()) - 1)
    return int(order[place]), y[place] - np.log(mass[-1])


def sample(z, u, **parameters):
    """(token, logp) of rows; parameters are numbers or tensors of one per row."""
    rows = z.double().cpu().numpy()
    of = [{k: v[i].item() if torch.is_tensor(v) else v for k, v in parameters.items()} for i in range(len(rows))]
    got = [sample_row(rows[i], float(u[i]), **of[i]) for i in range(len(rows))]
    return torch.tensor([t for t, _ in got], dtype=torch.int32), torch.tensor([p for _, p in got], dtype=torch.float64)
