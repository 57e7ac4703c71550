"""Logits that lie far apart or far from zero: masks of every size beside one another, rows that hold nothing else, temperatures that take
exponents past what fp32 holds, teachers whose logits share a large offset.  Against 64 bits.

Tolerances.  U = 2^-24.  A term 2^((z - max) log2(e) / T) is off by 4 U d + 16 U of itself, d = (max - z) / T in units of e (the product's and the
exponential's rounding and the sum's).  The hardware's 2^x is 0 below 2^-126: a gradient, which is a term over T and over a sum of 1 or
more, may lack 2^-126 / T.  (Terms of 1e-38 of the largest, which 1e-40 / T left no room for.)  ln of the sum: the terms', and roundings at the size of
the result, of max / T and of ln V.  A loss past 3.4e38 has no number in fp32; p times -ln q = (max - z) / T below that has one, whatever -ln q is."""
import math

import numpy as np
import pytest
import torch

from paper_1907_07346_amd import binding as b
from tests import answers_plain as plain
from tests.test_gpu_answers import pack_pairs

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
LOWEST = torch.finfo(F32).min


def far_rows(rng, vocab, dtype):
    """(what, row): masks of one size over a stretch that threads, waves or parts see alone, beside other masks and ordinary logits."""
    usual = rng.standard_normal(vocab) * 3
    half, stretch = np.arange(vocab) < vocab // 2, np.arange(vocab) // 1024 % 2 == 0
    out = []
    for mask in (-1e4, -1e9, -1e10, -3e13, -1e20, -1e30, -1e38, -2e38, LOWEST):
        out += [(f"mask {mask}", np.where(half, mask, usual)), (f"mask {mask} last", np.where(half, usual, mask)), (f"mask {mask} in stretches", np.where(stretch, mask, usual)),
                (f"nothing but {mask}", np.full(vocab, mask))]
    for a, c in ((-1e38, -2e38), (-2.3e38, -2.4e38), (-1.7e38, LOWEST), (-1e30, LOWEST), (2.3e38, 2.4e38), (1e30, 1.1e30), (1e10, 1.5e10)):
        out += [(f"{a} and {c}", np.where(half, a, c)), (f"{c} and {a}", np.where(half, c, a)), (f"{a} and {c} in stretches", np.where(stretch, a, c)),
                (f"{a}, {c} and usual", np.where(stretch, a, np.where(half, c, usual)))]
    near = np.float32(1 << 28) + 32 * rng.integers(-4, 4, vocab)   # neighbours in fp32, whose exponents are far apart
    out += [("neighbours", near), ("30 and 29.99", np.where(half, 30.0, 29.99)), ("29.99 and 30", np.where(half, 29.99, 30.0))]
    return [n for n, _ in out], torch.from_numpy(np.stack([np.clip(r, LOWEST, -LOWEST) for _, r in out]).astype(np.float32)).clamp(min=torch.finfo(dtype).min, max=torch.finfo(dtype).max).to(dtype)


@pytest.mark.parametrize("temperature", [0.25, 0.5, 1.0, 2.0, 1e-37])
@pytest.mark.parametrize("vocab", [40, 5003, 20000, 150000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_sums_of_logits_far_apart(dtype, vocab, temperature):
    names, z = far_rows(np.random.default_rng(vocab), vocab, dtype)
    temperature = float(np.float32(temperature))
    rows, k = z.shape[0], 8
    zd = z.double()
    exact = plain.lse(zd / temperature)
    slack = U * (16 + 4 * 100 + 4 * math.log(vocab + 1))

    pairs, lse = b.ds_top_logits(z.cuda(), k, temperature)
    assert torch.equal(pairs.cpu()[..., 0].long(), plain.top(z, k))
    got = lse.cpu().double()
    biggest = (exact.abs() > 3.4028234e38)                        # (fp32 has no such number)
    want = torch.where(biggest, torch.sign(exact) * float("inf"), exact)
    off = torch.where(got == want, torch.zeros_like(got), (got - want).abs())
    bad = ~(off <= 4 * U * exact.abs() + slack) & ~(exact.abs() > 3.40e38)
    assert not bad.any(), f"lse: {[(names[i], got[i].item(), want[i].item()) for i in bad.nonzero()[:, 0].tolist()][:4]}"

    rng = np.random.default_rng(vocab + 1)
    index = torch.from_numpy(np.stack([np.sort(rng.permutation(vocab)[:k]) for _ in range(rows)])).long()
    index[:, 0] = 0                                               # ... one of which is surely not masked in some rows
    index, value = index.sort(dim=1).values, torch.from_numpy(rng.standard_normal((rows, k))).float() * temperature
    weight = torch.from_numpy(2.0 ** -rng.integers(0, 9, rows)).float()
    loss, dz = b.ds_distill(z.cuda(), pack_pairs(index, value).cuda(), temperature, weight=weight.cuda())
    want_loss, want = plain.distill(z, index, value, temperature, weight=weight)
    w = weight.double()
    log_q = plain.log_softmax(zd / temperature)
    dense = w[:, None] * log_q.exp() / temperature
    tol = U * (64 + 4 * 100) * (dense + want.abs()) + 2.0 ** -126 / temperature + plain.rounding(want, dtype)
    got = dz.cpu().double()
    over = want.abs() > 3.39e38
    off = torch.where((got == want) | over, torch.zeros_like(got), (got - want).abs())
    bad = ~(off <= tol)
    assert not bad.any(), f"dz: {[(names[i], j, got[i, j].item(), want[i, j].item()) for i, j in bad.nonzero().tolist()][:4]}"
    # the loss: sum p (ln p - ln q); ln q of a masked entry is as large as the mask
    p = torch.softmax(value.double() / temperature, dim=1)
    size = w * (p * log_q.gather(1, index).abs()).sum(dim=1)
    tol = 16 * U * size + w * U * (64 + 4 * 100 + 4 * math.log(vocab + 1)) + 4 * U * want_loss.abs()
    got = loss.cpu().double()
    over = size > 3.39e38
    bad = ~((got - want_loss).abs() <= tol) & ~over
    assert not bad.any(), f"loss: {[(names[i], got[i].item(), want_loss[i].item()) for i in bad.nonzero()[:, 0].tolist()][:4]}"


@pytest.mark.parametrize("offset", [0.0, 300.0, -5000.0, 1e5])
def test_teachers_and_students_with_a_common_offset(offset):
    """What logits have in common cancels: probabilities go by differences, which fp32 holds exactly."""
    rng = np.random.default_rng(3)
    rows, vocab, k = 12, 3001, 40
    step = 2.0 ** -7                                              # (a multiple of fp32's steps at 1e5: the differences are the same numbers)
    z = torch.from_numpy(np.round(rng.standard_normal((rows, vocab)) * 2 / step) * step + offset).float()
    index = torch.from_numpy(np.stack([np.sort(rng.permutation(vocab)[:k]) for _ in range(rows)])).long()
    value = torch.from_numpy(np.round(rng.standard_normal((rows, k)) * 2 / step) * step + offset).float()
    loss, dz = b.ds_distill(z.cuda(), pack_pairs(index, value).cuda(), 1.0)
    want_loss, want = plain.distill(z, index, value, 1.0)
    spread = (z.amax(dim=1) - z.amin(dim=1)).double() + (value.amax(dim=1) - value.amin(dim=1)).double()
    rel = U * (32 + 4 * spread)[:, None]
    tol = rel * (plain.log_softmax(z.double()).exp() + want.abs()) + plain.rounding(want, F32)
    bad = ~((dz.cpu().double() - want).abs() <= tol)
    assert not bad.any(), f"dz: {int(bad.sum())} off, by up to {((dz.cpu().double() - want).abs() / tol).max()} of the tolerance"
    tol = rel[:, 0] * (8 + 2 * spread + math.log(vocab))
    assert ((loss.cpu().double() - want_loss).abs() <= tol).all(), ((loss.cpu().double() - want_loss).abs() / tol).max()


@pytest.mark.parametrize("temperature", [0.5, 1.0, 4.0])
def test_teachers_whose_entries_are_masked(temperature):
    """Entries of any size of mask, beside usual ones and by themselves: alike ones share the probability."""
    rng = np.random.default_rng(5)
    vocab, k = 900, 130
    values = []
    for a, c in ((-1e10, 0.0), (-1e10, -1e10), (-1e30, -1e30), (LOWEST, LOWEST), (LOWEST, -1e38), (-1e38, LOWEST), (-2.3e38, -2.4e38), (2.4e38, 2.3e38), (-1e20, LOWEST)):
        v = np.where(np.arange(k) < 70, a, c + (rng.standard_normal(k) if c == 0 else 0.0))
        values += [v, rng.permutation(v)]
    value = torch.from_numpy(np.stack(values)).float()
    rows = value.shape[0]
    z = torch.from_numpy(rng.standard_normal((rows, vocab))).float()
    index = torch.from_numpy(np.stack([rng.permutation(vocab)[:k] for _ in range(rows)])).long()
    loss, dz = b.ds_distill(z.cuda(), pack_pairs(index, value).cuda(), temperature)
    want_loss, want = plain.distill(z, index, value, temperature)
    rel = U * (64 + 4 * 100)
    tol = rel * (plain.log_softmax(z.double() / temperature).exp() / temperature + want.abs()) + 2.0 ** -126 / temperature + plain.rounding(want, F32)
    assert ((dz.cpu().double() - want).abs() <= tol).all()
    assert ((loss.cpu().double() - want_loss).abs() <= rel * (16 + math.log(vocab))).all()       # (every -ln p and -ln q of a probable entry is below 16)


def test_temperatures_that_have_no_reciprocal_are_refused():
    z, pairs = torch.zeros((2, 50), device="cuda"), torch.zeros((2, 3, 2), dtype=torch.int32, device="cuda")
    for call in (lambda: b.ds_top_logits(z, 3, 1e-39), lambda: b.ds_distill(z, pairs, 1e-39)):
        with pytest.raises(b.DsqError, match="temperature"):
            call()
