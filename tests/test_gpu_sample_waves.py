"""Short rows of ds_sample by the numbers of rows that choose between a wave and a workgroup for a row, and their logits' extremes.  Tolerances as in test_gpu_sample.py."""
import numpy as np
import pytest
import torch

from paper_1907_07346_amd import binding as b
from tests import answers_plain as plain
from tests.test_gpu_sample import BF16, F16, F32, FILTERS, INF, LOWEST, NAN, check, normal, same, uniform

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, F16])
@pytest.mark.parametrize("rows,vocab", [(2048, 513), (2049, 1000), (2100, 2047), (2101, 2048)])
def test_many_rows_of_up_to_2048_logits(rows, vocab, dtype):
    """From 2048 rows on without a top_k a wave takes a row, below a workgroup: the same answers, bit for bit, and the formula's for some."""
    z, u = normal(rows, vocab, dtype, seed=vocab), uniform(rows, vocab)
    rng = np.random.default_rng(vocab)
    for row, mask in enumerate((-INF, LOWEST[dtype], LOWEST[dtype] / 2, -1e4)):
        z[row, torch.from_numpy(rng.random(vocab) < (0.5, 0.99)[row % 2])] = mask
    z[4], z[5, 7], z[6, vocab - 1], z[8] = -INF, NAN, INF, 1.5
    z[9, 5] = z[9, 50] = z[9, vocab - 3] = INF
    z[10], z[11], z[12], z[13] = torch.round(z[10]), z[11] * 1e-6, z[12] * 1000.0, INF
    z[14], z[15], z[16] = LOWEST[dtype], torch.round(z[15] * 0.3) * 1e-3, 0.0
    z[16, ::2] = -0.0
    z[17, :] = -INF
    z[17, vocab // 2] = LOWEST[dtype]
    z[18] = normal(1, vocab, dtype, seed=1, scale=torch.finfo(dtype).max / 8)[0]
    own, uc = z.cuda(), u.cuda()
    some = torch.tensor([*range(24), rows // 2, rows - 1])
    for f in (dict(), dict(top_p=0.9), dict(min_p=0.05), dict(top_p=0.97, min_p=0.001, temperature=1.7), dict(temperature=50.0), dict(temperature=1e-3, top_p=0.5),
              dict(top_p=0.0), dict(min_p=1.0), dict(temperature=0.0)):
        token, logp = b.ds_sample(own, uc, **f)
        for i in range(0, rows, 700):
            few_token, few_logp = b.ds_sample(own[i:i + 700], uc[i:i + 700], **f)
            assert torch.equal(few_token, token[i:i + 700]) and torch.equal(few_logp.view(torch.int32), logp[i:i + 700].view(torch.int32))
        same((token[some.cuda()], logp[some.cuda()]), plain.sample(z[some], u[some], **f), vocab)
    # rows of their own parameters, some with a top_k after all
    each = dict(temperature=torch.linspace(0.0, 3.0, rows), top_p=torch.linspace(1.1, 0.0, rows), min_p=torch.linspace(0.0, 0.2, rows))
    token, logp = b.ds_sample(own, uc, **{k: v.cuda() for k, v in each.items()})
    same((token[some.cuda()], logp[some.cuda()]), plain.sample(z[some], u[some], **{k: v[some] for k, v in each.items()}), vocab)


def test_many_short_rows_with_a_top_k_that_the_shape_does_not_tell_of():
    """top_k_dev beside top_k = 0 in C, where waves take the rows."""
    import ctypes
    rows, vocab = 2050, 900
    z, u = normal(rows, vocab, F32, seed=2), uniform(rows, 2)
    k = (torch.arange(rows, dtype=torch.int32) * 7) % 1000
    own, uc, kc = z.cuda(), u.cuda(), k.cuda()
    shape, each = b.ds_sampling(rows, vocab, 0, 0, 1.0, 0.9, 0.0, 0), b.ds_sampling_rows(None, kc.data_ptr(), None, None)
    assert b.lib().ds_sample_work_bytes(ctypes.byref(shape)) == 0
    token, logp = torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, device="cuda")
    assert b.lib().ds_sample(ctypes.byref(shape), ctypes.byref(each), own.data_ptr(), vocab, uc.data_ptr(), token.data_ptr(), logp.data_ptr(), None, 0,
                             torch.cuda.current_stream().cuda_stream, None, 0) == b.DS_OK
    same((token, logp), plain.sample(z, u, top_k=k, top_p=0.9), vocab)


SHORT = [70, 500, 512]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("vocab", SHORT)
@pytest.mark.parametrize("shift,scale", [(-30.0, 3.0), (0.0, 0.05), (-8.0, 0.01), (1000.0, 0.5), (0.0, 100.0), (0.0, 1e-6), (-500.0, 100.0)])
def test_short_rows_that_lie_close_or_far(shift, scale, vocab, dtype):
    z, u = normal(4, vocab, dtype, seed=7, scale=scale, shift=shift), uniform(4, 3)
    for f in FILTERS + [dict(top_k=60, top_p=0.7), dict(temperature=0.01), dict(temperature=50.0, top_p=0.6)]:
        check(z, u, **f)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("vocab", SHORT)
@pytest.mark.parametrize("temperature", [2.0 ** -126, 1e-20, 1e-3, 1e3, 1e20, 3e38])
def test_short_rows_at_temperatures_far_from_one(temperature, vocab, dtype):
    for z in (normal(3, vocab, dtype, seed=14), normal(3, vocab, dtype, seed=15, scale=torch.finfo(dtype).max / 8), normal(3, vocab, dtype, seed=16, scale=1e-6)):
        for f in (dict(), dict(top_p=0.6), dict(top_k=66, min_p=0.1)):
            check(z, uniform(3, 9), temperature=temperature, **f)


@pytest.mark.parametrize("vocab", SHORT)
def test_short_rows_of_numbers_below_the_normal_ones(vocab):
    for dtype, small in ((F32, 2.0 ** -149), (BF16, 2.0 ** -133), (F16, 2.0 ** -24)):
        z = (torch.from_numpy(np.random.default_rng(4).integers(-50, 50, (4, vocab))).double() * small).to(dtype)
        for t in (1.0, max(small * 10, 2.0 ** -126)):
            for f in (dict(), dict(top_p=0.3), dict(top_k=67)):
                check(z, uniform(4, 6), temperature=t, **f)


@pytest.mark.parametrize("rows,vocab,dtype", [(1, 131072, F32), (12, 70000, F16), (32, 33001, F32), (3, 600001, BF16)])
def test_rows_that_are_split_with_parameters_of_their_own(rows, vocab, dtype):
    rng = np.random.default_rng(rows)

    def of(lo, hi):
        return torch.from_numpy(rng.uniform(lo, hi, rows).astype(np.float32))

    z, u = normal(rows, vocab, dtype, seed=30), uniform(rows, 4)
    temperature, top_p, min_p = of(0.3, 2.0), of(0.2, 1.1), of(0.0, 0.1)
    if rows > 2:
        temperature[1], top_p[2], min_p[2] = 0.0, NAN, NAN
    if rows > 8:
        temperature[3], temperature[4], top_p[5], min_p[6], min_p[7] = NAN, INF, 0.0, 2.0, -1.0
    for f in (dict(temperature=temperature), dict(top_p=top_p), dict(min_p=min_p), dict(top_p=top_p, min_p=0.03), dict(top_p=0.9, min_p=min_p),
              dict(temperature=temperature, top_p=top_p, min_p=min_p)):
        check(z, u, **f)
