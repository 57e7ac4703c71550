"""Tokens drawn from logits against a sorted list in 64 bits.

Tokens have to be equal: masses are off by 4e-14 of themselves and half a unit of 2^-bits each (2^-bits: 2^62 over the power of two that reaches vocab, 2^-51 at most), so that a
token could differ where u S comes as near as 1e-12 or so to a border, in one of 1e8 rows.  logp is off by its rounding to fp32 and by what S is off: `unit` below."""
import math

import numpy as np
import pytest
import torch

from paper_1907_07346_amd import binding as b
from paper_1907_07346_amd import workloads as wl
from tests import answers_plain as plain

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
INF, NAN = float("inf"), float("nan")
LOWEST = {t: torch.finfo(t).min for t in (F32, BF16, F16)}


def normal(rows, vocab, dtype, seed, scale=3.0, shift=0.0):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal((rows, vocab)) * scale + shift).to(dtype)


def uniform(rows, seed):
    return torch.from_numpy(np.random.default_rng(seed + 10 ** 6).random(rows, np.float32))


def unit(vocab):
    return vocab * 2.0 ** (-1 - min(51, 62 - math.ceil(math.log2(vocab)))) + 1e-13


def same(got, want, vocab, what=""):
    token, logp = got[0].cpu(), got[1].cpu().double()
    bad = (token != want[0]).nonzero()[:, 0]
    assert not len(bad), f"{what}: {len(bad)} of {len(token)} tokens differ, first in row {bad[0]}: {token[bad[0]]} for {want[0][bad[0]]}"
    tol = plain.rounding(want[1], F32) + unit(vocab)
    off = ~((logp == want[1]) | (torch.isnan(logp) & torch.isnan(want[1])) | ((logp - want[1]).abs() <= tol))
    assert not off.any(), f"{what}: logp {logp[off][0]} for {want[1][off][0]}"


def check(z, u, what="", **parameters):
    own = {k: v.cuda() if torch.is_tensor(v) else v for k, v in parameters.items()}
    same(b.ds_sample(z.cuda(), u.cuda(), **own), plain.sample(z, u, **parameters), z.shape[1], f"{what} {parameters if not own or all(not torch.is_tensor(v) for v in own.values()) else ''}")


FILTERS = [dict(), dict(temperature=0.7), dict(top_k=1), dict(top_k=50), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=40, top_p=0.95, temperature=0.8),
           dict(top_k=600, top_p=0.99), dict(top_p=0.5, min_p=0.02, temperature=1.3), dict(top_k=100, top_p=0.8, min_p=0.01), dict(temperature=0.0)]
SIZES = [(1, 1), (3, 2), (5, 7), (4, 16), (7, 255), (3, 511), (3, 512), (3, 513), (2, 1000), (9, 2049), (2, 8191), (4, 16384), (2, 16385), (3, 32003), (2, 50001), (1, 131072)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_tokens_of_random_rows(rows, vocab, dtype):
    z, u = normal(rows, vocab, dtype, seed=rows * 100003 + vocab), uniform(rows, vocab)
    for f in FILTERS:
        check(z, u, **f)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("shift,scale", [(-30.0, 3.0), (30.0, 3.0), (0.0, 0.05), (-8.0, 0.01), (1000.0, 0.5), (0.0, 100.0), (0.0, 1e-6), (-500.0, 100.0)])
def test_logits_that_lie_close_or_far(shift, scale, dtype):
    z, u = normal(4, 20001, dtype, seed=7, scale=scale, shift=shift), uniform(4, 3)
    for f in (dict(), dict(top_p=0.9), dict(top_k=50, top_p=0.7), dict(top_k=5000), dict(min_p=0.3), dict(temperature=0.01), dict(temperature=50.0, top_p=0.6)):
        check(z, u, **f)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("vocab", [10, 1000, 40000])
def test_rows_of_equal_logits(vocab, dtype):
    for value in (0.0, -0.0, 5.0, -7.25, LOWEST[dtype], 1e-3):
        z = torch.full((6, vocab), value, dtype=dtype)
        u = torch.tensor([0.0, 0.25, 0.5, 0.75, 0.999, 1.0])
        for f in (dict(), dict(top_k=max(1, vocab // 4)), dict(top_p=0.5), dict(min_p=1.0), dict(top_k=vocab // 2, top_p=0.25), dict(temperature=0.0)):
            check(z, u, **f)
    z = torch.zeros((2, vocab), dtype=dtype)
    z[0, ::2] = -0.0                                                              # equal to +0
    check(z, torch.tensor([0.3, 0.9]))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_many_ties_on_several_levels(dtype):
    rng = np.random.default_rng(3)
    z = torch.from_numpy(rng.integers(0, 4, (8, 30000)).astype(np.float32) * 0.75 - 1.0).to(dtype)
    for f in FILTERS:
        check(z, uniform(8, 5), **f)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("vocab", [100, 5000, 33333])
def test_masks(vocab, dtype):
    rng = np.random.default_rng(vocab)
    z = normal(10, vocab, dtype, seed=11)
    for row, mask in enumerate((-INF, LOWEST[dtype], LOWEST[dtype] / 2, -1e4, -INF, LOWEST[dtype], -INF, -60000.0, -INF, -INF)):
        z[row, torch.from_numpy(rng.random(vocab) < (0.5, 0.99)[row % 2])] = mask
    z[4] = -INF
    z[4, vocab // 2] = 1.0                                                        # one is left
    z[6, :] = -INF                                                                # none is
    z[8] = -INF
    z[8, -1] = LOWEST[dtype]
    for f in FILTERS:
        check(z, uniform(10, 1), **f)
    token, logp = b.ds_sample(z.cuda(), uniform(10, 1).cuda())
    assert token[6] == -1 and logp[6] == -INF and token[8] == vocab - 1 and logp[8] == 0


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("vocab", [100, 5000, 33333])
def test_infinities_and_nan(vocab, dtype):
    z = normal(6, vocab, dtype, seed=12)
    z[0, 17] = NAN
    z[1, vocab - 1] = INF
    z[2, 5] = z[2, 50] = z[2, vocab - 3] = INF
    z[3, 3], z[3, 4] = INF, -INF
    z[4, 60], z[4, 70] = NAN, INF
    for f in FILTERS + [dict(temperature=0.0, min_p=0.5), dict(min_p=1.0)]:
        check(z, uniform(6, 2), **f)
    z[2] = INF                                                                    # all of them
    for f in (dict(), dict(top_k=10), dict(top_p=0.25), dict(min_p=0.5)):
        check(z, uniform(6, 2), **f)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("vocab", [30, 2000, 20000])
def test_random_numbers_at_the_ends(vocab, dtype):
    u = torch.tensor([0.0, -0.0, 1e-45, 1e-30, 2.0 ** -24, 1 - 2.0 ** -24, 1.0, 2.0, -1.0, INF, -INF, NAN])
    z = normal(len(u), vocab, dtype, seed=13, scale=1.0)
    for f in FILTERS:
        check(z, u, **f)


@pytest.mark.parametrize("temperature", [2.0 ** -126, 1e-20, 1e-3, 1e3, 1e20, 3e38])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_temperatures_far_from_one(temperature, dtype):
    for z in (normal(3, 3000, dtype, seed=14), normal(3, 3000, dtype, seed=15, scale=torch.finfo(dtype).max / 8), normal(3, 3000, dtype, seed=16, scale=1e-6)):
        for f in (dict(), dict(top_p=0.6), dict(top_k=700, min_p=0.1)):
            check(z, uniform(3, 9), temperature=temperature, **f)


def test_numbers_below_the_normal_ones():
    for dtype, small in ((F32, 2.0 ** -149), (BF16, 2.0 ** -133), (F16, 2.0 ** -24)):
        z = (torch.from_numpy(np.random.default_rng(4).integers(-50, 50, (4, 9000))).double() * small).to(dtype)
        for t in (1.0, max(small * 10, 2.0 ** -126)):
            for f in (dict(), dict(top_p=0.3), dict(top_k=900)):
                check(z, uniform(4, 6), temperature=t, **f)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_shares_at_the_ends(dtype):
    z = normal(3, 5000, dtype, seed=17)
    for f in (dict(top_p=0.0), dict(top_p=1e-30), dict(top_p=1 - 2.0 ** -24), dict(min_p=1.0), dict(min_p=1e-38), dict(min_p=1e-12), dict(top_k=4999),
              dict(top_k=5000), dict(top_k=2 ** 31 - 1)):
        check(z, uniform(3, 8), **f)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("vocab", [77, 3001, 20000])
def test_parameters_of_rows(vocab, dtype):
    temperature = torch.tensor([1.0, 0.5, 0.0, -1.0, NAN, INF, 1e-40, 2.0, 1.0, 1.0, 1.0, 1.0])
    top_k = torch.tensor([0, 5, 9, 9, 0, 0, 0, -3, 10 ** 9, 1, 600, 0], dtype=torch.int32)
    top_p = torch.tensor([1.0, 0.9, 0.5, 0.5, 0.5, 0.5, 0.5, 2.0, NAN, 0.7, 0.95, -1.0])
    min_p = torch.tensor([0.0, 0.1, 0.0, 0.0, 0.0, 0.0, 0.0, -1.0, NAN, 0.0, 2.0, 0.0])
    z, u = normal(12, vocab, dtype, seed=18), uniform(12, 8)
    all_of = dict(temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)
    check(z, u, **all_of)
    for name in all_of:
        check(z, u, **{**dict(temperature=0.8, top_k=30, top_p=0.9, min_p=0.01), name: all_of[name]})


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_rows_with_a_pitch_and_odd_addresses(dtype):
    for rows, vocab, pitch, first in ((5, 100, 107, 1), (4, 5001, 5003, 3), (3, 20001, 20011, 5)):
        base = torch.full((rows * pitch + first + 8,), NAN, dtype=dtype)
        z = base[first:first + rows * pitch].view(rows, pitch)[:, :vocab]
        z.copy_(normal(rows, vocab, dtype, seed=19))
        u = uniform(rows, 4)
        own = base.cuda()[first:first + rows * pitch].view(rows, pitch)[:, :vocab]
        for f in FILTERS:
            same(b.ds_sample(own, u.cuda(), **f), plain.sample(z, u, **f), vocab)


def test_rows_beyond_four_gigabytes():
    pitch = 2 ** 31 + 11
    base = torch.empty(2 * pitch + 1000, dtype=BF16, device="cuda")
    z = normal(3, 1000, BF16, seed=20)
    own = base.as_strided((3, 1000), (pitch, 1))
    own.copy_(z)
    for f in (dict(), dict(top_k=20, top_p=0.9)):
        same(b.ds_sample(own, uniform(3, 1).cuda(), **f), plain.sample(z, uniform(3, 1), **f), 1000)


def test_a_long_row():
    vocab = (1 << 24) + 5
    z = torch.randn((1, vocab), device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    for dtype in (F32, BF16):
        zt = z.to(dtype)
        for f in (dict(), dict(top_p=0.9), dict(top_k=1000), dict(min_p=0.5)):
            same(b.ds_sample(zt, uniform(1, 2).cuda(), **f), plain.sample(zt, uniform(1, 2), **f), vocab)


def test_many_rows():
    z, u = normal(5000, 40, BF16, seed=21), uniform(5000, 3)
    check(z, u, top_p=0.9)
    z, u = normal(1500, 3000, F32, seed=22), uniform(1500, 3)
    check(z, u, top_k=20)


def test_no_rows_and_results_without_logp():
    token, logp = b.ds_sample(torch.empty((0, 100), device="cuda"), torch.empty(0, device="cuda"))
    assert token.shape == (0,) and logp.shape == (0,) and token.dtype == torch.int32
    import ctypes
    z, u = normal(3, 1000, F32, seed=23).cuda(), uniform(3, 3).cuda()
    token = torch.full((5,), 77, dtype=torch.int32, device="cuda")
    shape = b.ds_sampling(3, 1000, 0, 0, 1.0, 1.0, 0.0, 0)
    size = b.lib().ds_sample_work_bytes(ctypes.byref(shape))
    work = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
    assert b.lib().ds_sample(ctypes.byref(shape), None, z.data_ptr(), 1000, u.data_ptr(), token.data_ptr(), None, work.data_ptr(), size,
                             torch.cuda.current_stream().cuda_stream, None, 0) == b.DS_OK
    assert torch.equal(token[:3], b.ds_sample(z, u)[0]) and (token[3:] == 77).all()


def test_rows_with_a_top_k_that_the_shape_does_not_tell_of():
    """top_k_dev beside top_k = 0 in C: right all the same."""
    import ctypes
    for dtype, vocab in ((F32, 40000), (F16, 70000), (BF16, 5000)):
        z, u, k = normal(4, vocab, dtype, seed=27), uniform(4, 7), torch.tensor([0, 3, 700, 50], dtype=torch.int32)
        own, uc, kc = z.cuda(), u.cuda(), k.cuda()
        shape = b.ds_sampling(4, vocab, {F32: 0, BF16: 1, F16: 2}[dtype], 0, 1.0, 0.9, 0.0, 0)
        each = b.ds_sampling_rows(None, kc.data_ptr(), None, None)
        size = b.lib().ds_sample_work_bytes(ctypes.byref(shape))
        work = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
        token, logp = torch.empty(4, dtype=torch.int32, device="cuda"), torch.empty(4, device="cuda")
        assert b.lib().ds_sample(ctypes.byref(shape), ctypes.byref(each), own.data_ptr(), vocab, uc.data_ptr(), token.data_ptr(), logp.data_ptr(), work.data_ptr(),
                                 size, torch.cuda.current_stream().cuda_stream, None, 0) == b.DS_OK
        same((token, logp), plain.sample(z, u, top_k=k, top_p=0.9), vocab)


MANY = [(513, 8193, F32), (600, 32003, F32), (513, 32767, F16), (700, 16385, BF16), (1025, 24001, F32), (1030, 49152, F16), (1100, 40001, BF16), (2049, 65535, BF16), (4097, 70001, BF16)]


@pytest.mark.parametrize("rows,vocab,dtype", MANY)
def test_many_rows_are_as_few_are(rows, vocab, dtype):
    """How rows are divided goes by their number: the same answers, bit for bit, as of a few at a time, and the formula's for some."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    z = (torch.randn((rows, vocab), generator=g, device="cuda") * 3).to(dtype)
    u = torch.rand(rows, generator=g, device="cuda")
    z[3], z[5, 7], z[6, 9], z[8] = -INF, NAN, INF, 1.5
    z[9, ::2] = torch.finfo(dtype).min
    z[10] = torch.round(z[10])
    z[11] *= 1e-6
    some = torch.tensor([*range(14), rows // 2, rows - 1])
    for f in (dict(), dict(top_p=0.9), dict(top_k=50, top_p=0.95), dict(top_k=5000), dict(min_p=0.05), dict(top_p=0.97, min_p=0.001, temperature=1.7)):
        token, logp = b.ds_sample(z, u, **f)
        for i in range(0, rows, 500):
            few_token, few_logp = b.ds_sample(z[i:i + 500], u[i:i + 500], **f)
            assert torch.equal(few_token, token[i:i + 500]) and torch.equal(few_logp.view(torch.int32), logp[i:i + 500].view(torch.int32))
        same((token[some.cuda()], logp[some.cuda()]), plain.sample(z.cpu()[some], u.cpu()[some], **f), vocab)


SPLIT = [(1, 131072, F32), (3, 65536, F16), (32, 33001, F32), (2, 600001, BF16)]


@pytest.mark.parametrize("rows,vocab,dtype", SPLIT)
def test_rows_that_are_split(rows, vocab, dtype):
    z, u = normal(rows, vocab, dtype, seed=28), uniform(rows, 9)
    for f in (dict(), dict(top_p=0.9), dict(top_p=0.999, min_p=1e-4), dict(temperature=0.3, top_p=0.5), dict(temperature=40.0), dict(min_p=0.9, top_p=0.99)):
        check(z, u, **f)
    z[0] = -INF
    if rows > 1:
        z[1, vocab // 3] = NAN
    if rows > 2:
        z[2, 5] = z[2, vocab - 1] = INF
    check(z, u, top_p=0.9)
    check(torch.full_like(z, 0.5), u, top_p=0.7)                                  # more ties than lists have room for
    check(torch.round(normal(rows, vocab, dtype, seed=29)), u, top_p=0.8)


@pytest.mark.parametrize("rows,vocab", [(3, 300), (2, 40000), (1, 131072)])
def test_a_captured_call_draws_from_what_it_finds(rows, vocab):
    z, u = torch.zeros((rows, vocab), dtype=BF16, device="cuda"), torch.zeros(rows, device="cuda")
    p = torch.ones(rows, device="cuda")
    b.ds_sample(z, u, top_p=p)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = b.ds_sample(z, u, top_p=p)
    for t in range(5):
        z.copy_(normal(rows, vocab, BF16, seed=t))
        u.copy_(uniform(rows, t))
        p.fill_(1.0 - 0.1 * t)
        graph.replay()
        torch.cuda.synchronize()
        same(got, plain.sample(z, u.cpu(), top_p=p.cpu()), vocab)
        eager = b.ds_sample(z, u, top_p=p)
        assert torch.equal(eager[0], got[0]) and torch.equal(eager[1], got[1])


def test_calls_on_another_stream_and_memory_freed_meanwhile():
    s = torch.cuda.Stream()
    want = plain.sample(normal(64, 20000, F32, seed=24), uniform(64, 5), top_p=0.9)
    host, uh = normal(64, 20000, F32, seed=24), uniform(64, 5)
    for _ in range(5):
        z, u, p = host.cuda(), uh.cuda(), torch.full((64,), 0.9, device="cuda")
        s.wait_stream(torch.cuda.current_stream())
        got = b.ds_sample(z, u, top_p=p, stream=s)
        del z, u, p
        torch.full((64, 20000), 9.0, device="cuda"), torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda")
        s.synchronize()
        same(got, want, 20000)


def test_a_neighbours_samples_are_learnt_from():
    """messages -> logits -> tokens -> loss and gradient -> clipped rows -> the next step, each against its plain form."""
    V, D, n, tokens = 1000, 128, 3, 5
    cfg, keep = b.make_config(n=n, N=V * D, topo=wl.TOPO_RING, kind=wl.KIND_QUANT_MAXABS, gamma=0.5, eta=0.3, bits=4, block=64, seed=0)
    ds = b.DeepSqueeze(cfg, keep)
    rng = np.random.default_rng(25)
    ds.ds_write_state(rng.standard_normal((n, V * D)).astype(np.float32) * 0.3, None, 0)
    ld = ds.ds_state_ptrs()[2]
    g = torch.zeros((n, ld), device="cuda")
    ds.ds_step(g)
    features = normal(tokens, D, F32, seed=26, scale=1.0).cuda()
    for t in range(2):
        x, _ = ds.ds_read_state(want_delta=False)
        grads = []
        for w in range(n):
            z = ds.ds_product((w + 1) % n, features, rows=V)
            u = uniform(tokens, 10 * t + w)
            token, logp = b.ds_sample(z, u.cuda(), temperature=0.8, top_k=40, top_p=0.9)
            same((token, logp), plain.sample(z, u, temperature=0.8, top_k=40, top_p=0.9), V)
            pairs = torch.stack([token, torch.zeros_like(token)], dim=1)[:, None, :].contiguous()            # one entry, of probability 1
            own = torch.from_numpy(x[w].reshape(V, D)).cuda()
            logits = features @ own.t()
            loss, dz = b.ds_distill(logits, pairs)
            want_loss, want_dz = plain.distill(logits.cpu(), token.cpu().long()[:, None], torch.zeros((tokens, 1)), 1.0)
            assert (loss.cpu().double() - want_loss).abs().max() <= 1e-5 * (1 + want_loss.abs().max())
            assert (dz.cpu().double() - want_dz).abs().max() <= 1e-5
            grads.append([dz.t() @ features])
        norm = b.ds_clip(grads, 5.0, out=g)
        for w in range(n):
            want = grads[w][0].double().reshape(-1)
            factor = min(1.0, 5.0 / float(want.norm()))
            assert abs(float(norm[w]) - float(want.norm())) <= 2.0 ** -23 * float(norm[w])
            assert (g[w, :V * D].double() - want * factor).abs().max() <= 2.0 ** -23 * (want * factor).abs().max()
        assert (norm > 5.0).any()
        ds.ds_step(g)
    assert ds.ds_step_count() == 3
    ds.ds_destroy()
