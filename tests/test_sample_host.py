"""What ds_sample refuses: host code alone, no kernel is launched."""
import ctypes

import pytest
import torch

from paper_1907_07346_amd import binding as b

BIG = 1 << 40                                       # an address that is never touched
NAN, INF = float("nan"), float("inf")


def sampling(**kw):
    args = dict(rows=10, vocab=1000, dtype=1, top_k=0, temperature=1.0, top_p=1.0, min_p=0.0, reserved=0)
    args.update(kw)
    return b.ds_sampling(**args)


def sample(s, each=None, z=BIG, z_ld=None, u=2 * BIG, token=3 * BIG, logp=4 * BIG, work=5 * BIG, size=1 << 40):
    buf = ctypes.create_string_buffer(256)
    rows = b.ds_sampling_rows(**each) if each is not None else None
    st = b.lib().ds_sample(ctypes.byref(s) if s else None, ctypes.byref(rows) if rows else None, z, s.vocab if z_ld is None and s else z_ld or 0, u, token, logp,
                           work, size, None, buf, 256)
    return st, buf.value.decode()


@pytest.mark.parametrize("kw,call,needle", [
    (None, {}, "NULL"), (dict(rows=1 << 31), {}, "rows"), (dict(vocab=0), {}, "vocab"), (dict(vocab=1 << 31), {}, "vocab"), (dict(dtype=3), {}, "dtype"),
    (dict(dtype=-1), {}, "dtype"), (dict(top_k=-1), {}, "top_k"), (dict(temperature=-1.0), {}, "temperature"), (dict(temperature=NAN), {}, "temperature"),
    (dict(temperature=INF), {}, "temperature"), (dict(temperature=1e-40), {}, "temperature"), (dict(top_p=-0.1), {}, "top_p"), (dict(top_p=1.1), {}, "top_p"),
    (dict(top_p=NAN), {}, "top_p"), (dict(min_p=-0.1), {}, "min_p"), (dict(min_p=1.1), {}, "min_p"), (dict(min_p=NAN), {}, "min_p"),
    (dict(reserved=1), {}, "reserved"), ({}, dict(z=None), "NULL"), ({}, dict(u=None), "NULL"), ({}, dict(token=None), "NULL"), ({}, dict(z=BIG + 1), "aligned"),
    ({}, dict(z_ld=999), "z_ld"), ({}, dict(z_ld=1 << 63), "address space"), ({}, dict(u=2 * BIG + 2), "4-byte"), ({}, dict(token=3 * BIG + 1), "4-byte"),
    ({}, dict(logp=4 * BIG + 2), "4-byte"), ({}, dict(each=dict(top_k_dev=BIG + 2)), "4-byte"), ({}, dict(token=BIG + 8), "overlaps z"),
    ({}, dict(logp=BIG + 8), "overlaps z"), ({}, dict(token=2 * BIG + 36), "another"), ({}, dict(logp=3 * BIG + 36), "another"),
    ({}, dict(each=dict(top_p_dev=3 * BIG - 36)), "another"), ({}, dict(each=dict(min_p_dev=4 * BIG)), "another"),
])
def test_sample_refuses(kw, call, needle):
    st, why = sample(sampling(**kw) if kw is not None else None, **call)
    assert st == b.DS_EINVAL and needle in why, why


def test_no_rows_do_nothing():
    assert sample(sampling(rows=0), z=None, u=None, token=None) == (b.DS_OK, "")
    assert b.lib().ds_sample_work_bytes(ctypes.byref(sampling(rows=0))) == 0
    assert b.lib().ds_sample_work_bytes(ctypes.byref(sampling(vocab=0))) == 0


def test_the_binding_refuses(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    z, u = torch.zeros((3, 10)), torch.zeros(3)
    for call, needle in ((lambda: b.ds_sample(z.double(), u), "matrix"), (lambda: b.ds_sample(z[0], u), "matrix"), (lambda: b.ds_sample(z.t(), u), "stride"),
                         (lambda: b.ds_sample(z, u.double()), "u must"), (lambda: b.ds_sample(z, u[:2]), "u must"), (lambda: b.ds_sample(z, u), "z must be on")):
        with pytest.raises(b.DsqError, match=needle) as e:
            call()
        assert e.value.status == b.DS_EINVAL
    monkeypatch.setattr(b, "_on_device", lambda *a: 0)
    for kw, needle in ((dict(top_k=1.5), "whole"), (dict(top_k=-1), "whole"), (dict(top_k=1 << 31), "whole"), (dict(temperature=torch.ones(2)), "temperature"),
                       (dict(top_k=torch.ones(3)), "top_k"), (dict(top_p=torch.ones(3).double()), "top_p"), (dict(min_p=torch.ones((3, 1))), "min_p"),
                       (dict(min_p=torch.ones(6)[::2]), "min_p")):
        with pytest.raises(b.DsqError, match=needle):
            b.ds_sample(z, u, **kw)
