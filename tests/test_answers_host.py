"""What the operators on messages and logits refuse, and their sizes: host code alone, no kernel is launched."""
import ctypes

import pytest
import torch

from paper_1907_07346_amd import binding as b
from paper_1907_07346_amd import workloads as wl
from tests.answers_plain import row_bytes

BIG = 1 << 40                                       # an address that is never touched


def matrix(**kw):
    args = dict(rows=100, cols=1000, tokens=3, block=128, dtype=1)
    args.update(kw)
    return b.ds_matrix(**args)


def logits(**kw):
    args = dict(rows=10, vocab=1000, k=16, dtype=1, temperature=1.0, reserved=0)
    args.update(kw)
    return b.ds_logits(**args)


def product(name, m, msg=BIG, x=2 * BIG, x_ld=None, y=3 * BIG, y_ld=None, work=4 * BIG, size=1 << 62):
    buf = ctypes.create_string_buffer(256)
    wide = (m.cols, m.rows) if name == "ds_product" else (m.rows, m.cols)
    st = getattr(b.lib(), name)(ctypes.byref(m), msg, x, wide[0] if x_ld is None else x_ld, y, wide[1] if y_ld is None else y_ld, work, size,
                                None, buf, 256)
    return st, buf.value.decode()


@pytest.mark.parametrize("name", ["ds_product", "ds_product_gradient"])
@pytest.mark.parametrize("kw,call,needle", [
    (dict(rows=0), {}, "rows"), (dict(rows=1 << 31), {}, "rows"), (dict(cols=0), {}, "cols"), (dict(cols=1 << 31), {}, "cols"),
    (dict(tokens=1 << 31), {}, "tokens"), (dict(block=32), {}, "block"), (dict(block=96), {}, "block"), (dict(block=4096), {}, "block"),
    (dict(block=0), {}, "block"), (dict(block=-64), {}, "block"), (dict(dtype=3), {}, "dtype"), (dict(dtype=-1), {}, "dtype"),
    ({}, dict(msg=None), "NULL"), ({}, dict(x=None), "NULL"), ({}, dict(y=None), "NULL"), ({}, dict(msg=BIG + 2), "4-byte"),
    ({}, dict(x=2 * BIG + 1), "aligned"), (dict(dtype=0), dict(y=3 * BIG + 2), "aligned"), ({}, dict(x_ld=99), "pitch"),
    ({}, dict(y_ld=99), "pitch"), ({}, dict(y=2 * BIG), "overlaps"), ({}, dict(y=BIG + 4), "overlaps"),
    ({}, dict(x_ld=1 << 63), "address space"), ({}, dict(y_ld=1 << 63), "address space"),
])
def test_products_refuse(name, kw, call, needle):
    st, msg = product(name, matrix(**kw), **call)
    assert st == b.DS_EINVAL and needle in msg, msg


def test_no_tokens_and_no_rows_do_nothing():
    assert product("ds_product", matrix(tokens=0), msg=None, x=None, y=None) == (b.DS_OK, "")
    assert product("ds_product_gradient", matrix(tokens=0), msg=None, x=None, y=None) == (b.DS_OK, "")
    L = b.lib()
    assert L.ds_top_logits(ctypes.byref(logits(rows=0)), None, 0, None, None, None, 0, None, None, 0) == b.DS_OK
    assert L.ds_distill(ctypes.byref(logits(rows=0)), None, 0, None, None, None, None, None, 0, None, 0, None, None, 0) == b.DS_OK
    for shape, name in ((matrix(tokens=0), "ds_product"), (matrix(tokens=0), "ds_product_gradient"), (logits(rows=0), "ds_top_logits"),
                        (logits(rows=0), "ds_distill")):
        assert getattr(L, name + "_work_bytes")(ctypes.byref(shape)) == 0


def top(l, z=BIG, z_ld=None, pairs=2 * BIG, lse=3 * BIG, work=4 * BIG, size=1 << 62):
    buf = ctypes.create_string_buffer(256)
    st = b.lib().ds_top_logits(ctypes.byref(l), z, l.vocab if z_ld is None else z_ld, pairs, lse, work, size, None, buf, 256)
    return st, buf.value.decode()


def distill(l, z=BIG, z_ld=None, pairs=2 * BIG, lse=None, weight=None, loss=3 * BIG, dz=5 * BIG, dz_ld=None, work=4 * BIG, size=1 << 62):
    buf = ctypes.create_string_buffer(256)
    st = b.lib().ds_distill(ctypes.byref(l), z, l.vocab if z_ld is None else z_ld, pairs, lse, weight, loss, dz,
                            l.vocab if dz_ld is None else dz_ld, work, size, None, buf, 256)
    return st, buf.value.decode()


BAD_LOGITS = [
    (dict(rows=1 << 31), {}, "rows"), (dict(vocab=0), {}, "vocab"), (dict(vocab=1 << 31), {}, "vocab"), (dict(k=0), {}, "k must"),
    (dict(k=257), {}, "k must"), (dict(dtype=7), {}, "dtype"), (dict(temperature=0.0), {}, "temperature"),
    (dict(temperature=-1.0), {}, "temperature"), (dict(temperature=float("nan")), {}, "temperature"),
    (dict(temperature=float("inf")), {}, "temperature"), (dict(reserved=1), {}, "reserved"), ({}, dict(z=None), "NULL"),
    ({}, dict(pairs=None), "NULL"), ({}, dict(z=BIG + 1), "aligned"), ({}, dict(pairs=BIG + 4), "aligned"), ({}, dict(z_ld=999), "z_ld"),
    ({}, dict(z_ld=1 << 63), "address space")]


@pytest.mark.parametrize("kw,call,needle", BAD_LOGITS + [(dict(vocab=15), {}, "k must"), ({}, dict(lse=BIG + 2), "aligned")])
def test_top_logits_refuses(kw, call, needle):
    st, msg = top(logits(**kw), **call)
    assert st == b.DS_EINVAL and needle in msg, msg


@pytest.mark.parametrize("kw,call,needle", BAD_LOGITS + [
    ({}, dict(loss=None, dz=None), "neither"), ({}, dict(dz_ld=999), "dz_ld"), ({}, dict(dz=5 * BIG + 1), "aligned"),
    ({}, dict(dz=BIG + 2), "overlaps"), ({}, dict(dz=BIG, dz_ld=1001), "overlaps"), ({}, dict(weight=BIG + 2), "aligned"),
    ({}, dict(lse=BIG + 1), "aligned"), ({}, dict(loss=BIG + 3), "aligned"), ({}, dict(dz_ld=1 << 63), "address space")])
def test_distill_refuses(kw, call, needle):
    st, msg = distill(logits(**kw), **call)
    assert st == b.DS_EINVAL and needle in msg, msg


def test_too_little_scratch_is_refused():
    """Shapes of every size: where scratch is asked for, one byte less, none, and misaligned scratch are refused."""
    L, seen = b.lib(), 0
    shapes = [("ds_product", matrix(rows=r, cols=c, tokens=t, dtype=d)) for r in (16, 5000, 65536) for c in (64, 16384) for t in (1, 16, 64, 300)
              for d in (0, 1)]
    shapes += [("ds_product_gradient", m) for _, m in shapes]
    shapes += [(n, logits(rows=r, vocab=v, dtype=d)) for n in ("ds_top_logits", "ds_distill") for r in (1, 100, 5000)
               for v in (1000, 131072, 1 << 20) for d in (0, 1)]
    for name, shape in shapes:
        size = getattr(L, name + "_work_bytes")(ctypes.byref(shape))
        assert size < 1 << 34
        if not size:
            continue
        seen += 1
        call = {"ds_top_logits": top, "ds_distill": distill}.get(name, lambda s, **kw: product(name, s, **kw))
        for kw, needle in ((dict(size=size - 1), "needed"), (dict(work=None), "needed"), (dict(work=4 * BIG + 8), "16-byte")):
            st, msg = call(shape, **kw)
            assert st == b.DS_EINVAL and needle in msg, (name, msg)
    print("shapes with scratch:", seen)


def test_matrix_bytes_are_the_message_bytes():
    for rows, cols, block in ((1, 1, 64), (7, 63, 64), (5, 65, 64), (3, 1000, 256), (4, 2048, 2048), (4, 2049, 2048), (9, 7, 2048)):
        cfg, _ = b.make_config(max(rows, 3), cols, wl.TOPO_RING, wl.KIND_QUANT_MAXABS, 0.1, 0.5, bits=4, block=block)
        want = b.ds_message_bytes(cfg) // max(rows, 3) * rows
        assert b.ds_matrix_bytes(rows, cols, block) == want == rows * row_bytes(cols, block)
    assert b.ds_matrix_bytes(0, 1, 64) == 0 and b.ds_matrix_bytes(1, 1, 100) == 0
    assert b.lib().ds_matrix_bytes(None) == 0 and b.lib().ds_product_work_bytes(None) == 0 and b.lib().ds_distill_work_bytes(None) == 0


def test_refusals_without_a_message_buffer():
    assert b.lib().ds_product(None, BIG, BIG, 1, BIG, 1, None, 0, None, None, 0) == b.DS_EINVAL
    short = ctypes.create_string_buffer(8)
    assert b.lib().ds_product(None, BIG, BIG, 1, BIG, 1, None, 0, None, short, 8) == b.DS_EINVAL
    assert short.value == b"the mat"


@pytest.mark.parametrize("call,needle", [
    (lambda x, m: b.ds_product(m, x.to(torch.float64), 2, 64), "float32"), (lambda x, m: b.ds_product(m, x[0], 2, 64), "matrix"),
    (lambda x, m: b.ds_product(m, x.t(), 2, 64), "stride"), (lambda x, m: b.ds_product(m[:10], x, 2, 64), "uint8"),
    (lambda x, m: b.ds_product(m.view(torch.int8), x, 2, 64), "uint8"), (lambda x, m: b.ds_top_logits(x, 0), "k must"),
    (lambda x, m: b.ds_top_logits(x.to(torch.int32), 1), "float32"), (lambda x, m: b.ds_distill(x, m), "pairs")])
def test_the_binding_refuses(call, needle, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    x = torch.zeros((3, 64))
    with pytest.raises(b.DsqError) as e:
        call(x, torch.zeros(2 * 36, dtype=torch.uint8))
    if "must be on" not in str(e.value):               # (the device is looked at before some of them)
        assert needle in str(e.value)
    assert e.value.status == b.DS_EINVAL


def test_tensors_of_another_device_are_refused(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    x, m = torch.zeros((3, 64)), torch.zeros(2 * 36, dtype=torch.uint8)
    pairs = torch.zeros((3, 4, 2), dtype=torch.int32)
    for call in (lambda: b.ds_product(m, x, 2, 64), lambda: b.ds_product_gradient(m, torch.zeros((3, 2)), 64, 64),
                 lambda: b.ds_top_logits(x, 4), lambda: b.ds_distill(x, pairs)):
        with pytest.raises(b.DsqError, match="current CUDA device"):
            call()


def test_subnormal_temperatures_are_refused():
    """log2(e) over one of them is no fp32 number."""
    for call in (top, distill):
        st, msg = call(logits(temperature=1e-39))
        assert st == b.DS_EINVAL and "temperature" in msg, msg
        assert b.lib().ds_distill_work_bytes(ctypes.byref(logits(vocab=1 << 20, temperature=1e-39))) == 0
