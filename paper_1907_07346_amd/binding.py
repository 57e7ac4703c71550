"""Thin ctypes binding of libdsq (argument marshalling only).

Function names mirror include/dsq.h.  Every step of the path runs in the library's HIP kernels;
there is no Python or CPU fallback: if libdsq.so is missing or fails to load, importing a symbol
from here raises.  torch is imported first on purpose, so that the library binds to the same HIP
runtime as the tensors whose device pointers are passed in.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np
import torch  # noqa: F401  (must be loaded before libdsq.so: one HIP runtime per process)

from .detgen import GRAD_KINDS
from .workloads import (KIND_IDENTITY, KIND_QUANT_MAXABS, KIND_SIGN_MEANABS, KIND_TOPK, KIND_QUANT_L2NORM, KIND_RAND_SPARSE, KIND_GSPAR,  # noqa: F401
                        ALGO_DEEPSQUEEZE, TOPO_CSR, TOPO_RING, TOPO_TORUS2D, Config)

DS_OK, DS_EINVAL, DS_ENOMEM, DS_EHIP, DS_ESTATE = range(5)
_STATUS = {0: "DS_OK", 1: "DS_EINVAL", 2: "DS_ENOMEM", 3: "DS_EHIP", 4: "DS_ESTATE"}

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libdsq.so")

EXPORTS = ["ds_validate_config", "ds_build_topology", "ds_message_bytes", "ds_init", "ds_step",
           "ds_read_state", "ds_write_state", "ds_read_messages", "ds_state_ptrs", "ds_message_ptr",
           "ds_step_count", "ds_plan_name", "ds_last_error", "ds_destroy", "ds_bench_copy",
           "ds_topk_candidate_rows", "ds_set_mixing", "ds_diagnostics", "ds_set_rates", "ds_workload_gradient", "ds_bench_stream", "ds_build_id", "ds_step_static", "ds_init_ex",
           "ds_matrix_bytes", "ds_product", "ds_product_work_bytes", "ds_product_gradient", "ds_product_gradient_work_bytes",
           "ds_top_logits", "ds_top_logits_work_bytes", "ds_distill", "ds_distill_work_bytes",
           "ds_sample", "ds_sample_work_bytes", "ds_gradients_bytes", "ds_gradients_lay", "ds_gradient_norm", "ds_gradient_norm_work_bytes", "ds_clip", "ds_clip_work_bytes"]


# torch's current stream as the pointer the library takes.  torch.cuda.current_stream() makes a Stream object for it: 2.9 us of
# the 10 to 18 us that a small problem's step costs the caller; the raw pointer takes 0.3.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_pointer(stream: Optional["torch.cuda.Stream"]) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


class ds_comp(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("bits", ctypes.c_int32), ("block", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("k", ctypes.c_uint64)]


class ds_workload(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("kind", ctypes.c_int32), ("N", ctypes.c_uint64), ("scale", ctypes.c_float),
                ("reserved", ctypes.c_float), ("seed", ctypes.c_uint64)]


class ds_plan_request(ctypes.Structure):
    _fields_ = [("variant", ctypes.c_int32), ("tile_plan", ctypes.c_int32), ("pitch_skew", ctypes.c_int64),
                ("autotune", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class ds_config(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("topo", ctypes.c_int32), ("N", ctypes.c_uint64),
                ("torus_rows", ctypes.c_int32), ("torus_cols", ctypes.c_int32),
                ("W_rowptr", ctypes.c_void_p), ("W_col", ctypes.c_void_p), ("W_val", ctypes.c_void_p),
                ("comp", ds_comp), ("gamma", ctypes.c_float), ("eta", ctypes.c_float),
                ("seed", ctypes.c_uint64), ("algo", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class ds_matrix(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_uint64), ("cols", ctypes.c_uint64), ("tokens", ctypes.c_uint64), ("block", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


class ds_logits(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_uint64), ("vocab", ctypes.c_uint64), ("k", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("temperature", ctypes.c_float), ("reserved", ctypes.c_int32)]


class ds_sampling(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_uint64), ("vocab", ctypes.c_uint64), ("dtype", ctypes.c_int32), ("top_k", ctypes.c_int32),
                ("temperature", ctypes.c_float), ("top_p", ctypes.c_float), ("min_p", ctypes.c_float), ("reserved", ctypes.c_int32)]


class ds_sampling_rows(ctypes.Structure):
    _fields_ = [("temperature_dev", ctypes.c_void_p), ("top_k_dev", ctypes.c_void_p), ("top_p_dev", ctypes.c_void_p), ("min_p_dev", ctypes.c_void_p)]


class ds_tensor(ctypes.Structure):
    _fields_ = [("data_dev", ctypes.c_void_p), ("count", ctypes.c_uint64), ("dtype", ctypes.c_int32), ("worker", ctypes.c_int32)]


class ds_gradients(ctypes.Structure):
    _fields_ = [("table_dev", ctypes.c_void_p), ("table_bytes", ctypes.c_uint64), ("workers", ctypes.c_uint64), ("tensors", ctypes.c_uint64),
                ("tiles", ctypes.c_uint64), ("columns", ctypes.c_uint64), ("worker_tiles", ctypes.c_uint64)]


class DsqError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str = ""):
        self.status = status
        super().__init__(f"{where}: {_STATUS.get(status, status)}{(': ' + detail) if detail else ''}")


_lib = None


def lib() -> ctypes.CDLL:
    """Loads libdsq.so (built by paper_1907_07346_amd/build.py); raises if it is not there."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_1907_07346_amd.build` "
                              "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        vp, u64, i32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_int
        cfgp, u64p = ctypes.POINTER(ds_config), ctypes.POINTER(ctypes.c_uint64)
        L.ds_validate_config.argtypes, L.ds_validate_config.restype = [cfgp, ctypes.c_char_p, u64], i32
        L.ds_build_topology.argtypes, L.ds_build_topology.restype = [cfgp, vp, vp, vp, u64, u64p], i32
        L.ds_message_bytes.argtypes, L.ds_message_bytes.restype = [cfgp], u64
        L.ds_build_id.argtypes, L.ds_build_id.restype = [], ctypes.c_char_p
        L.ds_step_static.argtypes = [cfgp, vp, vp, u64, vp, u64, vp, u64, vp, ctypes.c_char_p, u64]
        L.ds_step_static.restype = i32
        L.ds_init.argtypes, L.ds_init.restype = [cfgp, ctypes.POINTER(vp)], i32
        L.ds_init_ex.argtypes = [cfgp, ctypes.POINTER(ds_plan_request), ctypes.c_char_p, u64, ctypes.POINTER(vp)]
        L.ds_init_ex.restype = i32
        L.ds_step.argtypes, L.ds_step.restype = [vp, vp, u64, vp], i32
        L.ds_read_state.argtypes, L.ds_read_state.restype = [vp, vp, vp], i32
        L.ds_set_mixing.argtypes, L.ds_set_mixing.restype = [vp, vp, vp, vp], i32
        L.ds_set_rates.argtypes, L.ds_set_rates.restype = [vp, ctypes.c_float, ctypes.c_float], i32
        L.ds_workload_gradient.argtypes = [ctypes.POINTER(ds_workload), u64, vp, u64, vp, u64, vp]
        L.ds_workload_gradient.restype = i32
        L.ds_diagnostics.argtypes, L.ds_diagnostics.restype = [vp, ctypes.POINTER(ctypes.c_double)], i32
        L.ds_write_state.argtypes, L.ds_write_state.restype = [vp, vp, vp, u64], i32
        L.ds_read_messages.argtypes, L.ds_read_messages.restype = [vp, vp, u64, u64p], i32
        L.ds_state_ptrs.argtypes, L.ds_state_ptrs.restype = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), u64p], i32
        L.ds_message_ptr.argtypes, L.ds_message_ptr.restype = [vp, ctypes.POINTER(vp), u64p], i32
        L.ds_step_count.argtypes, L.ds_step_count.restype = [vp], u64
        L.ds_topk_candidate_rows.argtypes, L.ds_topk_candidate_rows.restype = [vp, ctypes.POINTER(ctypes.c_uint32)], i32
        L.ds_plan_name.argtypes, L.ds_plan_name.restype = [vp], ctypes.c_char_p
        L.ds_last_error.argtypes, L.ds_last_error.restype = [vp], ctypes.c_char_p
        L.ds_destroy.argtypes, L.ds_destroy.restype = [vp], None
        L.ds_bench_copy.argtypes, L.ds_bench_copy.restype = [vp, vp, u64, vp], i32
        L.ds_bench_stream.argtypes, L.ds_bench_stream.restype = [vp, vp, vp, u64, vp], i32
        mp, lp = ctypes.POINTER(ds_matrix), ctypes.POINTER(ds_logits)
        err = [ctypes.c_char_p, u64]
        for name, shape in (("ds_matrix_bytes", mp), ("ds_product_work_bytes", mp), ("ds_product_gradient_work_bytes", mp),
                            ("ds_top_logits_work_bytes", lp), ("ds_distill_work_bytes", lp)):
            getattr(L, name).argtypes, getattr(L, name).restype = [shape], u64
        L.ds_product.argtypes = L.ds_product_gradient.argtypes = [mp, vp, vp, u64, vp, u64, vp, u64, vp] + err
        L.ds_top_logits.argtypes = [lp, vp, u64, vp, vp, vp, u64, vp] + err
        L.ds_distill.argtypes = [lp, vp, u64, vp, vp, vp, vp, vp, u64, vp, u64, vp] + err
        sp = ctypes.POINTER(ds_sampling)
        L.ds_sample_work_bytes.argtypes, L.ds_sample_work_bytes.restype = [sp], u64
        L.ds_sample.argtypes = [sp, ctypes.POINTER(ds_sampling_rows), vp, u64, vp, vp, vp, vp, u64, vp] + err
        tp, gp = ctypes.c_void_p, ctypes.POINTER(ds_gradients)
        L.ds_gradients_bytes.argtypes, L.ds_gradients_bytes.restype = [tp, u64, u64], u64
        L.ds_gradients_lay.argtypes = [tp, u64, u64, vp, u64, gp, vp] + err
        for name in ("ds_gradient_norm_work_bytes", "ds_clip_work_bytes"):
            getattr(L, name).argtypes, getattr(L, name).restype = [gp], u64
        L.ds_gradient_norm.argtypes = [gp, vp, vp, u64, vp] + err
        L.ds_clip.argtypes = [gp, ctypes.c_double, vp, u64, vp, vp, u64, vp] + err
        for name in ("ds_product", "ds_product_gradient", "ds_top_logits", "ds_distill", "ds_sample", "ds_gradients_lay", "ds_gradient_norm", "ds_clip"):
            getattr(L, name).restype = i32
        _lib = L
    return _lib


def make_config(n: int, N: int, topo: int, kind: int, gamma: float, eta: float, *, bits: int = 0,
                block: int = 0, k: int = 0, torus=(0, 0), seed: int = 0, W_csr=None, algo: int = 0):
    """Fills a ds_config. W_csr = (rowptr int32, col int32, val float32) numpy arrays for TOPO_CSR.

    Returns (config, keepalive): keepalive holds the arrays the config points to.
    """
    c = ds_config()
    c.n, c.topo, c.N = n, topo, N
    c.torus_rows, c.torus_cols = torus
    keep = None
    if W_csr is not None:
        rp = np.ascontiguousarray(W_csr[0], dtype=np.int32)
        co = np.ascontiguousarray(W_csr[1], dtype=np.int32)
        va = np.ascontiguousarray(W_csr[2], dtype=np.float32)
        keep = (rp, co, va)
        c.W_rowptr, c.W_col, c.W_val = rp.ctypes.data, co.ctypes.data, va.ctypes.data
    c.comp.kind, c.comp.bits, c.comp.block, c.comp.k = kind, bits, block, k
    c.gamma, c.eta, c.seed = gamma, eta, seed
    c.algo = algo
    return c, keep


def ds_workload_gradient(kind: str, n: int, N: int, scale: float, seed: int, t: int, g: "torch.Tensor", x_ptr: int = 0,
                         x_ld: int = 0, stream: Optional["torch.cuda.Stream"] = None):
    """Fills the CUDA float32 tensor g (n, >= N) with the deterministic gradients of step t (see detgen.py)."""
    assert g.is_cuda and g.dtype == torch.float32 and g.dim() == 2 and g.shape[0] == n and g.stride(1) == 1
    w = ds_workload(n, GRAD_KINDS[kind], N, scale, 0.0, seed)
    st = lib().ds_workload_gradient(ctypes.byref(w), t, x_ptr, x_ld, g.data_ptr(), g.stride(0), _stream_pointer(stream))
    if st != DS_OK:
        raise RuntimeError(f"ds_workload_gradient failed with status {st}")


def config_from_workload(w: Config):
    return make_config(w.n, w.N, w.topo, w.kind, w.gamma, w.eta, bits=w.bits, block=w.block, k=w.k,
                       torus=w.torus, seed=w.seed, algo=w.algo)


def ds_validate_config(cfg: ds_config):
    buf = ctypes.create_string_buffer(256)
    st = lib().ds_validate_config(ctypes.byref(cfg), buf, 256)
    return st, buf.value.decode()


def ds_build_topology(cfg: ds_config):
    cap = max(1, cfg.n) * max(1, cfg.n)
    cap = min(cap, 16 * max(1, cfg.n) + 16)
    rowptr = np.zeros(max(1, cfg.n) + 1, np.int32)
    col = np.zeros(cap, np.int32)
    val = np.zeros(cap, np.float32)
    nnz = ctypes.c_uint64(0)
    st = lib().ds_build_topology(ctypes.byref(cfg), rowptr.ctypes.data, col.ctypes.data, val.ctypes.data,
                                 cap, ctypes.byref(nnz))
    if st != DS_OK:
        raise DsqError(st, "ds_build_topology")
    return rowptr, col[:nnz.value].copy(), val[:nnz.value].copy()


def ds_message_bytes(cfg: ds_config) -> int:
    return int(lib().ds_message_bytes(ctypes.byref(cfg)))


def ds_bench_copy(dst: "torch.Tensor", src: "torch.Tensor", stream=None):
    """Plain device copy of src into dst (same byte size, multiple of 16) with the library's copy kernel."""
    nbytes = src.numel() * src.element_size()
    assert dst.numel() * dst.element_size() == nbytes and dst.is_cuda and src.is_cuda
    st = lib().ds_bench_copy(dst.data_ptr(), src.data_ptr(), nbytes, _stream_pointer(stream))
    if st != DS_OK:
        raise DsqError(st, "ds_bench_copy")


def ds_bench_stream(x: "torch.Tensor", d: "Optional[torch.Tensor]", g: "torch.Tensor", stream=None):
    """x += g, d += g with the library's 3-loads / 2-stores streaming kernel (the access mix of ds_step); d = None:
    x += g alone, 2 loads / 1 store (the mix of the DCD-PSGD step)."""
    nbytes = x.numel() * x.element_size()
    assert (d is None or d.numel() * d.element_size() == nbytes) and g.numel() * g.element_size() == nbytes
    assert x.is_cuda and (d is None or d.is_cuda) and g.is_cuda
    st = lib().ds_bench_stream(x.data_ptr(), d.data_ptr() if d is not None else None, g.data_ptr(), nbytes, _stream_pointer(stream))
    if st != DS_OK:
        raise DsqError(st, "ds_bench_stream")


def ds_step_static(cfg: ds_config, x: "torch.Tensor", delta: "torch.Tensor", g: "torch.Tensor", msg: "torch.Tensor", t: int,
                   stream: Optional["torch.cuda.Stream"] = None):
    """One step on caller-owned CUDA tensors (x, delta: float32 (n, ld); g: float32 (n, >= N); msg: uint8), nothing allocated."""
    for a in (x, delta, g):
        assert a.is_cuda and a.dtype == torch.float32 and a.dim() == 2 and a.stride(1) == 1
    assert msg.is_cuda and msg.dtype == torch.uint8 and msg.is_contiguous() and msg.numel() >= ds_message_bytes(cfg)
    assert x.stride(0) == delta.stride(0)
    buf = ctypes.create_string_buffer(256)
    st = lib().ds_step_static(ctypes.byref(cfg), x.data_ptr(), delta.data_ptr(), x.stride(0), g.data_ptr(), g.stride(0),
                              msg.data_ptr(), t, _stream_pointer(stream), buf, 256)
    if st != DS_OK:
        raise DsqError(st, "ds_step_static", buf.value.decode())


# ---- answers: products with messages, logits (include/dsq.h says what each computes) -------------------------------

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _refuse(where: str, why: str):
    raise DsqError(DS_EINVAL, where, why)


def _on_device(where: str, names: str, *tensors) -> int:
    """The current device, on which they have to be."""
    here = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != here:
            _refuse(where, f"{names.split()[[t is other for other in tensors].index(True)]} must be on the current CUDA device")
    return here


def _rows_of(where: str, name: str, t: "torch.Tensor"):
    """(rows, columns, pitch) of a matrix whose rows are contiguous."""
    if t.dim() != 2 or t.dtype not in _DTYPES:
        _refuse(where, f"{name} must be a matrix of float32, bfloat16 or float16")
    rows, cols = t.shape
    if cols > 1 and t.stride(1) != 1:
        _refuse(where, f"{name} must have unit column stride")
    return rows, cols, t.stride(0) if rows > 1 else cols


def _vector(where: str, name: str, t: "Optional[torch.Tensor]", rows: int):
    if t is None:
        return None
    if t.dtype != torch.float32 or t.dim() != 1 or t.shape[0] != rows or not t.is_contiguous():
        _refuse(where, f"{name} must be a contiguous float32 vector of {rows}")
    return t.data_ptr()


def _new(stream, shape, dtype, like):
    """A tensor on like's device whose memory belongs to the stream that the call runs on."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _answer(name: str, work_bytes, call, shape, given, here: int, stream, *args):
    """Makes the call with scratch memory of its stream; the reason of a refusal goes into the exception.  given: the caller's tensors (the
    first is the scratch memory's pattern), whose memory, freed by its own stream, must wait for another one that the call runs on."""
    if stream is None:
        pointer = _raw_stream(here) if _raw_stream is not None else _stream_pointer(None)
    elif stream.device_index != here:
        _refuse(name, "stream must be of the current CUDA device")
    else:
        pointer = stream.cuda_stream
    size = work_bytes if type(work_bytes) is int else work_bytes(shape)
    work = _new(stream, (size,), torch.uint8, given[0]) if size else None
    at = work.data_ptr() if size else None
    st = call(shape, *args, at, size, pointer, None, 0)
    if st == DS_EINVAL:                                   # (checks only: nothing has been enqueued)
        buf = ctypes.create_string_buffer(256)
        call(shape, *args, at, size, pointer, buf, 256)
        raise DsqError(st, name, buf.value.decode())
    if stream is not None:
        for t in given:
            if t is not None:
                t.record_stream(stream)
    if st != DS_OK:
        raise DsqError(st, name)
    return pointer


def ds_matrix_bytes(rows: int, cols: int, block: int) -> int:
    return int(lib().ds_matrix_bytes(ctypes.byref(ds_matrix(rows, cols, 0, block, 0))))


def _through(name: str, work_bytes, call, msg: "torch.Tensor", x: "torch.Tensor", rows: int, cols: int, width: int, out_width: int, block: int,
             out: "Optional[torch.Tensor]", stream: Optional["torch.cuda.Stream"]):
    tokens, got, pitch = _rows_of(name, "the input", x)
    if x.requires_grad and torch.is_grad_enabled():
        _refuse(name, "the result would carry no graph: detach the input, and call ds_product_gradient for the way back")
    if got != width:
        _refuse(name, f"the input must have {width} columns")
    m = ctypes.byref(ds_matrix(rows, cols, tokens, block, _DTYPES[x.dtype]))
    if msg.dtype != torch.uint8 or not msg.is_contiguous() or msg.numel() < _lib.ds_matrix_bytes(m):
        _refuse(name, "msg must be a contiguous uint8 tensor that holds the matrix")
    here = _on_device(name, "msg x out", msg, x, out)
    out_pitch = out_width
    if out is None:
        out = _new(stream, (tokens, out_width), x.dtype, x)
    elif out.dtype != x.dtype or out.shape != (tokens, out_width):
        _refuse(name, f"out must be ({tokens}, {out_width}) and of the input's dtype")
    else:
        out_pitch = _rows_of(name, "out", out)[2]
    if tokens:
        _answer(name, work_bytes, call, m, (x, msg, out), here, stream, msg.data_ptr(), x.data_ptr(), pitch, out.data_ptr(), out_pitch)
    return out


def ds_product(msg: "torch.Tensor", x: "torch.Tensor", rows: int, block: int, out: "Optional[torch.Tensor]" = None,
               stream: Optional["torch.cuda.Stream"] = None) -> "torch.Tensor":
    """x (tokens, cols) through the matrix of `rows` rows held as 4-bit messages in msg (uint8): (tokens, rows) of x's dtype.  Autograd
    does not record the call: an x that requires a gradient is refused where gradients are recorded."""
    L, cols = lib(), x.shape[-1]
    return _through("ds_product", L.ds_product_work_bytes, L.ds_product, msg, x, rows, cols, cols, rows, block, out, stream)


def ds_product_gradient(msg: "torch.Tensor", dy: "torch.Tensor", cols: int, block: int, out: "Optional[torch.Tensor]" = None,
                        stream: Optional["torch.cuda.Stream"] = None) -> "torch.Tensor":
    """The gradient of ds_product with respect to x: dy (tokens, rows) gives (tokens, cols) of dy's dtype.  Not recorded either."""
    L, rows = lib(), dy.shape[-1]
    return _through("ds_product_gradient", L.ds_product_gradient_work_bytes, L.ds_product_gradient, msg, dy, rows, cols, rows, cols, block, out, stream)


def ds_top_logits(z: "torch.Tensor", k: int, temperature: float = 1.0, stream: Optional["torch.cuda.Stream"] = None):
    """The k largest logits of each row of z: (pairs, lse), pairs int32 (rows, k, 2) of index and float32 bits, ascending index.  They are
    what a teacher sends, numbers without a graph."""
    rows, vocab, pitch = _rows_of("ds_top_logits", "z", z)
    here = _on_device("ds_top_logits", "z", z)
    if not 1 <= k <= 256:
        _refuse("ds_top_logits", "k must be between 1 and 256")
    pairs, lse = _new(stream, (rows, k, 2), torch.int32, z), _new(stream, (rows,), torch.float32, z)
    if rows:
        L = lib()
        _answer("ds_top_logits", L.ds_top_logits_work_bytes, L.ds_top_logits,
                ctypes.byref(ds_logits(rows, vocab, k, _DTYPES[z.dtype], temperature, 0)), (z,), here, stream,
                z.data_ptr(), pitch, pairs.data_ptr(), lse.data_ptr())
    return pairs, lse


def ds_distill(z: "torch.Tensor", pairs: "torch.Tensor", temperature: float = 1.0, teacher_lse: "Optional[torch.Tensor]" = None,
               weight: "Optional[torch.Tensor]" = None, want_loss: bool = True, want_gradient: bool = True,
               dz: "Optional[torch.Tensor]" = None, stream: Optional["torch.cuda.Stream"] = None):
    """The loss of each row of z against the teacher's pairs (as ds_top_logits gives them) and its gradient: (loss, dz), None for
    what is not wanted.  dz may be given, also as z itself.  The gradient is dz and nothing else: the loss is a number without a graph,
    and a z that has one goes on with z.backward(dz)."""
    rows, vocab, pitch = _rows_of("ds_distill", "z", z)
    if pairs.dtype != torch.int32 or pairs.dim() != 3 or pairs.shape[0] != rows or pairs.shape[2] != 2 or not pairs.is_contiguous():
        _refuse("ds_distill", f"pairs must be a contiguous int32 tensor ({rows}, k, 2)")
    here = _on_device("ds_distill", "z pairs teacher_lse weight dz", z, pairs, teacher_lse, weight, dz)
    given = _vector("ds_distill", "teacher_lse", teacher_lse, rows), _vector("ds_distill", "weight", weight, rows)
    loss = _new(stream, (rows,), torch.float32, z) if want_loss else None
    dz_pitch = vocab if want_gradient else 0
    if want_gradient:
        if dz is None:
            dz = _new(stream, (rows, vocab), z.dtype, z)
        elif dz.dtype != z.dtype or dz.shape != z.shape:
            _refuse("ds_distill", "dz must have z's shape and dtype")
        else:
            dz_pitch = _rows_of("ds_distill", "dz", dz)[2]
    elif dz is not None:
        _refuse("ds_distill", "dz is given but no gradient is wanted")
    if rows:
        L = lib()
        _answer("ds_distill", L.ds_distill_work_bytes, L.ds_distill,
                ctypes.byref(ds_logits(rows, vocab, pairs.shape[1], _DTYPES[z.dtype], temperature, 0)), (z, pairs, teacher_lse, weight, dz), here, stream,
                z.data_ptr(), pitch, pairs.data_ptr(), *given, loss.data_ptr() if want_loss else None, dz.data_ptr() if want_gradient else None, dz_pitch)
    return loss, dz


def ds_sample(z: "torch.Tensor", u: "torch.Tensor", temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, stream: Optional["torch.cuda.Stream"] = None):
    """A token of each row of z from the random numbers u (float32, one per row, in [0, 1)): (token, logp), int32 and float32 (rows,).  Each
    parameter is a number, or a tensor with a number per row (float32; top_k int32).  Temperature 0 takes the largest logit.  What is drawn carries no graph."""
    rows, vocab, pitch = _rows_of("ds_sample", "z", z)
    if u.dtype != torch.float32 or u.dim() != 1 or u.shape[0] != rows or not u.is_contiguous():
        _refuse("ds_sample", f"u must be a contiguous float32 vector of {rows}")
    here = _on_device("ds_sample", "z u", z, u)
    s, each, own = ds_sampling(rows, vocab, _DTYPES[z.dtype], 0, 1.0, 1.0, 0.0, 0), None, []
    for name, value, dtype in (("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32), ("top_p", top_p, torch.float32),
                               ("min_p", min_p, torch.float32)):
        if not isinstance(value, torch.Tensor):
            if name == "top_k" and not (isinstance(value, (int, np.integer)) and 0 <= value < 1 << 31):
                _refuse("ds_sample", "top_k must be a whole number of at least 0 and below 2^31")
            setattr(s, name, int(value) if name == "top_k" else float(value))
            continue
        if value.dtype != dtype or value.dim() != 1 or value.shape[0] != rows or not value.is_contiguous():
            _refuse("ds_sample", f"{name} must be a number or a contiguous vector of {rows}, {dtype}")
        _on_device("ds_sample", name, value)
        each = each or ds_sampling_rows()
        setattr(each, name + "_dev", value.data_ptr())
        if name == "top_k":
            s.top_k = 1                                       # (some rows have one, here and of top_p: see include/dsq.h)
        if name == "top_p":                                   # (beside min_p = 0.01: 1 x 131072, fp32, 92 us, so 21.5; if all of them are 1 after all 12.5, so 19.5)
            s.top_p = 0.5
        own.append(value)
    token, logp = _new(stream, (rows,), torch.int32, z), _new(stream, (rows,), torch.float32, z)
    if rows:
        L = lib()
        _answer("ds_sample", L.ds_sample_work_bytes, L.ds_sample, ctypes.byref(s), (z, u, *own), here, stream,
                ctypes.byref(each) if each is not None else None, z.data_ptr(), pitch, u.data_ptr(), token.data_ptr(), logp.data_ptr())
    return token, logp


# ---- gradients in many tensors --------------------------------------------------------------------------------------

class Gradients:
    """Where the gradients of the workers lie, laid out once for ds_gradient_norm and ds_clip: `grads` is a list with a list of tensors per
    worker, or the tensors of one (contiguous, of float32, bfloat16 or float16, on the current CUDA device).  The calls take what the tensors hold then;
    their memory is kept as long as this is (not when a tensor's storage is resized: lay them out again).  Waits until the table is written."""

    def __init__(self, grads):
        grads = list(grads)
        if not grads or isinstance(grads[0], torch.Tensor):
            grads = [grads]
        grads = [list(of) for of in grads]
        flat = [t for of in grads for t in of]
        for t in flat:
            if not isinstance(t, torch.Tensor) or t.dtype not in _DTYPES or not t.is_contiguous():
                _refuse("Gradients", "gradients must be contiguous tensors of float32, bfloat16 or float16")
            if t.requires_grad and torch.is_grad_enabled():
                _refuse("Gradients", "a tensor requires a gradient, which the calls do not record: detach it")
        here = _on_device("Gradients", "gradients " * len(flat), *flat)
        if torch.cuda.is_current_stream_capturing():
            _refuse("Gradients", "a table cannot be laid out in a stream capture: make it before")
        self.workers, self.device = len(grads), here
        self.tensors = [t.detach() for t in flat]         # (of their own: what becomes of the caller's later does not free the memory)
        sizes = np.array([t.numel() for t in flat], np.uint64)
        worker = np.repeat(np.arange(len(grads), dtype=np.int32), [len(of) for of in grads])
        listed = np.zeros(len(flat), np.dtype([("data", "u8"), ("count", "u8"), ("dtype", "i4"), ("worker", "i4")]))
        listed["data"], listed["count"] = [t.data_ptr() for t in flat], sizes
        listed["dtype"], listed["worker"] = [_DTYPES[t.dtype] for t in flat], worker
        L, self._g = lib(), ds_gradients()
        size = L.ds_gradients_bytes(listed.ctypes.data, len(flat), len(grads))
        self.table = torch.empty(max(size, 16), dtype=torch.uint8, device=torch.device("cuda", here))
        buf = ctypes.create_string_buffer(256)
        st = L.ds_gradients_lay(listed.ctypes.data, len(flat), len(grads), self.table.data_ptr(), size, ctypes.byref(self._g),
                                _stream_pointer(None), buf, 256)
        if st != DS_OK:
            raise DsqError(st, "Gradients", buf.value.decode())
        made_on = torch.cuda.current_stream()
        made_on.synchronize()
        self._made_on, self._lent_to = made_on.cuda_stream, set()
        self._work = int(L.ds_gradient_norm_work_bytes(ctypes.byref(self._g))), int(L.ds_clip_work_bytes(ctypes.byref(self._g)))
        self.columns = int(self._g.columns)
        some = sizes > 0
        self._lo = listed["data"][some]
        self._hi = self._lo + sizes[some] * np.where(listed["dtype"][some] == 0, 4, 2).astype(np.uint64)
        self._f32, self._worker = listed["dtype"][some] == 0, worker[some].astype(np.uint64)
        before = np.concatenate([[0], np.cumsum(sizes)[:-1]]).astype(np.uint64) if len(flat) else sizes
        self._column = (before - before[np.searchsorted(worker, worker)])[some]            # (the workers' numbers do not descend)
        order = np.argsort(self._lo)
        self._apart = bool(np.all(self._hi[order][:-1] <= self._lo[order][1:]))
        self._span = (int(self._lo.min()), int(self._hi.max())) if some.any() else (0, 0)

    def _lent(self, pointer: int, stream: Optional["torch.cuda.Stream"]):
        """The memory of table and tensors, freed by the stream it is of, must wait for another one that a call ran on: one that was given, as in every call (the
        tensors may be of a third, wherever the table was laid), or a current one that the table was not laid on.  Once for each: what is freed waits for all that
        its streams have been asked for by then."""
        if pointer in self._lent_to or (stream is None and pointer == self._made_on):
            return
        if stream is None:
            stream = torch.cuda.current_stream()
        for t in (self.table, *self.tensors):
            t.record_stream(stream)
        self._lent_to.add(pointer)

    def _overlapped(self, lo: int, pitch: int) -> bool:
        """A tensor lies in the rows of this pitch from address lo on, and not where its elements go."""
        hi = lo + 4 * ((self.workers - 1) * pitch + self.columns)
        if hi <= self._span[0] or self._span[1] <= lo:
            return False
        there = np.uint64(lo) + np.uint64(4) * (self._worker * np.uint64(pitch) + self._column)
        return bool(np.any((self._lo < hi) & (self._hi > lo) & ~(self._f32 & (self._lo == there))))


def ds_gradient_norm(grads, stream: Optional["torch.cuda.Stream"] = None) -> "torch.Tensor":
    """The Euclidean norm of each worker's gradient over all its tensors: float32 (workers,).  grads: Gradients, or what they are made of
    (then they are laid out for this call, which waits for it)."""
    g, L = grads if type(grads) is Gradients else Gradients(grads), lib()
    here = _on_device("ds_gradient_norm", "gradients", g.table)
    norm = _new(stream, (g.workers,), torch.float32, g.table)
    pointer = _answer("ds_gradient_norm", g._work[0], L.ds_gradient_norm, ctypes.byref(g._g), (g.table,), here, stream, norm.data_ptr())
    g._lent(pointer, stream)
    return norm


def ds_clip(grads, max_norm: float, out: "Optional[torch.Tensor]" = None, stream: Optional["torch.cuda.Stream"] = None) -> "torch.Tensor":
    """Scales the gradients of workers whose norm is above max_norm to it, and returns the norms before: float32 (workers,).  With out, float32 (workers,
    >= columns), what ds_step takes: written there, each worker's tensors one behind the other, nothing behind them; otherwise in place.  A
    gradient that is not finite becomes zeros.  Autograd records neither, but counts both as a change in place: a graph that has saved them refuses to go backward."""
    g, L = grads if type(grads) is Gradients else Gradients(grads), lib()
    here = _on_device("ds_clip", "gradients out", g.table, out)
    at, pitch = None, 0
    if out is not None:
        rows, cols, pitch = _rows_of("ds_clip", "out", out)
        if out.dtype != torch.float32 or rows != g.workers or cols < g.columns:
            _refuse("ds_clip", f"out must be float32 ({g.workers}, at least {g.columns})")
        if out.requires_grad and torch.is_grad_enabled():
            _refuse("ds_clip", "out requires a gradient, which the call does not record")
        if rows > 1 and pitch < cols:
            _refuse("ds_clip", "the rows of out must not overlap")
        at = out.data_ptr()
        if g.columns and g._overlapped(at, pitch):
            _refuse("ds_clip", "out overlaps a gradient that does not lie where it goes")
        at = at or None
    elif not g._apart:
        _refuse("ds_clip", "tensors that overlap cannot be scaled in place")
    norm = _new(stream, (g.workers,), torch.float32, g.table)
    pointer = _answer("ds_clip", g._work[1], L.ds_clip, ctypes.byref(g._g), (g.table, out), here, stream, max_norm, at, pitch, norm.data_ptr())
    torch.autograd.graph.increment_version(g.tensors if out is None else out)    # (a graph that has saved them must notice; 1280 tensors take 27 us)
    g._lent(pointer, stream)
    return norm


class _Lent:
    """Bytes of the library's device memory for torch.as_tensor: no copy, and the owner lives as long as the tensor."""

    def __init__(self, pointer: int, size: int, owner):
        self.owner = owner
        self.__cuda_array_interface__ = {"shape": (size,), "typestr": "|u1", "data": (pointer, False), "version": 2}


class DeepSqueeze:
    """Owner of one ds_handle. Methods are the C calls with the same names."""

    def __init__(self, cfg: ds_config, keepalive=None, plan: Optional[dict] = None):
        """plan: None (ds_init) or a dict with any of variant, tile_plan, pitch_skew, autotune (ds_init_ex)."""
        self._h = ctypes.c_void_p()
        self.cfg = cfg
        self._keep = keepalive
        buf = ctypes.create_string_buffer(256)
        if plan is None:
            st = lib().ds_init_ex(ctypes.byref(cfg), None, buf, 256, ctypes.byref(self._h))
        else:
            req = ds_plan_request(plan.get("variant", 0), plan.get("tile_plan", -1), plan.get("pitch_skew", -1),
                                  plan.get("autotune", 1), 0)
            st = lib().ds_init_ex(ctypes.byref(cfg), ctypes.byref(req), buf, 256, ctypes.byref(self._h))
        if st != DS_OK:
            raise DsqError(st, "ds_init", buf.value.decode())
        self.n, self.N = int(cfg.n), int(cfg.N)
        self._stepped = False

    @classmethod
    def from_workload(cls, w: Config, plan: Optional[dict] = None) -> "DeepSqueeze":
        cfg, keep = config_from_workload(w)
        return cls(cfg, keep, plan)

    def _check(self, st: int, where: str):
        if st != DS_OK:
            raise DsqError(st, where, self.ds_last_error())

    def ds_step(self, g: "torch.Tensor", stream: Optional["torch.cuda.Stream"] = None):
        """g: CUDA float32 tensor (n, >=N) with unit column stride; runs on `stream` (default: current)."""
        assert g.is_cuda and g.dtype == torch.float32 and g.dim() == 2 and g.shape[0] == self.n
        assert g.stride(1) == 1 and g.shape[1] >= self.N
        self._check(lib().ds_step(self._h, g.data_ptr(), g.stride(0) if self.n > 1 else max(g.stride(0), g.shape[1]),
                                  _stream_pointer(stream)), "ds_step")
        self._stepped = True

    def ds_step_raw(self, g_ptr: int, g_ld: int, stream_ptr: int = 0) -> int:
        st = lib().ds_step(self._h, g_ptr, g_ld, stream_ptr)
        self._stepped = self._stepped or st == DS_OK
        return st

    def ds_set_mixing(self, W_csr):
        """W_csr = (rowptr int32, col int32, val float32): the mixing matrix for the following steps."""
        rp = np.ascontiguousarray(W_csr[0], dtype=np.int32)
        co = np.ascontiguousarray(W_csr[1], dtype=np.int32)
        va = np.ascontiguousarray(W_csr[2], dtype=np.float32)
        self._check(lib().ds_set_mixing(self._h, rp.ctypes.data, co.ctypes.data, va.ctypes.data), "ds_set_mixing")

    def ds_set_rates(self, gamma: float, eta: float):
        self._check(lib().ds_set_rates(self._h, gamma, eta), "ds_set_rates")

    def ds_read_state(self, want_delta: bool = True):
        x = np.empty((self.n, self.N), np.float32)
        d = np.empty((self.n, self.N), np.float32) if want_delta else None
        self._check(lib().ds_read_state(self._h, x.ctypes.data, d.ctypes.data if want_delta else None), "ds_read_state")
        return x, d

    def ds_write_state(self, x: Optional[np.ndarray], delta: Optional[np.ndarray], t: int):
        if x is not None:
            x = np.ascontiguousarray(x, np.float32)
            assert x.shape == (self.n, self.N)
        if delta is not None:
            delta = np.ascontiguousarray(delta, np.float32)
            assert delta.shape == (self.n, self.N)
        self._check(lib().ds_write_state(self._h, x.ctypes.data if x is not None else None,
                                         delta.ctypes.data if delta is not None else None, t), "ds_write_state")

    def ds_read_messages(self) -> np.ndarray:
        total = ds_message_bytes(self.cfg)
        buf = np.empty(total, np.uint8)
        got = ctypes.c_uint64(0)
        self._check(lib().ds_read_messages(self._h, buf.ctypes.data, total, ctypes.byref(got)), "ds_read_messages")
        assert got.value == total
        return buf

    def ds_state_ptrs(self):
        x, d, ld = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_uint64()
        self._check(lib().ds_state_ptrs(self._h, ctypes.byref(x), ctypes.byref(d), ctypes.byref(ld)), "ds_state_ptrs")
        return x.value, d.value, ld.value

    def ds_message_ptr(self):
        p, b = ctypes.c_void_p(), ctypes.c_uint64()
        self._check(lib().ds_message_ptr(self._h, ctypes.byref(p), ctypes.byref(b)), "ds_message_ptr")
        return p.value, b.value

    def ds_product(self, worker: int, x: "torch.Tensor", rows: int, first: int = 0, out: "Optional[torch.Tensor]" = None,
                   stream: Optional["torch.cuda.Stream"] = None) -> "torch.Tensor":
        """x (tokens, cols) through parameters first .. first + rows * cols - 1 of `worker` as the message of the last ds_step holds
        them (4-bit QUANT_MAXABS and DeepSqueeze's own update, whose messages are parameters; first and cols multiples of the block).  Some launch plans alternate between two message buffers:
        the call then waits for the last ds_step (see ds_message_ptr).  Otherwise the order is the caller's: the call runs on `stream`, which
        must be the last ds_step's or wait for it, and the next ds_step must not overtake the call."""
        return ds_product(self._matrix("ds_product", worker, rows, x.shape[-1], first), x, rows, self.cfg.comp.block, out, stream)

    def ds_product_gradient(self, worker: int, dy: "torch.Tensor", cols: int, first: int = 0, out: "Optional[torch.Tensor]" = None,
                            stream: Optional["torch.cuda.Stream"] = None) -> "torch.Tensor":
        """The gradient of ds_product (same worker and parameters) with respect to x."""
        return ds_product_gradient(self._matrix("ds_product_gradient", worker, dy.shape[-1], cols, first), dy, cols, self.cfg.comp.block, out, stream)

    def _matrix(self, name, worker, rows, cols, first):
        comp = self.cfg.comp
        if comp.kind != KIND_QUANT_MAXABS or comp.bits != 4:
            _refuse(name, "messages of the 4-bit block quantiser only")
        if self.cfg.algo != ALGO_DEEPSQUEEZE:
            _refuse(name, "the messages of DCD-PSGD and CHOCO-SGD are differences, no parameters")
        if not self._stepped:
            raise DsqError(DS_ESTATE, name, "no step has been taken yet")
        if not 0 <= worker < self.n:
            _refuse(name, f"there is no worker {worker}")
        if first < 0 or first % comp.block or cols % comp.block or rows < 1 or cols < 1 or first + rows * cols > self.N:
            _refuse(name, "first and cols must be multiples of the block and the matrix must lie inside the worker's parameters")
        msg, total = self.ds_message_ptr()
        lo = worker * (total // self.n) + first // comp.block * (4 + comp.block // 2)
        return torch.as_tensor(_Lent(msg + lo, ds_matrix_bytes(rows, cols, comp.block), self), device="cuda")

    def ds_diagnostics(self) -> dict:
        out = (ctypes.c_double * 4)()
        self._check(lib().ds_diagnostics(self._h, out), "ds_diagnostics")
        return {"consensus_sq": out[0], "delta_sq": out[1], "delta_mixed_sq": out[2], "message_bytes": int(out[3])}

    def ds_topk_candidate_rows(self) -> int:
        c = ctypes.c_uint32(0)
        self._check(lib().ds_topk_candidate_rows(self._h, ctypes.byref(c)), "ds_topk_candidate_rows")
        return int(c.value)

    def ds_step_count(self) -> int:
        return int(lib().ds_step_count(self._h))

    def ds_plan_name(self) -> str:
        return lib().ds_plan_name(self._h).decode()

    def ds_last_error(self) -> str:
        return lib().ds_last_error(self._h).decode()

    def ds_destroy(self):
        if self._h:
            lib().ds_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.ds_destroy()
        except Exception:
            pass
