"""Thin ctypes binding of libvf.so: argument marshalling only.

Every function has the name of the C entry point it calls (see include/vf.h) and
takes / returns torch tensors on the context's GPU.  PyTorch is used for device
memory and for the stream; every step of the scheduler runs in the library's HIP
kernels.  There is no CPU fallback: if libvf.so is missing or cannot be loaded the
import of this module's library raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Any, NamedTuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvf.so")

VF_OK, VF_EINVAL, VF_ESTATE, VF_ENOMEM, VF_EHIP = 0, -1, -2, -3, -4
VF_X_RAW_I32, VF_X_SEQ_BF16 = 0, 1
VF_FP32, VF_BF16, VF_E4M3, VF_E2M1 = 0, 1, 2, 3

EXPORTS = [
    "vf_create", "vf_destroy", "vf_set_space", "vf_set_pipeline", "vf_set_model", "vf_reset_state",
    "vf_set_state", "vf_n_scheduled", "vf_dense_count", "vf_padded_count", "vf_enumerate",
    "vf_featurize", "vf_score", "vf_score_static", "vf_score_static_max", "vf_argmin_step", "vf_greedy_schedule", "vf_beam_search", "vf_set_noise", "vf_strerror",
    "vf_last_hip_error", "vf_timer_start", "vf_timer_stop", "vf_timer_elapsed_ms",
    "vf_profile_enable", "vf_profile_read", "vf_profile_counts", "vf_set_wait_limit", "vf_sync_status",
    "vf_rms_norm", "vf_mx_quantize", "vf_mx_dequantize", "vf_mx_matmul", "vf_ssm_scan", "vf_ssm_step",
    "vf_kv_append", "vf_kv_read", "vf_kv_attend",
]

_lib = None


class VfError(RuntimeError):
    def __init__(self, code, hip=0):
        msg = lib().vf_strerror(code).decode()
        if hip:
            msg += f" (hip status {hip})"
        super().__init__(msg)
        self.code = code
        self.hip = hip


def lib():
    """Loads libvf.so (built in-tree by paper_2011_14486_amd.build).  Raises if absent."""
    global _lib
    if _lib is None:
        # PyTorch ships its own HIP runtime (soname libamdhip64.so.7).  It has to be in the
        # process first so that libvf.so binds to that same runtime: streams and device
        # pointers are only meaningful within one runtime instance.
        import torch  # noqa: F401
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with paper_2011_14486_amd.build.build_lib(); "
                              "there is no fallback path")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        L.vf_create.argtypes = [C.POINTER(vp), C.c_int, vp]
        L.vf_destroy.argtypes = [vp]
        L.vf_destroy.restype = None
        L.vf_set_space.argtypes = [vp, vp]
        L.vf_set_pipeline.argtypes = [vp, vp, C.c_int, C.c_int]
        L.vf_set_model.argtypes = [vp, vp, vp, C.c_size_t]
        L.vf_reset_state.argtypes = [vp]
        L.vf_set_state.argtypes = [vp, vp, C.c_int]
        L.vf_n_scheduled.argtypes = [vp]
        L.vf_dense_count.argtypes = [vp]
        L.vf_dense_count.restype = i64
        L.vf_padded_count.argtypes = [vp]
        L.vf_padded_count.restype = i64
        L.vf_enumerate.argtypes = [vp, C.c_int, vp, vp, vp]
        L.vf_featurize.argtypes = [vp, C.c_int, vp]
        L.vf_score.argtypes = [vp, vp, i32, i64, i64, i32, vp, vp, vp]
        L.vf_score_static.argtypes = [vp, vp, i32, i64, i64, i32, vp, vp, vp]
        L.vf_score_static_max.argtypes = [vp]
        L.vf_score_static_max.restype = i64
        L.vf_argmin_step.argtypes = [vp, C.c_int, C.c_int, vp, vp]
        L.vf_greedy_schedule.argtypes = [vp, C.c_int, C.c_int, vp, vp, vp]
        L.vf_set_noise.argtypes = [vp, C.c_float, C.c_uint64, i32]
        L.vf_beam_search.argtypes = [vp, C.c_int, C.c_int, vp, vp, vp, vp]
        L.vf_strerror.argtypes = [C.c_int]
        L.vf_strerror.restype = C.c_char_p
        L.vf_last_hip_error.argtypes = [vp]
        L.vf_timer_start.argtypes = [vp]
        L.vf_timer_stop.argtypes = [vp]
        L.vf_timer_elapsed_ms.argtypes = [vp, C.POINTER(C.c_float)]
        L.vf_profile_enable.argtypes = [vp, C.c_int]
        L.vf_profile_read.argtypes = [vp, C.c_int, C.POINTER(C.c_double), C.POINTER(i64)]
        L.vf_profile_counts.argtypes = [vp, C.POINTER(i64), C.POINTER(i64)]
        L.vf_set_wait_limit.argtypes = [vp, C.c_uint]
        L.vf_sync_status.argtypes = [vp]
        L.vf_rms_norm.argtypes = [vp, i32, vp, i64, vp, i64, vp, C.c_float, i64, i64, vp, i64, i32, vp, i64, vp]
        L.vf_mx_quantize.argtypes = [vp, i32, vp, i64, i64, i64, i32, vp, vp]
        L.vf_mx_dequantize.argtypes = [vp, i32, vp, vp, i64, i64, i32, vp, i64]
        L.vf_mx_matmul.argtypes = [vp, i32, vp, vp, vp, vp, i64, i64, i64, vp, i32, vp, i64]
        L.vf_ssm_scan.argtypes = [vp, vp, vp]
        L.vf_ssm_step.argtypes = [vp, vp, vp]
        L.vf_kv_append.argtypes = [vp, vp, vp, vp, i32, vp, i64, vp, i64, i32, vp, i64, vp, i64]
        L.vf_kv_read.argtypes = [vp, vp, vp, i32, vp, i64, vp, i64]
        L.vf_kv_attend.argtypes = [vp, vp, vp, i32, i32, vp, i64, i32, i32, C.c_float, i64, vp, i64]
        _lib = L
    return _lib


def _check(ctx, rc):
    if rc != VF_OK:
        raise VfError(rc, lib().vf_last_hip_error(ctx.handle) if ctx is not None and ctx.handle else 0)


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _np32(a, n=None):
    a = np.ascontiguousarray(a, dtype=np.int32)
    if n is not None:
        assert a.size == n, (a.size, n)
    return a


class Context:
    """Owns one vf_ctx.  Holds the torch device and stream the context was made on."""

    def __init__(self, device=0, stream=None):
        import torch
        self.torch = torch
        self.device = torch.device("cuda", device)
        with torch.cuda.device(self.device):
            self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self.index, self.raw_stream, self.current = device, self.stream.cuda_stream, torch._C._cuda_getCurrentRawStream
        h = C.c_void_p()
        rc = lib().vf_create(C.byref(h), device, C.c_void_p(self.stream.cuda_stream))
        self.handle = h if rc == VF_OK else None
        _check(None, rc)
        self.F = self.S = self.B = 0

    def close(self):
        if self.handle:
            lib().vf_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def empty(self, shape, dtype):
        return self.torch.empty(shape, dtype=dtype, device=self.device)


def vf_create(device=0, stream=None):
    return Context(device, stream)


def vf_destroy(ctx):
    ctx.close()


def vf_set_space(ctx, space):
    s = _np32(space, 65)
    _check(ctx, lib().vf_set_space(ctx.handle, s.ctypes.data_as(C.c_void_p)))
    ctx.F = int(s[64])


def vf_set_pipeline(ctx, stages):
    """stages: [S][16] (one problem) or [B][S][16] int32."""
    st = _np32(stages)
    if st.ndim == 2:
        st = st[None]
    assert st.ndim == 3 and st.shape[2] == 16
    _check(ctx, lib().vf_set_pipeline(ctx.handle, st.ctypes.data_as(C.c_void_p), st.shape[1], st.shape[0]))
    ctx.B, ctx.S = st.shape[0], st.shape[1]


def vf_set_model(ctx, model, weights):
    """model: 11-word record; weights: fp32 numpy array or CUDA tensor (flat blob)."""
    torch = ctx.torch
    m = _np32(model, 11)
    if not isinstance(weights, torch.Tensor):
        weights = torch.from_numpy(np.ascontiguousarray(weights, np.float32))
    w = weights.to(device=ctx.device, dtype=torch.float32).contiguous()
    ctx.stream.wait_stream(torch.cuda.current_stream(ctx.device))
    _check(ctx, lib().vf_set_model(ctx.handle, m.ctypes.data_as(C.c_void_p), _ptr(w), w.numel()))


def vf_reset_state(ctx):
    _check(ctx, lib().vf_reset_state(ctx.handle))


def vf_set_state(ctx, cids):
    c = _np32(cids)
    if c.ndim == 1:
        c = c[None]
    assert c.shape[0] == ctx.B
    _check(ctx, lib().vf_set_state(ctx.handle, c.ctypes.data_as(C.c_void_p) if c.size else None, c.shape[1]))


def vf_n_scheduled(ctx):
    return int(lib().vf_n_scheduled(ctx.handle))


def vf_dense_count(ctx):
    return int(lib().vf_dense_count(ctx.handle))


def vf_padded_count(ctx):
    return int(lib().vf_padded_count(ctx.handle))


def vf_enumerate(ctx, stage):
    """Returns (dec int32-viewed-as-uint32 [B][M_pad], valid uint8 [B][M_pad], n_valid int32 [B])."""
    torch = ctx.torch
    Mp = vf_padded_count(ctx)
    dec = ctx.empty((ctx.B, Mp), torch.int32)
    valid = ctx.empty((ctx.B, Mp), torch.uint8)
    nv = ctx.empty((ctx.B,), torch.int32)
    _check(ctx, lib().vf_enumerate(ctx.handle, stage, _ptr(dec), _ptr(valid), _ptr(nv)))
    return dec, valid, nv


def vf_featurize(ctx, stage, out=None):
    """Returns feat int32 [B][F][M_pad]."""
    torch = ctx.torch
    Mp = vf_padded_count(ctx)
    if out is None:
        out = ctx.empty((ctx.B, ctx.F, Mp), torch.int32)
    assert out.is_contiguous() and out.numel() == ctx.B * ctx.F * Mp and out.dtype == torch.int32
    _check(ctx, lib().vf_featurize(ctx.handle, stage, _ptr(out)))
    return out


def vf_score(ctx, x, x_kind=VF_X_RAW_I32, M=None, group=0, want_scores=True, want_min=True):
    """x: int32 [F][ld] (VF_X_RAW_I32) or bf16 [M][T][F] (VF_X_SEQ_BF16) CUDA tensor.
    Returns (scores float32 [M] or None, best_idx int32 [groups] or None, best_val float32 or None)."""
    torch = ctx.torch
    assert x.is_cuda and x.is_contiguous()
    if x_kind == VF_X_RAW_I32:
        assert x.dtype == torch.int32 and x.dim() == 2
        ld = x.shape[1]
        M = ld if M is None else M
    else:
        assert x.dtype == torch.bfloat16 and x.dim() == 3
        M = x.shape[0] if M is None else M
        ld = x.shape[1]
    ng = 1 if group == 0 else max((M + group - 1) // group, 1)
    scores = ctx.empty((M,), torch.float32) if want_scores else None
    bi = ctx.empty((ng,), torch.int32) if want_min else None
    bv = ctx.empty((ng,), torch.float32) if want_min else None
    _check(ctx, lib().vf_score(ctx.handle, _ptr(x), x_kind, M, ld, group, _ptr(scores), _ptr(bi), _ptr(bv)))
    return scores, bi, bv


def vf_score_static(ctx, x, x_kind=VF_X_RAW_I32, M=None, group=0, out=None):
    """vf_score through the entry point that allocates nothing.  out = (scores or None, best_idx,
    best_val): tensors the caller made beforehand (this wrapper makes them when out is None, which
    is an allocation by torch, outside the library call)."""
    torch = ctx.torch
    assert x.is_cuda and x.is_contiguous()
    if x_kind == VF_X_RAW_I32:
        ld = x.shape[1]
        M = ld if M is None else M
    else:
        M = x.shape[0] if M is None else M
        ld = x.shape[1]
    ng = 1 if group == 0 else max((M + group - 1) // group, 1)
    if out is None:
        out = (ctx.empty((M,), torch.float32), ctx.empty((ng,), torch.int32), ctx.empty((ng,), torch.float32))
    scores, bi, bv = out
    _check(ctx, lib().vf_score_static(ctx.handle, _ptr(x), x_kind, M, ld, group, _ptr(scores), _ptr(bi), _ptr(bv)))
    return scores, bi, bv


def vf_score_static_max(ctx):
    return int(lib().vf_score_static_max(ctx.handle))


def vf_argmin_step(ctx, stage, commit=True):
    torch = ctx.torch
    bc = ctx.empty((ctx.B,), torch.int32)
    bv = ctx.empty((ctx.B,), torch.float32)
    _check(ctx, lib().vf_argmin_step(ctx.handle, stage, 1 if commit else 0, _ptr(bc), _ptr(bv)))
    return bc, bv


def vf_greedy_schedule(ctx, first=0, last=None, out=None):
    """Returns (states int32 [B][S][16], cids int32 [B][S], values float32 [B][S])."""
    torch = ctx.torch
    last = ctx.S - 1 if last is None else last
    if out is None:
        out = (ctx.empty((ctx.B, ctx.S, 16), torch.int32), ctx.empty((ctx.B, ctx.S), torch.int32),
               ctx.empty((ctx.B, ctx.S), torch.float32))
    st, cids, vals = out
    _check(ctx, lib().vf_greedy_schedule(ctx.handle, first, last, _ptr(st), _ptr(cids), _ptr(vals)))
    return st, cids, vals


def vf_set_noise(ctx, eps, seed=0, first_rollout=0):
    _check(ctx, lib().vf_set_noise(ctx.handle, C.c_float(eps), seed, first_rollout))


def vf_beam_search(ctx, first=0, last=None):
    """Beam search of width ctx.B.  Returns (states [B][S][16], cids [B][S], values [B][S], n_beams [1])."""
    torch = ctx.torch
    last = ctx.S - 1 if last is None else last
    st = ctx.empty((ctx.B, ctx.S, 16), torch.int32)
    cids = ctx.empty((ctx.B, ctx.S), torch.int32)
    vals = ctx.empty((ctx.B, ctx.S), torch.float32)
    nb = ctx.empty((1,), torch.int32)
    _check(ctx, lib().vf_beam_search(ctx.handle, first, last, _ptr(st), _ptr(cids), _ptr(vals), _ptr(nb)))
    return st, cids, vals, nb


def vf_timer_start(ctx):
    _check(ctx, lib().vf_timer_start(ctx.handle))


def vf_timer_stop(ctx):
    _check(ctx, lib().vf_timer_stop(ctx.handle))


def vf_timer_elapsed_ms(ctx):
    ms = C.c_float()
    _check(ctx, lib().vf_timer_elapsed_ms(ctx.handle, C.byref(ms)))
    return float(ms.value)


VF_PROF_FEATURIZE, VF_PROF_SCORE, VF_PROF_COMMIT = 0, 1, 2


def vf_profile_enable(ctx, enable=True):
    _check(ctx, lib().vf_profile_enable(ctx.handle, 1 if enable else 0))


def vf_profile_read(ctx, which):
    """Returns (total milliseconds, launches) of one kernel kind since the last read."""
    ms, n = C.c_double(), C.c_int64()
    _check(ctx, lib().vf_profile_read(ctx.handle, which, C.byref(ms), C.byref(n)))
    return float(ms.value), int(n.value)


def vf_set_wait_limit(ctx, rounds):
    """Bound (polling rounds) of the waits between workgroups that share a problem in vf_greedy_schedule."""
    _check(ctx, lib().vf_set_wait_limit(ctx.handle, int(rounds)))


def vf_sync_status(ctx):
    """Waits for the context's stream; raises VfError(VF_ESTATE) if the last whole-schedule launch gave
    up a wait (its layers have then been run again per layer where the state was still there)."""
    _check(ctx, lib().vf_sync_status(ctx.handle))


def vf_profile_counts(ctx):
    """Returns (ids pushed through V, valid candidates among them) by the fused step since the last call."""
    a, b = C.c_int64(), C.c_int64()
    _check(ctx, lib().vf_profile_counts(ctx.handle, C.byref(a), C.byref(b)))
    return int(a.value), int(b.value)


# ---- sequence operators: the parts of a state-space value network ----
#
# They take and return torch tensors on the context's GPU.  Where torch's current stream is not the
# context's, the context's waits for it first and it waits for the context's afterwards, so that
# tensors may be made and used on either.  Tensors may be views; only their last dimension has to be dense.

class MX(NamedTuple):
    """A microscaled matrix of `cols` columns: codes uint8 [rows][32 kb] (VF_E4M3) or [rows][16 kb]
    (VF_E2M1), scales uint8 [rows][kb], kb = ceil(cols / 32)."""
    codes: Any
    scales: Any
    fmt: int
    cols: int


def _fail(what):
    raise ValueError(what)


def _type_of(torch, t):
    return VF_BF16 if t.dtype == torch.bfloat16 else VF_FP32 if t.dtype == torch.float32 else _fail(
        f"bfloat16 or float32 is wanted, not {t.dtype}")


def _dtype_of(torch, vf_type):
    return torch.bfloat16 if vf_type == VF_BF16 else torch.float32 if vf_type == VF_FP32 else _fail(f"no such type: {vf_type}")


def _addr(t):
    return None if t is None else t.data_ptr()


def _rows_of(ctx, t, rows, cols, dtype, name):
    """Checks a matrix [rows][cols]; returns the distance of its rows."""
    if t.shape != (rows, cols) or t.dtype != dtype or t.device != ctx.device:
        _fail(f"{name}: {dtype} [{rows}][{cols}] on {ctx.device} is wanted, got {t.dtype} {tuple(t.shape)} on {t.device}")
    ld, step = t.stride()
    if step != 1 and cols > 1 and rows > 0:   # (tensors without elements come with any strides)
        _fail(f"{name}: the last dimension has to be dense")
    return ld if rows > 1 or ld > cols else cols


def _vector(ctx, t, n, name, dtype=None):
    if t is None:
        return None
    if t.dtype != (dtype or ctx.torch.float32) or t.numel() != n or not t.is_contiguous() or t.device != ctx.device:
        _fail(f"{name}: {n} dense values of {dtype or ctx.torch.float32} on {ctx.device} are wanted")
    return t.data_ptr()


def _mx_shape(fmt, cols):
    """Bytes of codes and of scales in a row."""
    if fmt not in (VF_E4M3, VF_E2M1):
        _fail(f"no microscaled format: {fmt}")
    kb = (cols + 31) // 32
    return (32 if fmt == VF_E4M3 else 16) * kb, kb


def _mx_check(ctx, m, name):
    codes, scales, fmt, cols = m
    rows = codes.shape[0]
    nb, kb = _mx_shape(fmt, cols)
    u8, dev = ctx.torch.uint8, ctx.device
    if (codes.dtype != u8 or codes.shape != (rows, nb) or not codes.is_contiguous() or codes.device != dev or
            scales.dtype != u8 or scales.shape != (rows, kb) or not scales.is_contiguous() or scales.device != dev):
        _fail(f"{name}: codes [{rows}][{nb}] and scales [{rows}][{kb}] as dense uint8 on {dev} are wanted")
    return rows


def _out(ctx, out, rows, cols, dtype):
    """The caller's matrix or a new one, and the distance of its rows."""
    if out is None:
        return ctx.empty((rows, cols), dtype), cols
    return out, _rows_of(ctx, out, rows, cols, dtype, "out")


def _mx_empty(ctx, rows, cols, fmt):
    nb, kb = _mx_shape(fmt, cols)
    u8 = ctx.torch.uint8
    return MX(ctx.empty((rows, nb), u8), ctx.empty((rows, kb), u8), fmt, cols)


def _call(ctx, fn, args, tensors):
    """Runs a library call on the context's stream, ordered with torch's current one."""
    if ctx.current(ctx.index) == ctx.raw_stream:
        rc = fn(ctx.handle, *args)
        if rc != VF_OK:
            _check(ctx, rc)
        return
    torch = ctx.torch
    here = torch.cuda.current_stream(ctx.device)
    ctx.stream.wait_stream(here)
    for t in tensors:
        if t is not None:
            t.record_stream(ctx.stream)
    _check(ctx, fn(ctx.handle, *args))
    here.wait_stream(ctx.stream)


def vf_rms_norm(ctx, x, gain=None, eps=1e-5, residual=None, sum_out=None, out_type=None, out=None):
    """(x + residual) / sqrt(mean of squares + eps) * gain for the rows of x [rows][width].

    out_type VF_FP32 / VF_BF16 (default: x's): a tensor; VF_E4M3 / VF_E2M1: an MX.  Returns (out, sum): sum
    is x + residual in x's type, written to sum_out if given (x or residual itself is fine), None without a
    residual and a sum_out."""
    torch = ctx.torch
    kind = _type_of(torch, x)
    rows, width = x.shape
    ld_x = _rows_of(ctx, x, rows, width, x.dtype, "x")
    ld_r = _rows_of(ctx, residual, rows, width, x.dtype, "residual") if residual is not None else 0
    if sum_out is not None:
        ld_s = _rows_of(ctx, sum_out, rows, width, x.dtype, "sum_out")
    elif residual is not None:
        sum_out, ld_s = ctx.empty((rows, width), x.dtype), width
    else:
        ld_s = 0
    out_type = kind if out_type is None else out_type
    if out_type in (VF_E4M3, VF_E2M1):
        if out is None:
            out = _mx_empty(ctx, rows, width, out_type)
        elif _mx_check(ctx, out, "out") != rows or out.fmt != out_type or out.cols != width:
            _fail("out: another shape or format")
        codes, scales, ld_o = out.codes, out.scales, 0
    else:
        out, ld_o = _out(ctx, out, rows, width, _dtype_of(torch, out_type))
        codes, scales = out, None
    g = _vector(ctx, gain, width, "gain")
    _call(ctx, lib().vf_rms_norm, (kind, _addr(x), ld_x, _addr(residual), ld_r, g, eps, rows, width, _addr(sum_out), ld_s, out_type,
                                   _addr(codes), ld_o, _addr(scales)), (x, residual, gain, sum_out, codes, scales))
    return out, sum_out


def vf_mx_quantize(ctx, x, fmt, out=None):
    """x [rows][cols] as a microscaled matrix."""
    rows, cols = x.shape
    kind = _type_of(ctx.torch, x)
    ld = _rows_of(ctx, x, rows, cols, x.dtype, "x")
    if out is None:
        q = _mx_empty(ctx, rows, cols, fmt)
    else:
        q = out
        if _mx_check(ctx, q, "out") != rows or q.fmt != fmt or q.cols != cols:
            _fail("out: another shape or format")
    _call(ctx, lib().vf_mx_quantize, (kind, _addr(x), ld, rows, cols, fmt, _addr(q.codes), _addr(q.scales)), (x, q.codes, q.scales))
    return q


def vf_mx_dequantize(ctx, q, out_type=VF_BF16, out=None):
    """The values of a microscaled matrix, [rows][cols]."""
    rows = _mx_check(ctx, q, "q")
    out, ld = _out(ctx, out, rows, q.cols, _dtype_of(ctx.torch, out_type))
    _call(ctx, lib().vf_mx_dequantize, (q.fmt, _addr(q.codes), _addr(q.scales), rows, q.cols, out_type, _addr(out), ld),
          (q.codes, q.scales, out))
    return out


def vf_mx_matmul(ctx, a, w, bias=None, out_type=VF_BF16, out=None):
    """a [M][K] (MX, 8 or 4 bits) times w [N][K] (MX, VF_E2M1) transposed, plus bias[N]: [M][N]."""
    M, N = _mx_check(ctx, a, "a"), _mx_check(ctx, w, "w")
    if w.fmt != VF_E2M1 or a.cols != w.cols:
        _fail("w: VF_E2M1 with the columns of a is wanted")
    out, ld = _out(ctx, out, M, N, _dtype_of(ctx.torch, out_type))
    b = _vector(ctx, bias, N, "bias")
    _call(ctx, lib().vf_mx_matmul, (a.fmt, _addr(a.codes), _addr(a.scales), _addr(w.codes), _addr(w.scales), M, N, a.cols, b, out_type,
                                    _addr(out), ld), (a.codes, a.scales, w.codes, w.scales, bias, out))
    return out


class _Ssm(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("heads", "head_dim", "groups", "n_state", "taps")] + [
        (n, C.c_void_p) for n in ("conv_w_dev", "conv_b_dev", "a_dev", "d_dev", "dt_bias_dev")]


class _SsmIo(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("type", "n_seq", "n_slots_in", "n_slots_out")] + [
        (n, C.c_int64) for n in ("tokens", "longest")] + [
        (n, C.c_void_p) for n in ("offsets_dev", "slots_in_dev", "slots_out_dev", "xbc_dev", "dt_dev", "z_dev", "out_dev")] + [
        (n, C.c_int64) for n in ("ld_xbc", "ld_dt", "ld_z", "ld_out")] + [
        (n, C.c_void_p) for n in ("conv_in_dev", "ssm_in_dev", "conv_out_dev", "ssm_out_dev")]


class SsmLayer:
    """A scan layer: sizes and fp32 CUDA tensors conv_w [C][W], conv_b [C] or None, a [H], d [H] or None,
    dt_bias [H] or None (C = H P + 2 G N).  Holds the tensors, copies nothing."""

    def __init__(self, heads, head_dim, groups, n_state, conv_w, a, conv_b=None, d=None, dt_bias=None):
        import torch
        self.heads, self.head_dim, self.groups, self.n_state = heads, head_dim, groups, n_state
        self.channels = heads * head_dim + 2 * groups * n_state
        if conv_w.dim() != 2 or conv_w.shape[0] != self.channels:
            _fail(f"conv_w: [{self.channels}][taps] is wanted, got {tuple(conv_w.shape)}")
        self.taps = conv_w.shape[1]
        self.device = conv_w.device
        self.tensors = (conv_w, conv_b, a, d, dt_bias)
        for t, n, name in ((conv_w, self.channels * self.taps, "conv_w"), (conv_b, self.channels, "conv_b"), (a, heads, "a"),
                           (d, heads, "d"), (dt_bias, heads, "dt_bias")):
            if t is not None and (t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous() or not t.is_cuda or
                                  t.device != self.device):
                _fail(f"{name}: {n} dense float32 values on one GPU are wanted")
        self.record = _Ssm(heads, head_dim, groups, n_state, self.taps, *(_addr(t) for t in self.tensors))
        self.ref = C.byref(self.record)

    def state(self, slots, dtype):
        """Zeroed state buffers of `slots` slots: (conv [slots][C][W - 1] of dtype, ssm [slots][H][P][N] fp32)."""
        import torch
        return (torch.zeros((slots, self.channels, self.taps - 1), dtype=dtype, device=self.device),
                torch.zeros((slots, self.heads, self.head_dim, self.n_state), device=self.device))


def _ssm_state(ctx, layer, state, slots, n_seq, dtype, name):
    """Checks one direction's buffers and slot list; returns the number of slots and the addresses."""
    if state is None:
        if slots is not None:
            _fail(f"{name}: slots without state buffers")
        return 0, None, None, None
    conv, ssm = state
    n = ssm.shape[0]
    if conv.shape != (n, layer.channels, layer.taps - 1) or conv.dtype != dtype or not conv.is_contiguous():
        _fail(f"{name}: a dense {dtype} [{n}][{layer.channels}][{layer.taps - 1}] is wanted for the convolution")
    if ssm.shape != (n, layer.heads, layer.head_dim, layer.n_state) or ssm.dtype != ctx.torch.float32 or not ssm.is_contiguous():
        _fail(f"{name}: a dense float32 [slots][{layer.heads}][{layer.head_dim}][{layer.n_state}] is wanted")
    if conv.device != ctx.device or ssm.device != ctx.device:
        _fail(f"{name}: buffers on {ctx.device} are wanted")
    return n, conv.data_ptr(), ssm.data_ptr(), _vector(ctx, slots, n_seq, name + " slots", ctx.torch.int32)


def _ssm_call(ctx, fn, layer, xbc, dt, z, n_seq, longest, offsets, state, slots, state_out, slots_out, out):
    torch = ctx.torch
    if layer.device != ctx.device:
        _fail("the layer's weights are on another GPU")
    kind, dtype, tokens = _type_of(torch, xbc), xbc.dtype, xbc.shape[0]
    inner = layer.heads * layer.head_dim
    out, ld_o = _out(ctx, out, tokens, inner, dtype)
    ld_x = _rows_of(ctx, xbc, tokens, layer.channels, dtype, "xbc")
    ld_dt = _rows_of(ctx, dt, tokens, layer.heads, dtype, "dt")
    ld_z = _rows_of(ctx, z, tokens, inner, dtype, "z") if z is not None else 0
    off = _vector(ctx, offsets, n_seq + 1, "offsets", torch.int32)
    n_in, conv_in, ssm_in, s_in = _ssm_state(ctx, layer, state, slots, n_seq, dtype, "state")
    n_out, conv_out, ssm_out, s_out = _ssm_state(ctx, layer, state_out, slots_out, n_seq, dtype, "state_out")
    io = _SsmIo(kind, n_seq, n_in, n_out, tokens, longest, off, s_in, s_out, xbc.data_ptr(), dt.data_ptr(), _addr(z), out.data_ptr(),
                ld_x, ld_dt, ld_z, ld_o, conv_in, ssm_in, conv_out, ssm_out)
    _call(ctx, fn, (layer.ref, C.byref(io)), (xbc, dt, z, offsets, slots, slots_out, out, *(state or ()), *(state_out or ()),
                                              *layer.tensors))
    return out


def vf_ssm_scan(ctx, layer, xbc, dt, z=None, n_seq=1, longest=None, offsets=None, state=None, slots=None, state_out=None,
                slots_out=None, out=None):
    """Convolution, selective scan and gate over n_seq whole sequences.

    xbc [tokens][C], dt [tokens][H], z [tokens][H P] (or None), one type; offsets int32 [n_seq + 1] (None: all
    sequences have tokens / n_seq rows); longest: the longest sequence's length (default: without offsets the
    length, with offsets all tokens).  state / state_out: (conv, ssm) buffers as SsmLayer.state makes them,
    slots / slots_out int32 [n_seq] (None: slot s for sequence s, -1: none).  Returns out [tokens][H P]."""
    if longest is None:
        longest = xbc.shape[0] if offsets is not None or n_seq == 0 else xbc.shape[0] // n_seq
    return _ssm_call(ctx, lib().vf_ssm_scan, layer, xbc, dt, z, n_seq, longest, offsets, state, slots, state_out, slots_out, out)


def vf_ssm_step(ctx, layer, xbc, dt, z=None, state=None, slots=None, state_out=None, slots_out=None, out=None):
    """One more token for every row: row s continues slot slots[s] of state and leaves its state in slot
    slots_out[s] of state_out.  Arguments as vf_ssm_scan."""
    return _ssm_call(ctx, lib().vf_ssm_step, layer, xbc, dt, z, xbc.shape[0], 1, None, state, slots, state_out, slots_out, out)


# ---- attention operators: a paged cache of keys and values ----

class _Kv(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("format", "kv_heads", "head_dim", "page", "pages")] + [
        (n, C.c_void_p) for n in ("k_dev", "v_dev", "k_scales_dev", "v_scales_dev")]


class _KvSeqs(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_seq", "max_pages")] + [(n, C.c_int64) for n in ("tokens", "longest", "ld_table")] + [
        (n, C.c_void_p) for n in ("offsets_dev", "lengths_dev", "table_dev")]


class _Rope(C.Structure):
    _fields_ = [("rotary", C.c_int32), ("interleaved", C.c_int32), ("freq_dev", C.c_void_p), ("magnitude", C.c_float)]


class KvCache:
    """A paged cache of keys and values on one GPU.  Holds the tensors, copies nothing.

    VF_FP32 / VF_BF16: k and v are dense [pages][kv_heads][page][w] of that type, w = head_dim filled up with zeros to a multiple of
    8; VF_E4M3: k and v are codes, uint8 [pages][kv_heads][page][32 kb], k_scales and v_scales uint8 [pages][kv_heads][page][kb],
    kb = ceil(head_dim / 32).  `page` tokens: a power of two, 16..1024."""

    def __init__(self, fmt, head_dim, k, v, k_scales=None, v_scales=None):
        import torch
        kb = (head_dim + 31) // 32
        if fmt not in (VF_FP32, VF_BF16, VF_E4M3):
            _fail(f"no format of a cache: {fmt}")
        if not 1 <= head_dim <= 256:
            _fail(f"head_dim: 1..256 is wanted, not {head_dim}")
        dtype, width = (torch.uint8, 32 * kb) if fmt == VF_E4M3 else (_dtype_of(torch, fmt), (head_dim + 7) // 8 * 8)
        if k.dim() != 4:
            _fail(f"k: [pages][kv_heads][page][{width}] is wanted, got {tuple(k.shape)}")
        shape = tuple(k.shape[:3])
        rows = [(k, width, dtype, "k"), (v, width, dtype, "v")]
        if fmt == VF_E4M3:
            rows += [(k_scales, kb, torch.uint8, "k_scales"), (v_scales, kb, torch.uint8, "v_scales")]
        elif k_scales is not None or v_scales is not None:
            _fail("scales belong to VF_E4M3")
        for t, w, dt, name in rows:
            if t is None or t.shape != (*shape, w) or t.dtype != dt or not t.is_contiguous() or not t.is_cuda or t.device != k.device:
                _fail(f"{name}: dense {dt} {[*shape, w]} on one GPU are wanted")
        if shape[0] < 1 or shape[1] < 1 or shape[2] not in (16, 32, 64, 128, 256, 512, 1024):
            _fail(f"a page, a head and a power of two of tokens from 16 to 1024 are wanted, not {shape}")
        self.fmt, self.head_dim, self.device = fmt, head_dim, k.device
        self.pages, self.kv_heads, self.page = shape
        self.k, self.v, self.k_scales, self.v_scales = k, v, k_scales, v_scales
        self.tensors = (k, v, k_scales, v_scales)
        self.record = _Kv(fmt, self.kv_heads, head_dim, self.page, self.pages, *(_addr(t) for t in self.tensors))
        self.ref = C.byref(self.record)

    @classmethod
    def zeros(cls, fmt, pages, page, kv_heads, head_dim, device="cuda"):
        """A cache of new memory, all zeros."""
        import torch
        kb = (head_dim + 31) // 32
        new = lambda w, dt: torch.zeros((pages, kv_heads, page, w), dtype=dt, device=device)   # noqa: E731
        if fmt == VF_E4M3:
            return cls(fmt, head_dim, new(32 * kb, torch.uint8), new(32 * kb, torch.uint8), new(kb, torch.uint8), new(kb, torch.uint8))
        dtype, width = _dtype_of(torch, fmt), (head_dim + 7) // 8 * 8
        return cls(fmt, head_dim, new(width, dtype), new(width, dtype))


class Rope:
    """Rotary positions: freq float64 [rotary / 2] on the GPU, radians a position (inputs.rotary_frequencies); pairs are numbers j and
    j + rotary / 2 of a head, or 2 j and 2 j + 1 if interleaved; cosines and sines are multiplied by magnitude.  Holds the tensor."""

    def __init__(self, freq, interleaved=False, magnitude=1.0):
        import torch
        if freq.dim() != 1 or freq.dtype != torch.float64 or not freq.is_contiguous() or not freq.is_cuda:
            _fail("freq: dense float64 values on a GPU are wanted")
        self.freq, self.interleaved, self.magnitude, self.device = freq, bool(interleaved), float(magnitude), freq.device
        self.record = _Rope(2 * freq.numel(), int(self.interleaved), freq.data_ptr(), self.magnitude)
        self.ref = C.byref(self.record)


def _kv_seqs(ctx, cache, table, lengths, tokens, offsets, longest):
    """Checks what the calls share; returns the record.  (Calls of single tokens are as long as this takes: one look at each thing.)"""
    i32, dev = ctx.torch.int32, ctx.device
    if cache.device != dev:
        _fail("the cache is on another GPU")
    if table.dim() != 2:
        _fail(f"table: [n_seq][max_pages] is wanted, got {tuple(table.shape)}")
    n, wide = table.shape
    ld, step = table.stride()
    if table.dtype is not i32 or table.device != dev or (step != 1 and wide > 1 and n > 0):
        _fail(f"table: int32 rows on {dev} whose last dimension is dense are wanted, got {table.dtype} on {table.device}, strides {(ld, step)}")
    if n <= 1 and ld < wide:
        ld = wide
    if lengths.dtype is not i32 or lengths.numel() != n or not lengths.is_contiguous() or lengths.device != dev:
        _fail(f"lengths: {n} dense values of int32 on {dev} are wanted")
    if offsets is None:
        each = tokens // n if n else 0
        if each * n != tokens:
            _fail(f"{tokens} rows cannot be dealt to {n} sequences; offsets are wanted")
        return _KvSeqs(n, wide, tokens, each if longest is None else longest, ld, None, lengths.data_ptr(), table.data_ptr())
    return _KvSeqs(n, wide, tokens, tokens if longest is None else longest, ld, _vector(ctx, offsets, n + 1, "offsets", i32), lengths.data_ptr(),
                   table.data_ptr())


def _like(ctx, out, t, ld_t, rows, cols, dtype):
    """The caller's matrix or a new one of t's sizes and type, and the distance of its rows."""
    if out is None:
        torch = ctx.torch
        return torch.empty_like(t, memory_format=torch.contiguous_format), cols
    return out, ld_t if out is t else _rows_of(ctx, out, rows, cols, dtype, "out")


def _queries(ctx, cache, q, tokens, dtype):
    """Checks a matrix of heads; returns its rows, columns, heads and the distance of its rows."""
    shape = q.shape
    if len(shape) != 2 or shape[1] % cache.head_dim != 0:
        _fail(f"q: rows of heads of {cache.head_dim} are wanted, got {tuple(shape)}")
    rows, cols = shape
    if (tokens is not None and rows != tokens) or q.dtype != dtype or q.device != ctx.device:
        _fail(f"q: {dtype} [{rows if tokens is None else tokens}][{cols}] on {ctx.device} is wanted, got {q.dtype} {tuple(shape)} on {q.device}")
    ld, step = q.stride()
    if step != 1 and cols > 1 and rows > 0:
        _fail("q: the last dimension has to be dense")
    return rows, cols, cols // cache.head_dim, ld if rows > 1 or ld > cols else cols


def vf_kv_append(ctx, cache, k, v, table, lengths, q=None, rope=None, offsets=None, longest=None, q_out=None):
    """Writes new tokens' keys and values k, v [tokens][kv_heads head_dim] into the cache, keys turned by `rope` (a Rope or None).

    Sequence s has rows offsets[s] .. offsets[s + 1] - 1 (int32 [n_seq + 1]; None: all sequences have tokens / n_seq rows),
    the last of its lengths[s] positions (int32 [n_seq]), which are in the pages table[s] (int32 [n_seq][max_pages]); longest: the
    most rows of a sequence (default: without offsets their number, with offsets all tokens).  q [tokens][heads head_dim] is
    turned into q_out (default: a new tensor; q itself is fine).  Returns q_out, None without q."""
    torch = ctx.torch
    kind, dtype, tokens = _type_of(torch, k), k.dtype, k.shape[0]
    seqs = _kv_seqs(ctx, cache, table, lengths, tokens, offsets, longest)
    wide = cache.kv_heads * cache.head_dim
    ld_k = _rows_of(ctx, k, tokens, wide, dtype, "k")
    ld_v = _rows_of(ctx, v, tokens, wide, dtype, "v")
    heads = ld_q = ld_o = 0
    if q is not None:
        _, wide, heads, ld_q = _queries(ctx, cache, q, tokens, dtype)
        q_out, ld_o = _like(ctx, q_out, q, ld_q, tokens, wide, dtype)
    elif q_out is not None:
        _fail("q_out without q")
    if rope is not None and rope.device != ctx.device:
        _fail("the rotation's frequencies are on another GPU")
    _call(ctx, lib().vf_kv_append, (cache.ref, C.byref(seqs), None if rope is None else rope.ref, kind, _addr(k), ld_k, _addr(v), ld_v, heads,
                                    _addr(q), ld_q, _addr(q_out), ld_o),
          (k, v, q, q_out, table, lengths, offsets, None if rope is None else rope.freq, *cache.tensors))
    return q_out


def vf_kv_read(ctx, cache, table, lengths, tokens, offsets=None, longest=None, out_type=None, out=None):
    """Keys and values of the last positions of every sequence, `tokens` rows in all, as vf_kv_append deals rows to sequences: (k, v),
    each [tokens][kv_heads head_dim] of out_type (default: the cache's type, VF_BF16 of 8 bits); out: a pair of matrices to write to,
    either may be None and is then not read."""
    seqs = _kv_seqs(ctx, cache, table, lengths, tokens, offsets, longest)
    if out_type is None:
        out_type = VF_BF16 if cache.fmt == VF_E4M3 else cache.fmt
    dtype, wide = _dtype_of(ctx.torch, out_type), cache.kv_heads * cache.head_dim
    if out is None:
        k = ctx.empty((tokens, wide), dtype)
        out, ld = (k, ctx.torch.empty_like(k)), (wide, wide)
    else:
        ld = tuple(0 if t is None else _rows_of(ctx, t, tokens, wide, dtype, "out") for t in out)
    k, v = out
    _call(ctx, lib().vf_kv_read, (cache.ref, C.byref(seqs), out_type, _addr(k), ld[0], _addr(v), ld[1]),
          (k, v, table, lengths, offsets, *cache.tensors))
    return out


def vf_kv_attend(ctx, cache, q, table, lengths, causal=True, window=0, scale=None, offsets=None, longest=None, longest_kv=None, out=None):
    """Attention of the rows q [tokens][heads head_dim] over their sequences' keys and values in the cache: [tokens][heads head_dim].

    heads is a multiple of the cache's; rows, table, lengths, offsets and longest as for vf_kv_append.  causal: row i of m sees the keys up
    to position lengths[s] - m + i, with a window only the last `window` of them; otherwise all lengths[s] keys, whatever the window.
    scale: default head_dim ** -0.5.  longest_kv: the longest length (default: what the table can hold).  Rows without keys are zeros."""
    dtype = q.dtype
    kind = _type_of(ctx.torch, q)
    tokens, wide, heads, ld_q = _queries(ctx, cache, q, None, dtype)
    seqs = _kv_seqs(ctx, cache, table, lengths, tokens, offsets, longest)
    out, ld_o = _like(ctx, out, q, ld_q, tokens, wide, dtype)
    if window and not 0 < window < 1 << 31:
        _fail(f"window: 0 or 1 to 2^31 - 1 is wanted, not {window}")
    if longest_kv is None:
        longest_kv = seqs.max_pages * cache.page
    _call(ctx, lib().vf_kv_attend, (cache.ref, C.byref(seqs), kind, heads, q.data_ptr(), ld_q, 1 if causal else 0, window if causal else 0,
                                    cache.head_dim ** -0.5 if scale is None else scale, longest_kv, out.data_ptr(), ld_o),
          (q, out, table, lengths, offsets, *cache.tensors))
    return out
