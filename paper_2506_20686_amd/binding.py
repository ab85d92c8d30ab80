"""Python binding of libtriattn.so (ctypes).

The functions named like the C entry points pass raw pointers through; the
convenience wrappers fwd() / bwd() check torch tensors (device, dtype, shape,
contiguity), allocate outputs and workspace with torch and call the library
on torch's current stream.  All arithmetic happens in the library's HIP
kernels; there is no fallback path.
"""
from __future__ import annotations

import array
import ctypes
import math
import os
from typing import Optional

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libtriattn.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP, ERR_TOO_LARGE = 0, 1, 2, 3, 4, 5
FWD_NOALLOC_SCRATCH_BYTES = 32 << 20  # TRIATTN_FWD_NOALLOC_SCRATCH_BYTES
STARTING, ENDING = 0, 1
F32, BF16 = 0, 1
HEAD_DIM = 32
ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU = 0, 1, 2, 3

_LIB = None
_vp, _i64, _f, _int, _sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_float, ctypes.c_int, ctypes.c_size_t


class TriAttnError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {tri_attn_status_string(status)} (status {status})")


def lib():
    """Load libtriattn.so (raises if it has not been built)."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2506_20686_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        L.tri_attn_fwd_workspace_bytes.argtypes = [_int, _int, _i64, _i64, _i64,
                                                   ctypes.POINTER(_sz)]
        L.tri_attn_bwd_workspace_bytes.argtypes = L.tri_attn_fwd_workspace_bytes.argtypes
        L.tri_attn_fwd.argtypes = [_int, _int, _i64, _i64, _i64, _f] + [_vp] * 9 + [_sz, _vp]
        L.tri_attn_bwd.argtypes = [_int, _int, _i64, _i64, _i64, _f] + [_vp] * 15 + [_sz, _vp]
        L.tri_attn_fwd_noalloc.argtypes = [_int, _int, _i64, _i64, _i64, _f] + [_vp] * 9
        L.tri_attn_fwd_noalloc.restype = _int
        L.tri_attn_mfma_probe.argtypes = [_i64, _i64, _vp, _vp]
        L.tri_attn_mfma_probe.restype = _int
        L.tri_attn_rows_fwd_workspace_bytes.argtypes = [_int, _i64, _i64, _i64, _i64,
                                                        ctypes.POINTER(_sz)]
        L.tri_attn_rows_bwd_workspace_bytes.argtypes = L.tri_attn_rows_fwd_workspace_bytes.argtypes
        L.tri_attn_rows_fwd.argtypes = [_int, _i64, _i64, _i64, _i64, _f] + [_vp] * 9 + [_sz, _vp]
        L.tri_attn_rows_bwd.argtypes = [_int, _i64, _i64, _i64, _i64, _f] + [_vp] * 15 + [_sz,
                                                                                          _vp]
        L.tri_attn_fwd_batched.argtypes = [_int, _int, _i64, _i64, _i64, _i64, _f] + [_vp] * 9 + \
            [_sz, _vp]
        L.tri_attn_bwd_batched.argtypes = [_int, _int, _i64, _i64, _i64, _i64, _f] + [_vp] * 15 + \
            [_sz, _vp]
        L.tri_attn_fwd_batched.restype = _int
        L.tri_attn_bwd_batched.restype = _int
        L.tri_attn_fwd_batched_workspace_bytes.argtypes = [_int, _int, _i64, _i64, _i64, _i64,
                                                           ctypes.POINTER(_sz)]
        L.tri_attn_bwd_batched_workspace_bytes.argtypes = \
            L.tri_attn_fwd_batched_workspace_bytes.argtypes
        L.tri_attn_fwd_batched_workspace_bytes.restype = _int
        L.tri_attn_bwd_batched_workspace_bytes.restype = _int
        L.tri_attn_status_string.argtypes = [_int]
        L.tri_attn_status_string.restype = ctypes.c_char_p
        L.tri_attn_timing_enable.argtypes = [_int]
        L.tri_attn_timing_select.argtypes = [ctypes.c_uint64]
        L.tri_attn_timing_reset.argtypes = []
        L.tri_attn_timing_read.argtypes = [_int, ctypes.POINTER(ctypes.c_char_p),
                                           ctypes.POINTER(ctypes.c_double),
                                           ctypes.POINTER(ctypes.c_int64)]
        _i64p = ctypes.POINTER(_i64)
        L.tri_ln_linear_fwd.argtypes = [_int, _i64, _i64, _int, _i64p, _f, _vp, _vp, _vp, _vp,
                                        ctypes.POINTER(_vp), _vp, _vp, _vp]
        L.tri_ln_linear_bwd_workspace_bytes.argtypes = [_int, _i64, _i64, _int, _i64p,
                                                        ctypes.POINTER(_sz)]
        L.tri_ln_linear_bwd.argtypes = [_int, _i64, _i64, _int, _i64p, _vp, _vp, _vp, _vp, _vp,
                                        _vp, ctypes.POINTER(_vp), _vp, _vp, _vp, _vp, _vp, _sz,
                                        _vp]
        L.tri_transition_fwd_workspace_bytes.argtypes = [_int, _i64, _i64, _i64,
                                                         ctypes.POINTER(_sz)]
        L.tri_transition_bwd_workspace_bytes.argtypes = \
            L.tri_transition_fwd_workspace_bytes.argtypes
        L.tri_transition_fwd.argtypes = [_int, _i64, _i64, _i64, _f] + [_vp] * 9 + [_sz, _vp]
        L.tri_transition_bwd.argtypes = [_int, _i64, _i64, _i64] + [_vp] * 14 + [_sz, _vp]
        L.tri_layer_norm_fwd.argtypes = [_int, _i64, _i64, _f] + [_vp] * 7
        L.tri_layer_norm_bwd_workspace_bytes.argtypes = [_int, _i64, _i64, ctypes.POINTER(_sz)]
        L.tri_layer_norm_bwd.argtypes = [_int, _i64, _i64] + [_vp] * 9 + [_sz, _vp]
        L.tri_linear_fwd.argtypes = [_int, _i64, _i64, _i64, _int] + [_vp] * 7
        L.tri_linear_bwd_workspace_bytes.argtypes = [_int, _i64, _i64, _i64, _int,
                                                     ctypes.POINTER(_sz)]
        L.tri_linear_bwd.argtypes = [_int, _i64, _i64, _i64, _int] + [_vp] * 8 + [_sz, _vp]
        _i32p = ctypes.POINTER(ctypes.c_int32)
        L.tri_rel_bias_fwd.argtypes = [_int, _i64, _i64, _i64, _int, _i32p] + [_vp] * 6
        L.tri_rel_bias_bwd_workspace_bytes.argtypes = [_int, _i64, _i64, _i64, _int,
                                                       ctypes.POINTER(_sz)]
        L.tri_rel_bias_bwd.argtypes = [_int, _i64, _i64, _i64, _int, _i32p] + [_vp] * 5 + \
            [_sz, _vp]
        for name in ("tri_layer_norm_fwd", "tri_layer_norm_bwd_workspace_bytes",
                     "tri_layer_norm_bwd", "tri_linear_fwd", "tri_linear_bwd_workspace_bytes",
                     "tri_linear_bwd", "tri_rel_bias_fwd", "tri_rel_bias_bwd_workspace_bytes",
                     "tri_rel_bias_bwd"):
            getattr(L, name).restype = _int
        for name in ("tri_transition_fwd_workspace_bytes", "tri_transition_bwd_workspace_bytes",
                     "tri_transition_fwd", "tri_transition_bwd"):
            getattr(L, name).restype = _int
        for name in ("tri_attn_fwd_workspace_bytes", "tri_attn_bwd_workspace_bytes",
                     "tri_attn_fwd", "tri_attn_bwd", "tri_attn_timing_enable",
                     "tri_attn_timing_reset", "tri_attn_timing_read", "tri_attn_timing_select",
                     "tri_ln_linear_fwd", "tri_ln_linear_bwd_workspace_bytes",
                     "tri_ln_linear_bwd", "tri_attn_rows_fwd_workspace_bytes",
                     "tri_attn_rows_bwd_workspace_bytes", "tri_attn_rows_fwd",
                     "tri_attn_rows_bwd"):
            getattr(L, name).restype = _int
        _LIB = L
    return _LIB


# ---- the C entry points, same names -----------------------------------------------

def tri_attn_status_string(status: int) -> str:
    return lib().tri_attn_status_string(int(status)).decode()


def tri_attn_fwd_workspace_bytes(node: int, dtype: int, n: int, h: int, d: int) -> int:
    out = _sz(0)
    st = lib().tri_attn_fwd_workspace_bytes(node, dtype, n, h, d, ctypes.byref(out))
    if st != OK:
        raise TriAttnError(st, "tri_attn_fwd_workspace_bytes")
    return out.value


def tri_attn_fwd_batched_workspace_bytes(node: int, dtype: int, batch: int, n: int, h: int,
                                         d: int) -> int:
    out = _sz(0)
    st = lib().tri_attn_fwd_batched_workspace_bytes(node, dtype, batch, n, h, d,
                                                    ctypes.byref(out))
    if st != OK:
        raise TriAttnError(st, "tri_attn_fwd_batched_workspace_bytes")
    return out.value


def tri_attn_bwd_batched_workspace_bytes(node: int, dtype: int, batch: int, n: int, h: int,
                                         d: int) -> int:
    out = _sz(0)
    st = lib().tri_attn_bwd_batched_workspace_bytes(node, dtype, batch, n, h, d,
                                                    ctypes.byref(out))
    if st != OK:
        raise TriAttnError(st, "tri_attn_bwd_batched_workspace_bytes")
    return out.value


def tri_attn_bwd_workspace_bytes(node: int, dtype: int, n: int, h: int, d: int) -> int:
    out = _sz(0)
    st = lib().tri_attn_bwd_workspace_bytes(node, dtype, n, h, d, ctypes.byref(out))
    if st != OK:
        raise TriAttnError(st, "tri_attn_bwd_workspace_bytes")
    return out.value


def tri_attn_fwd(node, dtype, n, h, d, scale, q, k, v, g, bias, mask, out, lse, workspace,
                 workspace_bytes, stream) -> int:
    """Raw call: every tensor argument is an integer device address (or None)."""
    return lib().tri_attn_fwd(node, dtype, n, h, d, scale, q, k, v, g, bias, mask, out, lse,
                              workspace, workspace_bytes, stream)


def tri_attn_mfma_probe(blocks: int, iters: int, out, stream) -> int:
    """Raw call of the MFMA counter-calibration kernel (out: device address)."""
    return lib().tri_attn_mfma_probe(blocks, iters, out, stream)


def tri_attn_fwd_noalloc(node, dtype, n, h, d, scale, q, k, v, g, bias, mask, out, lse,
                         stream) -> int:
    """Raw call: every tensor argument is an integer device address (or None)."""
    return lib().tri_attn_fwd_noalloc(node, dtype, n, h, d, scale, q, k, v, g, bias, mask, out,
                                      lse, stream)


def tri_attn_bwd(node, dtype, n, h, d, scale, q, k, v, g, bias, mask, out, lse, dout, dq, dk,
                 dv, dg, dbias, workspace, workspace_bytes, stream) -> int:
    """Raw call: every tensor argument is an integer device address (or None)."""
    return lib().tri_attn_bwd(node, dtype, n, h, d, scale, q, k, v, g, bias, mask, out, lse,
                              dout, dq, dk, dv, dg, dbias, workspace, workspace_bytes, stream)


def tri_attn_rows_fwd_workspace_bytes(dtype: int, n: int, rows: int, h: int, d: int) -> int:
    out = _sz(0)
    st = lib().tri_attn_rows_fwd_workspace_bytes(dtype, n, rows, h, d, ctypes.byref(out))
    if st != OK:
        raise TriAttnError(st, "tri_attn_rows_fwd_workspace_bytes")
    return out.value


def tri_attn_rows_bwd_workspace_bytes(dtype: int, n: int, rows: int, h: int, d: int) -> int:
    out = _sz(0)
    st = lib().tri_attn_rows_bwd_workspace_bytes(dtype, n, rows, h, d, ctypes.byref(out))
    if st != OK:
        raise TriAttnError(st, "tri_attn_rows_bwd_workspace_bytes")
    return out.value


def tri_attn_rows_fwd(dtype, n, rows, h, d, scale, q, k, v, g, bias, mask, out, lse, workspace,
                      workspace_bytes, stream) -> int:
    """Raw call: every tensor argument is an integer device address (or None)."""
    return lib().tri_attn_rows_fwd(dtype, n, rows, h, d, scale, q, k, v, g, bias, mask, out, lse,
                                   workspace, workspace_bytes, stream)


def tri_attn_rows_bwd(dtype, n, rows, h, d, scale, q, k, v, g, bias, mask, out, lse, dout, dq,
                      dk, dv, dg, dbias_partial, workspace, workspace_bytes, stream) -> int:
    """Raw call: every tensor argument is an integer device address (or None)."""
    return lib().tri_attn_rows_bwd(dtype, n, rows, h, d, scale, q, k, v, g, bias, mask, out, lse,
                                   dout, dq, dk, dv, dg, dbias_partial, workspace,
                                   workspace_bytes, stream)


def tri_attn_fwd_batched(node, dtype, batch, n, h, d, scale, q, k, v, g, bias, mask, out, lse,
                         workspace, workspace_bytes, stream) -> int:
    """Raw call: every tensor argument is an integer device address (or None)."""
    return lib().tri_attn_fwd_batched(node, dtype, batch, n, h, d, scale, q, k, v, g, bias, mask,
                                      out, lse, workspace, workspace_bytes, stream)


def tri_attn_bwd_batched(node, dtype, batch, n, h, d, scale, q, k, v, g, bias, mask, out, lse,
                         dout, dq, dk, dv, dg, dbias, workspace, workspace_bytes, stream) -> int:
    """Raw call: every tensor argument is an integer device address (or None)."""
    return lib().tri_attn_bwd_batched(node, dtype, batch, n, h, d, scale, q, k, v, g, bias, mask,
                                      out, lse, dout, dq, dk, dv, dg, dbias, workspace,
                                      workspace_bytes, stream)


def _cols_arr(cols):
    return (_i64 * len(cols))(*[int(c) for c in cols])


def tri_ln_linear_fwd(dtype, m, k, cols, eps, x, gamma, beta, w, outs, mean, rstd,
                      stream) -> int:
    """Raw call: tensor arguments are integer device addresses; cols and outs
    are Python sequences (passed as host arrays)."""
    outs_arr = (_vp * len(outs))(*outs)
    return lib().tri_ln_linear_fwd(dtype, m, k, len(cols), _cols_arr(cols), eps, x, gamma, beta,
                                   w, outs_arr, mean, rstd, stream)


def tri_ln_linear_bwd_workspace_bytes(dtype: int, m: int, k: int, cols) -> int:
    out = _sz(0)
    st = lib().tri_ln_linear_bwd_workspace_bytes(dtype, m, k, len(cols), _cols_arr(cols),
                                                 ctypes.byref(out))
    if st != OK:
        raise TriAttnError(st, "tri_ln_linear_bwd_workspace_bytes")
    return out.value


def tri_ln_linear_bwd(dtype, m, k, cols, x, gamma, beta, w, mean, rstd, douts, dx, dw, dgamma,
                      dbeta, workspace, workspace_bytes, stream) -> int:
    """Raw call: tensor arguments are integer device addresses; cols and douts
    are Python sequences (passed as host arrays)."""
    douts_arr = (_vp * len(douts))(*douts)
    return lib().tri_ln_linear_bwd(dtype, m, k, len(cols), _cols_arr(cols), x, gamma, beta, w,
                                   mean, rstd, douts_arr, dx, dw, dgamma, dbeta, workspace,
                                   workspace_bytes, stream)


def tri_transition_fwd_workspace_bytes(dtype: int, m: int, c: int, f: int) -> int:
    out = _sz(0)
    st = lib().tri_transition_fwd_workspace_bytes(dtype, m, c, f, ctypes.byref(out))
    if st != OK:
        raise TriAttnError(st, "tri_transition_fwd_workspace_bytes")
    return out.value


def tri_transition_bwd_workspace_bytes(dtype: int, m: int, c: int, f: int) -> int:
    out = _sz(0)
    st = lib().tri_transition_bwd_workspace_bytes(dtype, m, c, f, ctypes.byref(out))
    if st != OK:
        raise TriAttnError(st, "tri_transition_bwd_workspace_bytes")
    return out.value


def tri_transition_fwd(dtype, m, c, f, eps, x, gamma, beta, w1, w2, out, mean, rstd, workspace,
                       workspace_bytes, stream) -> int:
    """Raw call: every tensor argument is an integer device address (or None)."""
    return lib().tri_transition_fwd(dtype, m, c, f, eps, x, gamma, beta, w1, w2, out, mean,
                                    rstd, workspace, workspace_bytes, stream)


def tri_transition_bwd(dtype, m, c, f, x, gamma, beta, w1, w2, mean, rstd, dout, dx, dw1, dw2,
                       dgamma, dbeta, workspace, workspace_bytes, stream) -> int:
    """Raw call: every tensor argument is an integer device address (or None)."""
    return lib().tri_transition_bwd(dtype, m, c, f, x, gamma, beta, w1, w2, mean, rstd, dout,
                                    dx, dw1, dw2, dgamma, dbeta, workspace, workspace_bytes,
                                    stream)


def tri_layer_norm_fwd(dtype, m, c, eps, x, gamma, beta, out, mean, rstd, stream) -> int:
    """Raw call: every tensor argument is an integer device address (or None)."""
    return lib().tri_layer_norm_fwd(dtype, m, c, eps, x, gamma, beta, out, mean, rstd, stream)


def tri_layer_norm_bwd_workspace_bytes(dtype: int, m: int, c: int) -> int:
    out = _sz(0)
    st = lib().tri_layer_norm_bwd_workspace_bytes(dtype, m, c, ctypes.byref(out))
    if st != OK:
        raise TriAttnError(st, "tri_layer_norm_bwd_workspace_bytes")
    return out.value


def tri_layer_norm_bwd(dtype, m, c, x, gamma, mean, rstd, dout, dx, dgamma, dbeta, workspace,
                       workspace_bytes, stream) -> int:
    """Raw call: every tensor argument is an integer device address (or None)."""
    return lib().tri_layer_norm_bwd(dtype, m, c, x, gamma, mean, rstd, dout, dx, dgamma, dbeta,
                                    workspace, workspace_bytes, stream)


def tri_linear_fwd(dtype, m, k, n, act, x, w, bias, residual, out, z, stream) -> int:
    """Raw call: every tensor argument is an integer device address (or None)."""
    return lib().tri_linear_fwd(dtype, m, k, n, act, x, w, bias, residual, out, z, stream)


def tri_linear_bwd_workspace_bytes(dtype: int, m: int, k: int, n: int, act: int) -> int:
    out = _sz(0)
    st = lib().tri_linear_bwd_workspace_bytes(dtype, m, k, n, act, ctypes.byref(out))
    if st != OK:
        raise TriAttnError(st, "tri_linear_bwd_workspace_bytes")
    return out.value


def tri_linear_bwd(dtype, m, k, n, act, x, w, z, dout, dx, dw, dbias, workspace, workspace_bytes,
                   stream) -> int:
    """Raw call: every tensor argument is an integer device address (or None)."""
    return lib().tri_linear_bwd(dtype, m, k, n, act, x, w, z, dout, dx, dw, dbias, workspace,
                                workspace_bytes, stream)


def _edges_arr(edges):
    if isinstance(edges, (bytes, bytearray)):  # would be taken as the array's memory
        raise TypeError("edges must be a sequence of integers")
    try:
        values = array.array("i", edges)  # 32 bits; checks every value
    except OverflowError as e:
        raise ValueError("edges must fit 32 bits") from e
    except TypeError as e:
        raise TypeError("edges must be a sequence of integers") from e
    return (ctypes.c_int32 * len(values)).from_buffer(values)


def tri_rel_bias_fwd(dtype, batch, n, h, edges, pos, chain, table, base, out, stream) -> int:
    """Raw call: tensor arguments are integer device addresses (or None); edges
    is a Python sequence (passed as a host array)."""
    return lib().tri_rel_bias_fwd(dtype, batch, n, h, len(edges), _edges_arr(edges), pos, chain,
                                  table, base, out, stream)


def tri_rel_bias_bwd_workspace_bytes(dtype: int, batch: int, n: int, h: int,
                                     n_edges: int) -> int:
    out = _sz(0)
    st = lib().tri_rel_bias_bwd_workspace_bytes(dtype, batch, n, h, n_edges, ctypes.byref(out))
    if st != OK:
        raise TriAttnError(st, "tri_rel_bias_bwd_workspace_bytes")
    return out.value


def tri_rel_bias_bwd(dtype, batch, n, h, edges, pos, chain, dout, dtable, workspace,
                     workspace_bytes, stream) -> int:
    """Raw call: tensor arguments are integer device addresses (or None); edges
    is a Python sequence (passed as a host array)."""
    return lib().tri_rel_bias_bwd(dtype, batch, n, h, len(edges), _edges_arr(edges), pos, chain,
                                  dout, dtable, workspace, workspace_bytes, stream)


def tri_attn_timing_enable(on: bool) -> None:
    st = lib().tri_attn_timing_enable(1 if on else 0)
    if st != OK:
        raise TriAttnError(st, "tri_attn_timing_enable")


def tri_attn_timing_select(names=None) -> None:
    """Time only the kernels named in `names` (None: every kernel)."""
    mask = 0
    if names is not None:
        index = {}
        i = 0
        while True:
            r = tri_attn_timing_read(i)
            if r is None:
                break
            index[r[0]] = i
            i += 1
        for n in names:
            if n not in index:
                raise ValueError(f"unknown kernel name {n!r}")
            mask |= 1 << index[n]
    st = lib().tri_attn_timing_select(mask)
    if st != OK:
        raise TriAttnError(st, "tri_attn_timing_select")


def tri_attn_timing_reset() -> None:
    st = lib().tri_attn_timing_reset()
    if st != OK:
        raise TriAttnError(st, "tri_attn_timing_reset")


def tri_attn_timing_read(index: int):
    """(name, total_ms, launches) of kernel `index`, or None past the last one."""
    name, ms, cnt = ctypes.c_char_p(), ctypes.c_double(), ctypes.c_int64()
    st = lib().tri_attn_timing_read(index, ctypes.byref(name), ctypes.byref(ms),
                                    ctypes.byref(cnt))
    if st == ERR_INVALID_ARG:
        return None
    if st != OK:
        raise TriAttnError(st, "tri_attn_timing_read")
    return name.value.decode(), ms.value, cnt.value


def kernel_times():
    """{kernel name: (total ms, launches)} accumulated since the last reset."""
    out, i = {}, 0
    while True:
        r = tri_attn_timing_read(i)
        if r is None:
            return out
        out[r[0]] = (r[1], r[2])
        i += 1


# ---- torch convenience wrappers -------------------------------------------------------

_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}


def _check(name, t, shape, dtype, device):
    # what a good call passes, in one expression (a third less time than the
    # tests one by one, which name the fault): up to eight tensors a call,
    # where the smallest calls' kernels take 20 to 45 us in all
    if (isinstance(t, torch.Tensor) and t.shape == shape and t.dtype is dtype
            and t.device == device and device.type == "cuda" and t.is_contiguous()):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device != device or t.device.type != "cuda":
        raise ValueError(f"{name} must be on {device} (got {t.device})")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype} (got {t.dtype})")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)} (got {tuple(t.shape)})")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _common(q, k, v, g, bias, mask):
    """Shapes of a single map ([n, n, h, d]) or a batch ([b, n, n, h, d]);
    returns (lead, n, h, d, dtype code, device) with lead = () or (b,)."""
    if q.dim() not in (4, 5):
        raise ValueError("q must be [n, n, h, d] or [b, n, n, h, d]")
    lead = tuple(q.shape[:-4])
    n, n2, h, d = q.shape[-4:]
    if n != n2:
        raise ValueError("q must be square in its two pair axes")
    if q.dtype not in _DTYPES:
        raise ValueError(f"unsupported dtype {q.dtype}")
    dev = q.device
    shape, dtype = q.shape, q.dtype
    _check("q", q, shape, dtype, dev)
    _check("k", k, shape, dtype, dev)
    _check("v", v, shape, dtype, dev)
    _check("g", g, shape, dtype, dev)
    _check("bias", bias, lead + (n, n, h), dtype, dev)
    if mask is not None:
        _check("mask", mask, lead + (n, n), torch.uint8, dev)
    return lead, n, h, d, _DTYPES[q.dtype], dev


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(dev):
    # the handle alone: 0.1 us, against 2 us for the stream object around it
    if dev.index is None:
        return torch.cuda.current_stream(dev).cuda_stream
    return torch._C._cuda_getCurrentRawStream(dev.index)


# The torch wrappers give a batch one workspace copy per sample (one launch per
# kernel for the whole batch) up to this size, and the unbatched workspace
# (sample by sample) beyond it.
BATCH_WORKSPACE_LIMIT = 4 << 30


def _batch_workspace(batched: int, one: int) -> int:
    return batched if batched <= max(one, BATCH_WORKSPACE_LIMIT) else one


def default_scale(d: int) -> float:
    return 1.0 / math.sqrt(d)


def fwd(q, k, v, g, bias, mask=None, node: int = STARTING, scale: Optional[float] = None,
        workspace: Optional[torch.Tensor] = None):
    """Triangle attention forward.  Returns (out [n,n,h,d], lse [n,n,h] fp32);
    with a leading batch axis on every tensor, the batched call."""
    lead, n, h, d, dt, dev = _common(q, k, v, g, bias, mask)
    scale = default_scale(d) if scale is None else float(scale)
    out = torch.empty_like(q)
    lse = torch.empty(lead + (n, n, h), dtype=torch.float32, device=dev)
    # a batch gets one copy of the workspace per sample (one launch per kernel
    # for the whole batch); a smaller workspace passed in runs it sample by sample
    one = tri_attn_fwd_workspace_bytes(node, dt, n, h, d)
    need = _batch_workspace(tri_attn_fwd_batched_workspace_bytes(node, dt, lead[0], n, h, d),
                            one) if lead else one
    if workspace is None or workspace.numel() < one:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    args = (scale, _ptr(q), _ptr(k), _ptr(v), _ptr(g), _ptr(bias), _ptr(mask), _ptr(out),
            _ptr(lse), _ptr(workspace), workspace.numel(), _stream(dev))
    if lead:
        st = tri_attn_fwd_batched(node, dt, lead[0], n, h, d, *args)
    else:
        st = tri_attn_fwd(node, dt, n, h, d, *args)
    if st != OK:
        raise TriAttnError(st, "tri_attn_fwd_batched" if lead else "tri_attn_fwd")
    return out, lse


def fwd_noalloc(q, k, v, g, bias, mask=None, node: int = STARTING,
                scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                lse: Optional[torch.Tensor] = None):
    """Triangle attention forward through the allocation-free entry point (the
    library's own scratch array instead of a workspace).  out and lse may be
    passed in; otherwise they are allocated here (the library allocates
    nothing).  Unbatched only."""
    lead, n, h, d, dt, dev = _common(q, k, v, g, bias, mask)
    if lead:
        raise ValueError("fwd_noalloc takes one pair map (no batch axis)")
    scale = default_scale(d) if scale is None else float(scale)
    if out is None:
        out = torch.empty_like(q)
    if lse is None:
        lse = torch.empty((n, n, h), dtype=torch.float32, device=dev)
    _check("out", out, (n, n, h, d), q.dtype, dev)
    _check("lse", lse, (n, n, h), torch.float32, dev)
    st = tri_attn_fwd_noalloc(node, dt, n, h, d, scale, _ptr(q), _ptr(k), _ptr(v), _ptr(g),
                              _ptr(bias), _ptr(mask), _ptr(out), _ptr(lse), _stream(dev))
    if st != OK:
        raise TriAttnError(st, "tri_attn_fwd_noalloc")
    return out, lse


def bwd(q, k, v, g, bias, out, lse, dout, mask=None, node: int = STARTING,
        scale: Optional[float] = None, workspace: Optional[torch.Tensor] = None):
    """Triangle attention backward.  Returns (dq, dk, dv, dg, dbias); batched
    when the tensors have a leading batch axis."""
    lead, n, h, d, dt, dev = _common(q, k, v, g, bias, mask)
    _check("out", out, q.shape, q.dtype, dev)
    _check("dout", dout, q.shape, q.dtype, dev)
    _check("lse", lse, lead + (n, n, h), torch.float32, dev)
    scale = default_scale(d) if scale is None else float(scale)
    dq, dk, dv, dg = [torch.empty_like(q) for _ in range(4)]
    dbias = torch.empty_like(bias)
    one = tri_attn_bwd_workspace_bytes(node, dt, n, h, d)
    need = _batch_workspace(tri_attn_bwd_batched_workspace_bytes(node, dt, lead[0], n, h, d),
                            one) if lead else one
    if workspace is None or workspace.numel() < one:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    args = (scale, _ptr(q), _ptr(k), _ptr(v), _ptr(g), _ptr(bias), _ptr(mask), _ptr(out),
            _ptr(lse), _ptr(dout), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dg), _ptr(dbias),
            _ptr(workspace), workspace.numel(), _stream(dev))
    if lead:
        st = tri_attn_bwd_batched(node, dt, lead[0], n, h, d, *args)
    else:
        st = tri_attn_bwd(node, dt, n, h, d, *args)
    if st != OK:
        raise TriAttnError(st, "tri_attn_bwd_batched" if lead else "tri_attn_bwd")
    return dq, dk, dv, dg, dbias


def _rows_common(q, k, v, g, bias, mask):
    if q.dim() != 4:
        raise ValueError("q must be [rows, n, h, d]")
    rows, n, h, d = q.shape
    if q.dtype not in _DTYPES:
        raise ValueError(f"unsupported dtype {q.dtype}")
    dev = q.device
    for name, t in (("q", q), ("k", k), ("v", v), ("g", g)):
        _check(name, t, (rows, n, h, d), q.dtype, dev)
    _check("bias", bias, (n, n, h), q.dtype, dev)
    if mask is not None:
        _check("mask", mask, (rows, n), torch.uint8, dev)
    return rows, n, h, d, _DTYPES[q.dtype], dev


def rows_fwd(q, k, v, g, bias, mask=None, scale: Optional[float] = None,
             workspace: Optional[torch.Tensor] = None):
    """Starting-node forward over a range of rows: q, k, v, g [rows, n, h, d]
    (the range's rows), bias [n, n, h] (whole map), mask [rows, n].  Returns
    (out [rows, n, h, d], lse [rows, n, h] fp32)."""
    rows, n, h, d, dt, dev = _rows_common(q, k, v, g, bias, mask)
    scale = default_scale(d) if scale is None else float(scale)
    out = torch.empty_like(q)
    lse = torch.empty((rows, n, h), dtype=torch.float32, device=dev)
    need = tri_attn_rows_fwd_workspace_bytes(dt, n, rows, h, d)
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    st = tri_attn_rows_fwd(dt, n, rows, h, d, scale, _ptr(q), _ptr(k), _ptr(v), _ptr(g),
                           _ptr(bias), _ptr(mask), _ptr(out), _ptr(lse), _ptr(workspace),
                           workspace.numel(), _stream(dev))
    if st != OK:
        raise TriAttnError(st, "tri_attn_rows_fwd")
    return out, lse


def rows_bwd(q, k, v, g, bias, out, lse, dout, mask=None, scale: Optional[float] = None,
             workspace: Optional[torch.Tensor] = None):
    """Starting-node backward over a range of rows.  Returns (dq, dk, dv, dg
    [rows, n, h, d], dbias_partial [n, n, h] fp32: the range's term of the
    bias gradient)."""
    rows, n, h, d, dt, dev = _rows_common(q, k, v, g, bias, mask)
    _check("out", out, (rows, n, h, d), q.dtype, dev)
    _check("dout", dout, (rows, n, h, d), q.dtype, dev)
    _check("lse", lse, (rows, n, h), torch.float32, dev)
    scale = default_scale(d) if scale is None else float(scale)
    dq, dk, dv, dg = [torch.empty_like(q) for _ in range(4)]
    dbp = torch.empty((n, n, h), dtype=torch.float32, device=dev)
    need = tri_attn_rows_bwd_workspace_bytes(dt, n, rows, h, d)
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    st = tri_attn_rows_bwd(dt, n, rows, h, d, scale, _ptr(q), _ptr(k), _ptr(v), _ptr(g),
                           _ptr(bias), _ptr(mask), _ptr(out), _ptr(lse), _ptr(dout), _ptr(dq),
                           _ptr(dk), _ptr(dv), _ptr(dg), _ptr(dbp), _ptr(workspace),
                           workspace.numel(), _stream(dev))
    if st != OK:
        raise TriAttnError(st, "tri_attn_rows_bwd")
    return dq, dk, dv, dg, dbp


class TriangleAttention(torch.autograd.Function):
    """autograd wrapper: out = triangle_attention(q, k, v, g, bias; mask, node)."""

    @staticmethod
    def forward(ctx, q, k, v, g, bias, mask=None, node=STARTING, scale=None):
        out, lse = fwd(q, k, v, g, bias, mask, node, scale)
        ctx.save_for_backward(q, k, v, g, bias, out, lse)
        ctx.mask, ctx.node, ctx.scale = mask, node, scale
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, g, bias, out, lse = ctx.saved_tensors
        grads = bwd(q, k, v, g, bias, out, lse, dout.contiguous(), ctx.mask, ctx.node, ctx.scale)
        return (*grads, None, None, None)


def triangle_attention(q, k, v, g, bias, mask=None, node: int = STARTING, scale=None):
    return TriangleAttention.apply(q, k, v, g, bias, mask, node, scale)


# ---- fused layer-norm + linear projection ---------------------------------------------

def ln_linear_fwd(x, gamma, beta, w, cols, eps: float = 1e-5):
    """o2 = layer_norm(x) * gamma + beta, then @ w, split column-wise into
    len(cols) tensors [m, cols[i]].  x [m, k] bf16.  Returns (outs, mean,
    rstd)."""
    if x.dim() != 2:
        raise ValueError("x must be [m, k]")
    m, k = x.shape
    dev = x.device
    ncols = int(sum(cols))
    _check("x", x, (m, k), torch.bfloat16, dev)
    _check("gamma", gamma, (k,), torch.bfloat16, dev)
    _check("beta", beta, (k,), torch.bfloat16, dev)
    _check("w", w, (k, ncols), torch.bfloat16, dev)
    outs = [torch.empty((m, int(c)), dtype=torch.bfloat16, device=dev) for c in cols]
    mean = torch.empty(m, dtype=torch.float32, device=dev)
    rstd = torch.empty(m, dtype=torch.float32, device=dev)
    st = tri_ln_linear_fwd(BF16, m, k, cols, float(eps), _ptr(x), _ptr(gamma), _ptr(beta),
                           _ptr(w), [o.data_ptr() for o in outs], _ptr(mean), _ptr(rstd),
                           _stream(dev))
    if st != OK:
        raise TriAttnError(st, "tri_ln_linear_fwd")
    return outs, mean, rstd


def ln_linear_bwd(x, gamma, beta, w, mean, rstd, douts, eps: float = 1e-5,
                  workspace: Optional[torch.Tensor] = None):
    """Gradients of sum(do2 * o2) for ln_linear_fwd: douts are do2 split like
    the forward's outputs.  Returns (dx [m, k] bf16, dw [k, ncols] fp32,
    dgamma [k] fp32, dbeta [k] fp32).  eps is unused (the saved rstd holds it)."""
    m, k = x.shape
    dev = x.device
    cols = [int(d.shape[1]) for d in douts]
    ncols = sum(cols)
    _check("x", x, (m, k), torch.bfloat16, dev)
    _check("gamma", gamma, (k,), torch.bfloat16, dev)
    _check("beta", beta, (k,), torch.bfloat16, dev)
    _check("w", w, (k, ncols), torch.bfloat16, dev)
    _check("mean", mean, (m,), torch.float32, dev)
    _check("rstd", rstd, (m,), torch.float32, dev)
    for i, d in enumerate(douts):
        _check(f"douts[{i}]", d, (m, cols[i]), torch.bfloat16, dev)
    dx = torch.empty_like(x)
    dw = torch.empty((k, ncols), dtype=torch.float32, device=dev)
    dgamma = torch.empty(k, dtype=torch.float32, device=dev)
    dbeta = torch.empty(k, dtype=torch.float32, device=dev)
    need = tri_ln_linear_bwd_workspace_bytes(BF16, m, k, cols)
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    st = tri_ln_linear_bwd(BF16, m, k, cols, _ptr(x), _ptr(gamma), _ptr(beta), _ptr(w),
                           _ptr(mean), _ptr(rstd), [d.data_ptr() for d in douts], _ptr(dx),
                           _ptr(dw), _ptr(dgamma), _ptr(dbeta), _ptr(workspace),
                           workspace.numel(), _stream(dev))
    if st != OK:
        raise TriAttnError(st, "tri_ln_linear_bwd")
    return dx, dw, dgamma, dbeta


# ---- fused transition layer -------------------------------------------------------------

def _trn_common(x, gamma, beta, w1, w2):
    if x.dim() != 2:
        raise ValueError("x must be [m, c]")
    m, c = x.shape
    f = w2.shape[0]
    dev = x.device
    _check("x", x, (m, c), torch.bfloat16, dev)
    _check("gamma", gamma, (c,), torch.bfloat16, dev)
    _check("beta", beta, (c,), torch.bfloat16, dev)
    _check("w1", w1, (c, 2 * f), torch.bfloat16, dev)
    _check("w2", w2, (f, c), torch.bfloat16, dev)
    return m, c, f, dev


def transition_fwd(x, gamma, beta, w1, w2, eps: float = 1e-5,
                   workspace: Optional[torch.Tensor] = None):
    """out = (silu(a) * b) @ w2 with [a | b] = layer_norm(x) * gamma + beta
    @ w1.  x [m, c] bf16, w1 [c, 2f], w2 [f, c].  Returns (out, mean, rstd)."""
    m, c, f, dev = _trn_common(x, gamma, beta, w1, w2)
    out = torch.empty_like(x)
    mean = torch.empty(m, dtype=torch.float32, device=dev)
    rstd = torch.empty(m, dtype=torch.float32, device=dev)
    need = tri_transition_fwd_workspace_bytes(BF16, m, c, f)
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    st = tri_transition_fwd(BF16, m, c, f, float(eps), _ptr(x), _ptr(gamma), _ptr(beta),
                            _ptr(w1), _ptr(w2), _ptr(out), _ptr(mean), _ptr(rstd),
                            _ptr(workspace), workspace.numel(), _stream(dev))
    if st != OK:
        raise TriAttnError(st, "tri_transition_fwd")
    return out, mean, rstd


def transition_bwd(x, gamma, beta, w1, w2, mean, rstd, dout,
                   workspace: Optional[torch.Tensor] = None):
    """Gradients of sum(dout * out) for transition_fwd.  Returns (dx [m, c]
    bf16, dw1 [c, 2f], dw2 [f, c], dgamma [c], dbeta [c], all fp32 but dx)."""
    m, c, f, dev = _trn_common(x, gamma, beta, w1, w2)
    _check("mean", mean, (m,), torch.float32, dev)
    _check("rstd", rstd, (m,), torch.float32, dev)
    _check("dout", dout, (m, c), torch.bfloat16, dev)
    dx = torch.empty_like(x)
    dw1 = torch.empty((c, 2 * f), dtype=torch.float32, device=dev)
    dw2 = torch.empty((f, c), dtype=torch.float32, device=dev)
    dgamma = torch.empty(c, dtype=torch.float32, device=dev)
    dbeta = torch.empty(c, dtype=torch.float32, device=dev)
    need = tri_transition_bwd_workspace_bytes(BF16, m, c, f)
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    st = tri_transition_bwd(BF16, m, c, f, _ptr(x), _ptr(gamma), _ptr(beta), _ptr(w1),
                            _ptr(w2), _ptr(mean), _ptr(rstd), _ptr(dout), _ptr(dx), _ptr(dw1),
                            _ptr(dw2), _ptr(dgamma), _ptr(dbeta), _ptr(workspace),
                            workspace.numel(), _stream(dev))
    if st != OK:
        raise TriAttnError(st, "tri_transition_bwd")
    return dx, dw1, dw2, dgamma, dbeta


# ---- layer norm, linear projection with epilogue, relative position bias -------------------
#
# Their smallest calls take the GPU less time than Python needs to make them, so the
# wrappers call the library's functions directly.

def _on(dev, fn, *args):
    """fn(*args, stream) on torch's current stream of `dev`, with `dev` current."""
    index = dev.index
    if index is not None and torch._C._cuda_getDevice() == index:
        return fn(*args, torch._C._cuda_getCurrentRawStream(index))
    with torch.cuda.device(dev):
        return fn(*args, _stream(dev))


def _workspace(workspace, need, dev):
    """The caller's workspace if it is large enough, else a new one."""
    if workspace is not None:
        if workspace.device != dev or workspace.dtype is not torch.uint8 or \
                not workspace.is_contiguous():
            raise ValueError(f"workspace must be a contiguous uint8 tensor on {dev}")
        if workspace.numel() >= need:
            return workspace
    return torch.empty(need, dtype=torch.uint8, device=dev)


def _check_2d(name, t):
    """t's dtype code, device and shape."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dim() != 2:
        raise ValueError(f"{name} must have two axes (got shape {tuple(t.shape)})")
    dt = _DTYPES.get(t.dtype)
    if dt is None:
        raise ValueError(f"unsupported dtype {t.dtype}")
    dev = t.device
    if dev.type != "cuda" or not t.is_contiguous():
        _check(name, t, t.shape, t.dtype, dev)
    m, n = t.shape
    return dt, dev, m, n


def layer_norm_fwd(x, gamma=None, beta=None, eps: float = 1e-5):
    """out = (x - mean) * rstd * gamma + beta over the rows of x [m, c] (fp32 or
    bf16; any c up to 8192); gamma and beta [c] may be None (ones, zeros).
    Returns (out, mean, rstd), the statistics [m] in fp32."""
    dt, dev, m, c = _check_2d("x", x)
    for name, t in (("gamma", gamma), ("beta", beta)):
        if t is not None:
            _check(name, t, (c,), x.dtype, dev)
    out = torch.empty_like(x)
    mean = torch.empty(m, dtype=torch.float32, device=dev)
    rstd = torch.empty(m, dtype=torch.float32, device=dev)
    st = _on(dev, lib().tri_layer_norm_fwd, dt, m, c, eps, x.data_ptr(), _ptr(gamma),
             _ptr(beta), out.data_ptr(), mean.data_ptr(), rstd.data_ptr())
    if st != OK:
        raise TriAttnError(st, "tri_layer_norm_fwd")
    return out, mean, rstd


def layer_norm_bwd(x, gamma, mean, rstd, dout, workspace: Optional[torch.Tensor] = None):
    """Gradients of sum(dout * out) for layer_norm_fwd.  Returns (dx [m, c],
    dgamma [c] fp32, dbeta [c] fp32)."""
    dt, dev, m, c = _check_2d("x", x)
    if gamma is not None:
        _check("gamma", gamma, (c,), x.dtype, dev)
    _check("mean", mean, (m,), torch.float32, dev)
    _check("rstd", rstd, (m,), torch.float32, dev)
    _check("dout", dout, (m, c), x.dtype, dev)
    dx = torch.empty_like(x)
    dgamma = torch.empty(c, dtype=torch.float32, device=dev)
    dbeta = torch.empty(c, dtype=torch.float32, device=dev)
    workspace = _workspace(workspace, tri_layer_norm_bwd_workspace_bytes(dt, m, c), dev)
    st = _on(dev, lib().tri_layer_norm_bwd, dt, m, c, x.data_ptr(), _ptr(gamma),
             mean.data_ptr(), rstd.data_ptr(), dout.data_ptr(), dx.data_ptr(), dgamma.data_ptr(),
             dbeta.data_ptr(), workspace.data_ptr(), workspace.numel())
    if st != OK:
        raise TriAttnError(st, "tri_layer_norm_bwd")
    return dx, dgamma, dbeta


def linear_fwd(x, w, bias=None, residual=None, act: int = ACT_NONE, save_z: bool = False):
    """out = act(x @ w + bias) + residual; x [m, k], w [k, n], bias [n] or None,
    residual [m, n] or None, all fp32 or all bf16; act one of ACT_NONE,
    ACT_RELU, ACT_GELU (error function), ACT_SILU.  Returns (out, z): z is the
    value before the activation, in x's dtype, if save_z (linear_bwd takes it
    when there is an activation), else None."""
    dt, dev, m, k = _check_2d("x", x)
    n = _check_2d("w", w)[3]
    dtype = x.dtype
    _check("w", w, (k, n), dtype, dev)
    if bias is not None:
        _check("bias", bias, (n,), dtype, dev)
    if residual is not None:
        _check("residual", residual, (m, n), dtype, dev)
    out = torch.empty((m, n), dtype=dtype, device=dev)
    z = torch.empty((m, n), dtype=dtype, device=dev) if save_z else None
    st = _on(dev, lib().tri_linear_fwd, dt, m, k, n, act, x.data_ptr(), w.data_ptr(),
             _ptr(bias), _ptr(residual), out.data_ptr(), _ptr(z))
    if st != OK:
        raise TriAttnError(st, "tri_linear_fwd")
    return out, z


def linear_bwd(x, w, dout, z=None, act: int = ACT_NONE,
               workspace: Optional[torch.Tensor] = None):
    """Gradients of sum(dout * out) for linear_fwd: z as it returned it (None
    without an activation).  Returns (dx [m, k] in x's dtype, dw [k, n] fp32,
    dbias [n] fp32); the residual's gradient is dout."""
    dt, dev, m, k = _check_2d("x", x)
    n = _check_2d("w", w)[3]
    dtype = x.dtype
    _check("w", w, (k, n), dtype, dev)
    _check("dout", dout, (m, n), dtype, dev)
    if z is not None:
        _check("z", z, (m, n), dtype, dev)
    dx = torch.empty_like(x)
    dw = torch.empty((k, n), dtype=torch.float32, device=dev)
    dbias = torch.empty(n, dtype=torch.float32, device=dev)
    workspace = _workspace(workspace, tri_linear_bwd_workspace_bytes(dt, m, k, n, act), dev)
    st = _on(dev, lib().tri_linear_bwd, dt, m, k, n, act, x.data_ptr(), w.data_ptr(), _ptr(z),
             dout.data_ptr(), dx.data_ptr(), dw.data_ptr(), dbias.data_ptr(),
             workspace.data_ptr(), workspace.numel())
    if st != OK:
        raise TriAttnError(st, "tri_linear_bwd")
    return dx, dw, dbias


def rel_bias_edges(exact: int, far: int = 0, steps: int = 0):
    """Ascending bucket borders for rel_bias_fwd, alike on both sides: the
    differences 1 - exact .. exact - 1 have buckets of their own, and beyond
    them `steps` buckets a side grow geometrically up to `far` (fewer where two
    borders would round to one); what is further shares the outermost bucket.
    With steps = 0, bucket i is the difference clipped to [-exact, exact],
    plus exact."""
    exact, far, steps = int(exact), int(far), int(steps)
    if exact < 1 or steps < 0 or (steps > 0 and far <= exact):
        raise ValueError("exact >= 1, steps >= 0 and, with steps, far > exact are needed")

    def border(i):
        """exact (far / exact)^(i / steps), rounded up; where it is an integer or close
        to one, whole numbers decide, which nothing rounds."""
        if i == steps:
            return far
        value = exact * (far / exact) ** (i / steps)
        near = round(value)
        if abs(value - near) > 1e-12 * value:
            return math.ceil(value)
        return near + (near ** steps < exact ** (steps - i) * far ** i)

    up = list(range(1, exact + 1)) + sorted({border(i + 1) for i in range(steps)})
    return [1 - e for e in reversed(up)] + up


def _rel_common(pos, chain, t, name):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype not in _DTYPES:
        raise ValueError(f"unsupported dtype {t.dtype}")
    if not isinstance(pos, torch.Tensor):
        raise TypeError("pos must be a torch.Tensor")
    if pos.dim() not in (1, 2):
        raise ValueError("pos must be [n] or [b, n]")
    dev = t.device
    _check("pos", pos, pos.shape, torch.int32, dev)
    if chain is not None:
        _check("chain", chain, pos.shape, torch.int32, dev)
    lead, n = tuple(pos.shape[:-1]), pos.shape[-1]
    return _DTYPES[t.dtype], lead, lead[0] if lead else 1, n, dev


def rel_bias_fwd(pos, edges, table, chain=None, base=None):
    """Relative position bias: out[q, k, :] = table[bucket][:] (+ base[q, k, :])
    with bucket the number of `edges` (ascending integers) at or below pos[q] -
    pos[k], or the table's last row where chain[q] != chain[k].  pos and chain
    [n] int32, table [len(edges) + 1 (+ 1 with chain), h] fp32 or bf16, base
    [n, n, h] or None.  Returns out [n, n, h], the layout of the attention's
    bias; with a leading batch axis on pos, chain and base, a batch."""
    dt, lead, batch, n, dev = _rel_common(pos, chain, table, "table")
    if table.dim() != 2:
        raise ValueError("table must be [rows, h]")
    h = table.shape[1]
    _check("table", table, (len(edges) + 1 + (chain is not None), h), table.dtype, dev)
    shape = lead + (n, n, h)
    if base is not None:
        _check("base", base, shape, table.dtype, dev)
    out = torch.empty(shape, dtype=table.dtype, device=dev)
    st = _on(dev, lib().tri_rel_bias_fwd, dt, batch, n, h, len(edges), _edges_arr(edges),
             pos.data_ptr(), _ptr(chain), table.data_ptr(), _ptr(base), out.data_ptr())
    if st != OK:
        raise TriAttnError(st, "tri_rel_bias_fwd")
    return out


def rel_bias_bwd(pos, edges, dout, chain=None, workspace: Optional[torch.Tensor] = None):
    """Gradient of sum(dout * out) for rel_bias_fwd: dout [n, n, h] (with a batch
    axis if pos has one).  Returns dtable [rows, h] fp32; base's gradient is
    dout."""
    dt, lead, batch, n, dev = _rel_common(pos, chain, dout, "dout")
    if dout.dim() != len(lead) + 3:
        raise ValueError("dout must be [n, n, h] ([b, n, n, h] with pos [b, n])")
    h = dout.shape[-1]
    _check("dout", dout, lead + (n, n, h), dout.dtype, dev)
    dtable = torch.empty((len(edges) + 1 + (chain is not None), h), dtype=torch.float32,
                         device=dev)
    need = tri_rel_bias_bwd_workspace_bytes(dt, batch, n, h, len(edges))
    workspace = _workspace(workspace, need, dev)
    st = _on(dev, lib().tri_rel_bias_bwd, dt, batch, n, h, len(edges), _edges_arr(edges),
             pos.data_ptr(), _ptr(chain), dout.data_ptr(), dtable.data_ptr(),
             workspace.data_ptr(), workspace.numel())
    if st != OK:
        raise TriAttnError(st, "tri_rel_bias_bwd")
    return dtable
