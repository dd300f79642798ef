"""ctypes binding of the sequence operators (include/seq_mi355x.h): short causal convolution, selective scan,
root-mean-square norm, products with 4-bit weights.

As ``conv``: argument marshalling only, no fallback.  A handle is created once for its sizes, types and strides; a call takes
the tensors.  Tensors of sequences are torch tensors [N, Cb, L, v], dense or not; give them (or tensors of the same strides) to
the create functions as ``views``, keyed by the argument's name, where they are not dense.  Calls check of each tensor what costs
next to nothing: its device, type and number of elements.
"""
from __future__ import annotations

import ctypes
import os  # noqa: F401

from . import conv
from .conv import ConvError  # noqa: F401  (what the calls raise)

SEQ_F32, SEQ_BF16, SEQ_I8 = 0, 1, 2

EXPORTS = (
    "seq_destroy", "seq_query", "seq_describe",
    "seq_conv_create", "seq_conv_fwd", "seq_conv_step", "seq_conv_bwd",
    "seq_scan_create", "seq_scan_fwd", "seq_scan_step", "seq_scan_bwd",
    "seq_norm_create", "seq_norm_fwd", "seq_norm_fwd_q8", "seq_norm_bwd",
    "seq_mv4_create", "seq_mv4", "seq_mv4_quant", "seq_mv4_unquant",
)


class SeqView(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("c", ctypes.c_int64), ("l", ctypes.c_int64)]


class SeqInfo(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("vlen", "Cb", "Cp", "reserved")] + \
               [(n, ctypes.c_size_t) for n in ("workspace_bytes", "state_bytes", "wt_bytes", "scale_bytes")]


def _desc(ints, views, floats=()):
    class Desc(ctypes.Structure):
        _fields_ = ([(n, ctypes.c_int32) for n in ints] + [(n, ctypes.c_float) for n in floats] + ([("reserved", ctypes.c_int32)]
                    if (len(ints) + len(floats)) % 2 else []) + [(n, SeqView) for n in views])
    return Desc


_CONV_VIEWS = ("x", "y", "dy", "dx")
_SCAN_VIEWS = ("x", "dt", "B", "C", "z", "y", "dy", "dx", "ddt", "dB", "dC", "dz")
_NORM_VIEWS = ("x", "res", "r", "y", "q", "dy", "dr", "dx")
SeqConvDesc = _desc(("N", "C", "L", "W", "silu", "slots", "dtype"), _CONV_VIEWS)
# (the descriptor has a number C and a view of the tensor C)
SeqScanDesc = _desc(("N", "Ch", "L", "S", "G", "softplus", "slots", "dtype"), _SCAN_VIEWS)
SeqNormDesc = _desc(("N", "C", "L", "dtype"), _NORM_VIEWS, ("eps",))
SeqMv4Desc = _desc(("M", "C", "K", "group", "dtype"), ())

_lib = None


def load():
    global _lib
    if _lib is None:
        lib = conv.load()
        vp, sz = ctypes.c_void_p, ctypes.c_size_t
        args = {"seq_destroy": [vp], "seq_query": [vp, vp], "seq_describe": [vp, ctypes.c_char_p, sz],
                "seq_conv_fwd": [vp] * 10, "seq_conv_step": [vp] * 8, "seq_conv_bwd": [vp] * 10 + [sz, vp],
                "seq_scan_fwd": [vp] * 15 + [sz, vp], "seq_scan_step": [vp] * 13, "seq_scan_bwd": [vp] * 20 + [sz, vp],
                "seq_norm_fwd": [vp] * 7, "seq_norm_fwd_q8": [vp] * 8, "seq_norm_bwd": [vp] * 8 + [sz, vp],
                "seq_mv4": [vp] * 8, "seq_mv4_quant": [vp] * 5, "seq_mv4_unquant": [vp] * 5}
        for name in EXPORTS:
            f = getattr(lib, name)
            f.argtypes = args.get(name, [vp, vp])
            f.restype = ctypes.c_int
        _lib = lib
    return _lib


class SeqPlan:
    """A handle, freed with the object, and what the calls check."""

    def __init__(self, create, desc, dtype, sizes):
        import torch
        self._h = ctypes.c_void_p()
        conv._check(getattr(load(), create)(ctypes.byref(desc), ctypes.byref(self._h)), create)
        self.info = SeqInfo()
        conv._check(load().seq_query(self._h, ctypes.byref(self.info)), "seq_query")
        self.kind = create[:-7]
        self.dtype = {SEQ_F32: torch.float32, SEQ_BF16: torch.bfloat16, SEQ_I8: torch.int8}[dtype]
        self.f32, self.i32, self.i8 = torch.float32, torch.int32, torch.int8
        self.__dict__.update(sizes)

    def close(self):
        if self._h:
            load().seq_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _t(x, dtype, least, name):
    """Device pointer of a tensor of `dtype` with at least `least` elements."""
    if x.dtype is not dtype or x.numel() < least or not x.is_cuda:
        raise ValueError("%s: a tensor of %s on the GPU with at least %d elements is wanted, not one of %s with %d on %s" % (
            name, dtype, least, x.dtype, x.numel(), x.device))
    return x.data_ptr()


def _o(x, dtype, least, name):
    return None if x is None else _t(x, dtype, least, name)


def _of(h, kind):
    if h.kind != kind:
        raise ValueError("a plan of %s is wanted, not one of %s" % (kind, h.kind))
    return h._h


def _views(views, names, desc, vlen, more=()):
    for name, t in (views or {}).items():
        if name not in names:
            continue
        v = 16 if name == "q" else vlen
        if t is None:
            continue
        if t.dim() != 4 or t.shape[3] != v or (t.stride(3) != 1 and v > 1):
            raise ValueError("%s: a tensor [N, Cb, L, %d] is wanted, its last dimension dense" % (name, v))
        # (a dimension of one place has any stride)
        setattr(desc, name, SeqView(*(t.stride(i) if t.shape[i] > 1 else v for i in range(3))))


def _vlen(dtype):
    return 4 if dtype == SEQ_F32 else 8


def seq_query(h) -> SeqInfo:
    return h.info


def seq_describe(h) -> str:
    buf = ctypes.create_string_buffer(512)
    conv._check(load().seq_describe(h._h, buf, 512), "seq_describe")
    return buf.value.decode()


def seq_destroy(h):
    h.close()


def seq_workspace(h, device="cuda"):
    """A workspace for all passes of a plan, or None where none needs one."""
    import torch
    n = h.info.workspace_bytes
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def _ws(ws):
    return (None, 0) if ws is None else (ws.data_ptr(), ws.numel() * ws.element_size())


# ---------------------------------------------------------------------------- short convolution
def seq_conv_create(N, C, L, W, dtype=SEQ_F32, silu=True, slots=0, views=None) -> SeqPlan:
    d = SeqConvDesc(N=N, C=C, L=L, W=W, silu=1 if silu else 0, slots=slots, dtype=dtype)
    _views(views, _CONV_VIEWS, d, _vlen(dtype))
    h = SeqPlan("seq_conv_create", d, dtype, {"N": N})
    h.rows, h.all = N * h.info.Cp, N * h.info.Cp * L
    h.w, h.state = W * h.info.Cp, slots * h.info.Cp * (W - 1)
    return h


def seq_conv_fwd(h, x, w, bias, y, state_in=None, state_out=None, slots=None, lengths=None, stream=None):
    T = h.dtype
    conv._check(load().seq_conv_fwd(
        _of(h, "seq_conv"), _t(x, T, h.all, "x"), _t(w, h.f32, h.w, "w"), _o(bias, h.f32, h.info.Cp, "bias"), _o(state_in, T, h.state, "state_in"),
        _t(y, T, h.all, "y"), _o(state_out, T, h.state, "state_out"), _o(slots, h.i32, h.N, "slots"), _o(lengths, h.i32, h.N, "lengths"),
        conv._stream(stream)), "seq_conv_fwd")


def seq_conv_step(h, x, w, bias, state, y, slots=None, stream=None):
    T = h.dtype
    conv._check(load().seq_conv_step(
        _of(h, "seq_conv"), _t(x, T, h.rows, "x"), _t(w, h.f32, h.w, "w"), _o(bias, h.f32, h.info.Cp, "bias"), _t(state, T, h.state, "state"),
        _t(y, T, h.rows, "y"), _o(slots, h.i32, h.N, "slots"), conv._stream(stream)), "seq_conv_step")


def seq_conv_bwd(h, x, w, bias, dy, dx, dw, dbias, ws, lengths=None, stream=None):
    T = h.dtype
    conv._check(load().seq_conv_bwd(
        _of(h, "seq_conv"), _t(x, T, h.all, "x"), _t(w, h.f32, h.w, "w"), _o(bias, h.f32, h.info.Cp, "bias"), _t(dy, T, h.all, "dy"),
        _t(dx, T, h.all, "dx"), _t(dw, h.f32, h.w, "dw"), _o(dbias, h.f32, h.info.Cp, "dbias"), _o(lengths, h.i32, h.N, "lengths"),
        *_ws(ws), conv._stream(stream)), "seq_conv_bwd")


# ---------------------------------------------------------------------------- selective scan
def seq_scan_create(N, C, L, S, dtype=SEQ_F32, G=1, softplus=True, slots=0, views=None) -> SeqPlan:
    d = SeqScanDesc(N=N, Ch=C, L=L, S=S, G=G, softplus=1 if softplus else 0, slots=slots, dtype=dtype)
    _views(views, _SCAN_VIEWS, d, _vlen(dtype))
    h = SeqPlan("seq_scan_create", d, dtype, {"N": N})
    h.rows, h.all = N * h.info.Cp, N * h.info.Cp * L
    v = h.info.vlen
    h.srows, h.A, h.state = N * -(-G * S // v) * v, S * h.info.Cp, slots * S * h.info.Cp
    h.sall = h.srows * L
    return h


def _scan_inputs(h, T, x, dt, A, B, C, D, z, dt_bias, rows, srows):
    f, Cp = h.f32, h.info.Cp
    return (_t(x, T, rows, "x"), _t(dt, T, rows, "dt"), _t(A, f, h.A, "A"), _t(B, T, srows, "B"), _t(C, T, srows, "C"), _o(D, f, Cp, "D"),
            _o(z, T, rows, "z"), _o(dt_bias, f, Cp, "dt_bias"))


def seq_scan_fwd(h, x, dt, A, B, C, y, ws=None, D=None, z=None, dt_bias=None, state_in=None, state_out=None, slots=None, lengths=None,
                 stream=None):
    T = h.dtype
    conv._check(load().seq_scan_fwd(
        _of(h, "seq_scan"), *_scan_inputs(h, T, x, dt, A, B, C, D, z, dt_bias, h.all, h.sall), _o(state_in, h.f32, h.state, "state_in"),
        _t(y, T, h.all, "y"), _o(state_out, h.f32, h.state, "state_out"), _o(slots, h.i32, h.N, "slots"), _o(lengths, h.i32, h.N, "lengths"),
        *_ws(ws), conv._stream(stream)), "seq_scan_fwd")


def seq_scan_step(h, x, dt, A, B, C, state, y, D=None, z=None, dt_bias=None, slots=None, stream=None):
    T = h.dtype
    conv._check(load().seq_scan_step(
        _of(h, "seq_scan"), *_scan_inputs(h, T, x, dt, A, B, C, D, z, dt_bias, h.rows, h.srows), _t(state, h.f32, h.state, "state"),
        _t(y, T, h.rows, "y"), _o(slots, h.i32, h.N, "slots"), conv._stream(stream)), "seq_scan_step")


def seq_scan_bwd(h, x, dt, A, B, C, dy, dx, ddt, dA, dB, dC, ws, D=None, z=None, dt_bias=None, dD=None, dz=None, ddt_bias=None, lengths=None,
                 stream=None):
    T, f, Cp = h.dtype, h.f32, h.info.Cp
    conv._check(load().seq_scan_bwd(
        _of(h, "seq_scan"), *_scan_inputs(h, T, x, dt, A, B, C, D, z, dt_bias, h.all, h.sall), _t(dy, T, h.all, "dy"), _t(dx, T, h.all, "dx"),
        _t(ddt, T, h.all, "ddt"), _t(dA, f, h.A, "dA"), _t(dB, T, h.sall, "dB"), _t(dC, T, h.sall, "dC"), _o(dD, f, Cp, "dD"), _o(dz, T, h.all, "dz"),
        _o(ddt_bias, f, Cp, "ddt_bias"), _o(lengths, h.i32, h.N, "lengths"), *_ws(ws), conv._stream(stream)), "seq_scan_bwd")


# ---------------------------------------------------------------------------- norm
def seq_norm_create(N, C, L, dtype=SEQ_F32, eps=1e-5, views=None) -> SeqPlan:
    d = SeqNormDesc(N=N, C=C, L=L, dtype=dtype, eps=eps)
    _views(views, _NORM_VIEWS, d, _vlen(dtype))
    h = SeqPlan("seq_norm_create", d, dtype, {"N": N, "positions": N * L})
    h.all, h.q = N * h.info.Cp * L, N * L * (-(-C // 16) * 16)
    return h


def seq_norm_fwd(h, x, res, w, r, y, stream=None):
    T, n = h.dtype, h.all
    conv._check(load().seq_norm_fwd(_of(h, "seq_norm"), _t(x, T, n, "x"), _o(res, T, n, "res"), _t(w, h.f32, h.info.Cp, "w"), _o(r, T, n, "r"),
                                    _t(y, T, n, "y"), conv._stream(stream)), "seq_norm_fwd")


def seq_norm_fwd_q8(h, x, res, w, r, q, scale, stream=None):
    T, n = h.dtype, h.all
    conv._check(load().seq_norm_fwd_q8(_of(h, "seq_norm"), _t(x, T, n, "x"), _o(res, T, n, "res"), _t(w, h.f32, h.info.Cp, "w"), _o(r, T, n, "r"),
                                       _t(q, h.i8, h.q, "q"), _t(scale, h.f32, h.positions, "scale"), conv._stream(stream)), "seq_norm_fwd_q8")


def seq_norm_bwd(h, r, w, dy, dr, dx, dw, ws, stream=None):
    T, n = h.dtype, h.all
    conv._check(load().seq_norm_bwd(_of(h, "seq_norm"), _t(r, T, n, "r"), _t(w, h.f32, h.info.Cp, "w"), _t(dy, T, n, "dy"), _o(dr, T, n, "dr"),
                                    _t(dx, T, n, "dx"), _t(dw, h.f32, h.info.Cp, "dw"), *_ws(ws), conv._stream(stream)), "seq_norm_bwd")


# ---------------------------------------------------------------------------- products with 4-bit weights
def seq_mv4_create(M, C, K, group, dtype=SEQ_BF16) -> SeqPlan:
    import torch
    h = SeqPlan("seq_mv4_create", SeqMv4Desc(M=M, C=C, K=K, group=group, dtype=dtype), dtype, {"M": M, "K": K, "C": C})
    v = 4 if dtype == SEQ_F32 else 8
    h.x, h.y, h.ydtype = M * h.info.Cp, M * (-(-K // v) * v), torch.float32 if dtype == SEQ_F32 else torch.bfloat16
    h.u8, h.scales = torch.uint8, h.info.scale_bytes // 4
    return h


def seq_mv4(h, x, wt, scale, y, xscale=None, bias=None, stream=None):
    conv._check(load().seq_mv4(_of(h, "seq_mv4"), _t(x, h.dtype, h.x, "x"), _o(xscale, h.f32, h.M, "xscale"), _t(wt, h.u8, h.info.wt_bytes, "wt"),
                               _t(scale, h.f32, h.scales, "scale"), _o(bias, h.f32, h.K, "bias"), _t(y, h.ydtype, h.y, "y"), conv._stream(stream)),
                "seq_mv4")


def seq_mv4_quant(h, w, wt, scale, stream=None):
    """w: fp32 [K, C], dense."""
    if not w.is_contiguous():
        raise ValueError("w: a dense tensor is wanted")
    conv._check(load().seq_mv4_quant(_of(h, "seq_mv4"), _t(w, h.f32, h.K * h.C, "w"), _t(wt, h.u8, h.info.wt_bytes, "wt"),
                                     _t(scale, h.f32, h.scales, "scale"), conv._stream(stream)), "seq_mv4_quant")


def seq_mv4_unquant(h, wt, scale, w, stream=None):
    if not w.is_contiguous():
        raise ValueError("w: a dense tensor is wanted")
    conv._check(load().seq_mv4_unquant(_of(h, "seq_mv4"), _t(wt, h.u8, h.info.wt_bytes, "wt"), _t(scale, h.f32, h.scales, "scale"),
                                       _t(w, h.f32, h.K * h.C, "w"), conv._stream(stream)), "seq_mv4_unquant")
