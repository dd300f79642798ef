"""ctypes binding of the sequence operators (include/seq_mi355x.h): short causal convolution, selective scan,
root-mean-square norm, products with 4-bit weights.

As ``conv``: argument marshalling only, no fallback.  A handle is created once for its sizes, types and strides; a call takes
the tensors.  Tensors of sequences are torch tensors [N, Cb, L, v], dense or not; give them (or tensors of the same strides) to
the create functions as ``views``, keyed by the argument's name, where they are not dense.  Calls check each tensor's device, type,
extents and strides against the plan's, so that a tensor of another layout is refused rather than read past its end.
"""
from __future__ import annotations

import ctypes
import math

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


def _s(h, name, x):
    """Device pointer of a sequence tensor that is as the plan has it."""
    if x.dtype is not h.dtype or x.shape != h.shapes[name] or not x.is_cuda or x.stride() != h.strides[name]:
        _misfit(h, name, x, h.dtype)
    return x.data_ptr()


def _so(h, name, x):
    return None if x is None else _s(h, name, x)


def _misfit(h, name, x, dtype):
    """What _s found may be more places than there are, the stride of a dimension of one place, or a dense tensor of other dimensions."""
    shape, strides = h.shapes[name], h.strides[name]
    if x.dtype is dtype and x.is_cuda:
        if x.dim() == 4 and all(x.shape[i] >= shape[i] and (shape[i] == 1 or x.stride(i) == strides[i]) for i in range(4)):
            return
        one_after_the_other = x.dim() != 4 or all(x.shape[i] == 1 or x.stride(i) == strides[i] for i in range(4))
        if one_after_the_other and x.is_contiguous() and strides == h.dense[name] and x.numel() >= math.prod(shape):
            return
    raise ValueError("%s: a tensor %s of %s on the GPU with strides %s is wanted, not one of %s of %s with %s on %s" % (
        name, list(shape), dtype, strides, tuple(x.shape), x.dtype, tuple(x.stride()), x.device))


def _t(x, dtype, least, name):
    """Device pointer of a dense tensor of `dtype` with at least `least` elements."""
    if x.dtype is not dtype or x.numel() < least or not x.is_cuda or not x.is_contiguous():
        raise ValueError("%s: a dense tensor of %s on the GPU with at least %d elements is wanted, not one of %s with %d and strides %s on %s" % (
            name, dtype, least, x.dtype, x.numel(), tuple(x.stride()), x.device))
    return x.data_ptr()


def _o(x, dtype, least, name):
    return None if x is None else _t(x, dtype, least, name)


def _of(h, kind):
    if h.kind != kind:
        raise ValueError("a plan of %s is wanted, not one of %s" % (kind, h.kind))
    return h._h


def _strides(h, names, views, N, C, L, wide=()):
    """The extents and strides of each sequence tensor of a plan, given or dense; `wide`: channels of those that have others than C."""
    h.dense, h.strides, h.shapes = {}, {}, {}
    for name in names:
        v = 16 if name == "q" else h.info.vlen
        Cb = -(-dict(wide).get(name, C) // v)
        h.dense[name], h.shapes[name] = (Cb * L * v, L * v, v, 1), (N, Cb, L, v)
        t = (views or {}).get(name)
        h.strides[name] = h.dense[name] if t is None else tuple(t.stride())


def _views(views, names, desc, vlen, N, C, L, wide=()):
    for name, t in (views or {}).items():
        if name not in names:
            continue
        v = 16 if name == "q" else vlen
        if t is None:
            continue
        if t.dim() != 4 or t.shape[3] != v or (t.stride(3) != 1 and v > 1):
            raise ValueError("%s: a tensor [N, Cb, L, %d] is wanted, its last dimension dense" % (name, v))
        extents = (N, -(-dict(wide).get(name, C) // v), L)
        if any(t.shape[i] == 1 < extents[i] for i in range(3)):
            raise ValueError("%s: a tensor of %s does not give the strides of one of %s" % (name, tuple(t.shape), (*extents, v)))
        # (a dimension of one place has any stride)
        strides = [t.stride(i) if t.shape[i] > 1 else v for i in range(3)]
        if not any(strides):  # (which would mean a dense tensor)
            raise ValueError("%s: one block for all places" % name)
        setattr(desc, name, SeqView(*strides))


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
    if ws is None:
        return None, 0
    if not ws.is_cuda or not ws.is_contiguous():
        raise ValueError("ws: a dense tensor on the GPU is wanted, not one with strides %s on %s" % (tuple(ws.stride()), ws.device))
    return ws.data_ptr(), ws.numel() * ws.element_size()


# ---------------------------------------------------------------------------- short convolution
def seq_conv_create(N, C, L, W, dtype=SEQ_F32, silu=True, slots=0, views=None) -> SeqPlan:
    d = SeqConvDesc(N=N, C=C, L=L, W=W, silu=1 if silu else 0, slots=slots, dtype=dtype)
    _views(views, _CONV_VIEWS, d, _vlen(dtype), N, C, L)
    h = SeqPlan("seq_conv_create", d, dtype, {"N": N})
    _strides(h, _CONV_VIEWS, views, N, C, L)
    h.w, h.state = W * h.info.Cp, slots * h.info.Cp * (W - 1)
    return h


def seq_conv_fwd(h, x, w, bias, y, state_in=None, state_out=None, slots=None, lengths=None, stream=None):
    T = h.dtype
    conv._check(load().seq_conv_fwd(
        _of(h, "seq_conv"), _s(h, "x", x), _t(w, h.f32, h.w, "w"), _o(bias, h.f32, h.info.Cp, "bias"), _o(state_in, T, h.state, "state_in"),
        _s(h, "y", y), _o(state_out, T, h.state, "state_out"), _o(slots, h.i32, h.N, "slots"), _o(lengths, h.i32, h.N, "lengths"),
        conv._stream(stream)), "seq_conv_fwd")


def seq_conv_step(h, x, w, bias, state, y, slots=None, stream=None):
    T = h.dtype
    conv._check(load().seq_conv_step(
        _of(h, "seq_conv"), _s(h, "x", x), _t(w, h.f32, h.w, "w"), _o(bias, h.f32, h.info.Cp, "bias"), _t(state, T, h.state, "state"),
        _s(h, "y", y), _o(slots, h.i32, h.N, "slots"), conv._stream(stream)), "seq_conv_step")


def seq_conv_bwd(h, x, w, bias, dy, dx, dw, dbias, ws, lengths=None, stream=None):
    conv._check(load().seq_conv_bwd(
        _of(h, "seq_conv"), _s(h, "x", x), _t(w, h.f32, h.w, "w"), _o(bias, h.f32, h.info.Cp, "bias"), _s(h, "dy", dy),
        _s(h, "dx", dx), _t(dw, h.f32, h.w, "dw"), _o(dbias, h.f32, h.info.Cp, "dbias"), _o(lengths, h.i32, h.N, "lengths"),
        *_ws(ws), conv._stream(stream)), "seq_conv_bwd")


# ---------------------------------------------------------------------------- selective scan
def seq_scan_create(N, C, L, S, dtype=SEQ_F32, G=1, softplus=True, slots=0, views=None) -> SeqPlan:
    d = SeqScanDesc(N=N, Ch=C, L=L, S=S, G=G, softplus=1 if softplus else 0, slots=slots, dtype=dtype)
    wide = [(k, G * S) for k in ("B", "C", "dB", "dC")]
    _views(views, _SCAN_VIEWS, d, _vlen(dtype), N, C, L, wide)
    h = SeqPlan("seq_scan_create", d, dtype, {"N": N})
    _strides(h, _SCAN_VIEWS, views, N, C, L, wide)
    h.A, h.state = S * h.info.Cp, slots * S * h.info.Cp
    return h


def _scan_inputs(h, x, dt, A, B, C, D, z, dt_bias):
    f, Cp = h.f32, h.info.Cp
    return (_s(h, "x", x), _s(h, "dt", dt), _t(A, f, h.A, "A"), _s(h, "B", B), _s(h, "C", C), _o(D, f, Cp, "D"),
            _so(h, "z", z), _o(dt_bias, f, Cp, "dt_bias"))


def seq_scan_fwd(h, x, dt, A, B, C, y, ws=None, D=None, z=None, dt_bias=None, state_in=None, state_out=None, slots=None, lengths=None,
                 stream=None):
    conv._check(load().seq_scan_fwd(
        _of(h, "seq_scan"), *_scan_inputs(h, x, dt, A, B, C, D, z, dt_bias), _o(state_in, h.f32, h.state, "state_in"),
        _s(h, "y", y), _o(state_out, h.f32, h.state, "state_out"), _o(slots, h.i32, h.N, "slots"), _o(lengths, h.i32, h.N, "lengths"),
        *_ws(ws), conv._stream(stream)), "seq_scan_fwd")


def seq_scan_step(h, x, dt, A, B, C, state, y, D=None, z=None, dt_bias=None, slots=None, stream=None):
    conv._check(load().seq_scan_step(
        _of(h, "seq_scan"), *_scan_inputs(h, x, dt, A, B, C, D, z, dt_bias), _t(state, h.f32, h.state, "state"),
        _s(h, "y", y), _o(slots, h.i32, h.N, "slots"), conv._stream(stream)), "seq_scan_step")


def seq_scan_bwd(h, x, dt, A, B, C, dy, dx, ddt, dA, dB, dC, ws, D=None, z=None, dt_bias=None, dD=None, dz=None, ddt_bias=None, lengths=None,
                 stream=None):
    f, Cp = h.f32, h.info.Cp
    conv._check(load().seq_scan_bwd(
        _of(h, "seq_scan"), *_scan_inputs(h, x, dt, A, B, C, D, z, dt_bias), _s(h, "dy", dy), _s(h, "dx", dx),
        _s(h, "ddt", ddt), _t(dA, f, h.A, "dA"), _s(h, "dB", dB), _s(h, "dC", dC), _o(dD, f, Cp, "dD"), _so(h, "dz", dz),
        _o(ddt_bias, f, Cp, "ddt_bias"), _o(lengths, h.i32, h.N, "lengths"), *_ws(ws), conv._stream(stream)), "seq_scan_bwd")


# ---------------------------------------------------------------------------- norm
def seq_norm_create(N, C, L, dtype=SEQ_F32, eps=1e-5, views=None) -> SeqPlan:
    d = SeqNormDesc(N=N, C=C, L=L, dtype=dtype, eps=eps)
    _views(views, _NORM_VIEWS, d, _vlen(dtype), N, C, L)
    h = SeqPlan("seq_norm_create", d, dtype, {"N": N, "positions": N * L})
    _strides(h, _NORM_VIEWS, views, N, C, L)
    return h


def seq_norm_fwd(h, x, res, w, r, y, stream=None):
    conv._check(load().seq_norm_fwd(_of(h, "seq_norm"), _s(h, "x", x), _so(h, "res", res), _t(w, h.f32, h.info.Cp, "w"), _so(h, "r", r),
                                    _s(h, "y", y), conv._stream(stream)), "seq_norm_fwd")


def _q(h, q):
    if q.dtype is not h.i8 or q.shape != h.shapes["q"] or not q.is_cuda or q.stride() != h.strides["q"]:
        _misfit(h, "q", q, h.i8)
    return q.data_ptr()


def seq_norm_fwd_q8(h, x, res, w, r, q, scale, stream=None):
    conv._check(load().seq_norm_fwd_q8(_of(h, "seq_norm"), _s(h, "x", x), _so(h, "res", res), _t(w, h.f32, h.info.Cp, "w"), _so(h, "r", r),
                                       _q(h, q), _t(scale, h.f32, h.positions, "scale"), conv._stream(stream)), "seq_norm_fwd_q8")


def seq_norm_bwd(h, r, w, dy, dr, dx, dw, ws, stream=None):
    conv._check(load().seq_norm_bwd(_of(h, "seq_norm"), _s(h, "r", r), _t(w, h.f32, h.info.Cp, "w"), _s(h, "dy", dy), _so(h, "dr", dr),
                                    _s(h, "dx", dx), _t(dw, h.f32, h.info.Cp, "dw"), *_ws(ws), conv._stream(stream)), "seq_norm_bwd")


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
    """w: fp32 [K, C]."""
    conv._check(load().seq_mv4_quant(_of(h, "seq_mv4"), _t(w, h.f32, h.K * h.C, "w"), _t(wt, h.u8, h.info.wt_bytes, "wt"),
                                     _t(scale, h.f32, h.scales, "scale"), conv._stream(stream)), "seq_mv4_quant")


def seq_mv4_unquant(h, wt, scale, w, stream=None):
    conv._check(load().seq_mv4_unquant(_of(h, "seq_mv4"), _t(wt, h.u8, h.info.wt_bytes, "wt"), _t(scale, h.f32, h.scales, "scale"),
                                       _t(w, h.f32, h.K * h.C, "w"), conv._stream(stream)), "seq_mv4_unquant")
