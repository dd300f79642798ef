"""ctypes binding of the sequence operators (include/seq_mi355x.h): short causal convolution, selective scan, gated linear recurrence,
root-mean-square norm, layer norm, products with 4-bit weights, AdamW.

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
    "seq_rec_create", "seq_rec_fwd", "seq_rec_step", "seq_rec_bwd",
    "seq_norm_create", "seq_norm_fwd", "seq_norm_fwd_q8", "seq_norm_bwd",
    "seq_lnorm_create", "seq_lnorm_fwd", "seq_lnorm_fwd_q8", "seq_lnorm_bwd",
    "seq_adamw_create", "seq_adamw",
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
_REC_VIEWS = ("x", "f", "i", "z", "y", "dy", "dx", "df", "di", "dz")
_NORM_VIEWS = ("x", "res", "r", "y", "q", "dy", "dr", "dx")
SeqConvDesc = _desc(("N", "C", "L", "W", "silu", "slots", "dtype"), _CONV_VIEWS)
# (the descriptor has a number C and a view of the tensor C)
SeqScanDesc = _desc(("N", "Ch", "L", "S", "G", "softplus", "slots", "dtype"), _SCAN_VIEWS)
SeqRecDesc = _desc(("N", "C", "L", "slots", "dtype"), _REC_VIEWS)
SeqNormDesc = _desc(("N", "C", "L", "dtype"), _NORM_VIEWS, ("eps",))
SeqMv4Desc = _desc(("M", "C", "K", "group", "dtype"), ())


class SeqAdamwDesc(ctypes.Structure):
    _fields_ = [("sizes", ctypes.c_void_p), ("decays", ctypes.c_void_p)] + [(n, ctypes.c_double) for n in ("beta1", "beta2", "eps")] + \
               [(n, ctypes.c_int32) for n in ("count", "bits", "dtype", "reserved")]


_lib = None


def load():
    global _lib
    if _lib is None:
        lib = conv.load()
        vp, sz = ctypes.c_void_p, ctypes.c_size_t
        args = {"seq_destroy": [vp], "seq_query": [vp, vp], "seq_describe": [vp, ctypes.c_char_p, sz],
                "seq_conv_fwd": [vp] * 10, "seq_conv_step": [vp] * 8, "seq_conv_bwd": [vp] * 10 + [sz, vp],
                "seq_scan_fwd": [vp] * 15 + [sz, vp], "seq_scan_step": [vp] * 13, "seq_scan_bwd": [vp] * 20 + [sz, vp],
                "seq_rec_fwd": [vp] * 14 + [sz, vp], "seq_rec_step": [vp] * 12, "seq_rec_bwd": [vp] * 18 + [sz, vp],
                "seq_lnorm_fwd": [vp] * 9, "seq_lnorm_fwd_q8": [vp] * 10, "seq_lnorm_bwd": [vp] * 10 + [sz, vp], "seq_adamw": [vp] * 10,
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


_device = None  # the current device's number, once a tensor on one is there


def _here(*tensors):
    """Refuses tensors of different devices, or of another one than the current one, on which the library's calls run."""
    global _device
    at = None
    for x in tensors:
        if x is not None:
            d = x.get_device()
            if at is None:
                at = d
            elif d != at:
                raise ValueError("tensors on one device are wanted, not on %s and %s" % (at, d))
    if at is None or at < 0:
        return
    if _device is None:
        import torch
        torch.cuda.current_device()  # (initialises the runtime if need be)
        _device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    if at != _device():
        raise ValueError("tensors on the current device (%d) are wanted, not on %d" % (_device(), at))


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


# ---------------------------------------------------------------------------- gated linear recurrence
def seq_rec_create(N, C, L, dtype=SEQ_F32, slots=0, views=None) -> SeqPlan:
    d = SeqRecDesc(N=N, C=C, L=L, slots=slots, dtype=dtype)
    _views(views, _REC_VIEWS, d, _vlen(dtype), N, C, L)
    h = SeqPlan("seq_rec_create", d, dtype, {"N": N})
    _strides(h, _REC_VIEWS, views, N, C, L)
    h.state = slots * h.info.Cp
    return h


def _rec_inputs(h, x, f, i, A, z, f_bias, i_bias):
    t, Cp = h.f32, h.info.Cp
    return (_s(h, "x", x), _s(h, "f", f), _s(h, "i", i), _t(A, t, Cp, "A"), _so(h, "z", z), _o(f_bias, t, Cp, "f_bias"), _o(i_bias, t, Cp, "i_bias"))


def seq_rec_fwd(h, x, f, i, A, y, ws=None, z=None, f_bias=None, i_bias=None, state_in=None, state_out=None, slots=None, lengths=None, stream=None):
    _here(x, f, i, A, y, ws, z, f_bias, i_bias, state_in, state_out, slots, lengths)
    conv._check(load().seq_rec_fwd(
        _of(h, "seq_rec"), *_rec_inputs(h, x, f, i, A, z, f_bias, i_bias), _o(state_in, h.f32, h.state, "state_in"), _s(h, "y", y),
        _o(state_out, h.f32, h.state, "state_out"), _o(slots, h.i32, h.N, "slots"), _o(lengths, h.i32, h.N, "lengths"), *_ws(ws),
        conv._stream(stream)), "seq_rec_fwd")


def seq_rec_step(h, x, f, i, A, state, y, z=None, f_bias=None, i_bias=None, slots=None, stream=None):
    _here(x, f, i, A, state, y, z, f_bias, i_bias, slots)
    conv._check(load().seq_rec_step(
        _of(h, "seq_rec"), *_rec_inputs(h, x, f, i, A, z, f_bias, i_bias), _t(state, h.f32, h.state, "state"), _s(h, "y", y),
        _o(slots, h.i32, h.N, "slots"), conv._stream(stream)), "seq_rec_step")


def seq_rec_bwd(h, x, f, i, A, dy, dx, df, di, dA, ws, z=None, f_bias=None, i_bias=None, dz=None, df_bias=None, di_bias=None, lengths=None, stream=None):
    _here(x, f, i, A, dy, dx, df, di, dA, ws, z, f_bias, i_bias, dz, df_bias, di_bias, lengths)
    t, Cp = h.f32, h.info.Cp
    conv._check(load().seq_rec_bwd(
        _of(h, "seq_rec"), *_rec_inputs(h, x, f, i, A, z, f_bias, i_bias), _s(h, "dy", dy), _s(h, "dx", dx), _s(h, "df", df), _s(h, "di", di),
        _t(dA, t, Cp, "dA"), _so(h, "dz", dz), _o(df_bias, t, Cp, "df_bias"), _o(di_bias, t, Cp, "di_bias"), _o(lengths, h.i32, h.N, "lengths"),
        *_ws(ws), conv._stream(stream)), "seq_rec_bwd")


# ---------------------------------------------------------------------------- norm
def _norm_create(kind, N, C, L, dtype, eps, views):
    d = SeqNormDesc(N=N, C=C, L=L, dtype=dtype, eps=eps)
    _views(views, _NORM_VIEWS, d, _vlen(dtype), N, C, L)
    h = SeqPlan(kind, d, dtype, {"N": N, "positions": N * L})
    _strides(h, _NORM_VIEWS, views, N, C, L)
    return h


def seq_norm_create(N, C, L, dtype=SEQ_F32, eps=1e-5, views=None) -> SeqPlan:
    return _norm_create("seq_norm_create", N, C, L, dtype, eps, views)


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


# ---------------------------------------------------------------------------- layer norm
def seq_lnorm_create(N, C, L, dtype=SEQ_F32, eps=1e-5, views=None) -> SeqPlan:
    return _norm_create("seq_lnorm_create", N, C, L, dtype, eps, views)


def _lnorm_inputs(h, x, res, w, b, r):
    return (_s(h, "x", x), _so(h, "res", res), _t(w, h.f32, h.info.Cp, "w"), _o(b, h.f32, h.info.Cp, "b"), _so(h, "r", r))


def seq_lnorm_fwd(h, x, res, w, b, r, y, lengths=None, stream=None):
    _here(x, res, w, b, r, y, lengths)
    conv._check(load().seq_lnorm_fwd(_of(h, "seq_lnorm"), *_lnorm_inputs(h, x, res, w, b, r), _s(h, "y", y), _o(lengths, h.i32, h.N, "lengths"),
                                     conv._stream(stream)), "seq_lnorm_fwd")


def seq_lnorm_fwd_q8(h, x, res, w, b, r, q, scale, lengths=None, stream=None):
    _here(x, res, w, b, r, q, scale, lengths)
    conv._check(load().seq_lnorm_fwd_q8(_of(h, "seq_lnorm"), *_lnorm_inputs(h, x, res, w, b, r), _q(h, q), _t(scale, h.f32, h.positions, "scale"),
                                        _o(lengths, h.i32, h.N, "lengths"), conv._stream(stream)), "seq_lnorm_fwd_q8")


def seq_lnorm_bwd(h, r, w, dy, dr, dx, dw, db, ws, lengths=None, stream=None):
    _here(r, w, dy, dr, dx, dw, db, ws, lengths)
    conv._check(load().seq_lnorm_bwd(_of(h, "seq_lnorm"), _s(h, "r", r), _t(w, h.f32, h.info.Cp, "w"), _s(h, "dy", dy), _so(h, "dr", dr),
                                     _s(h, "dx", dx), _t(dw, h.f32, h.info.Cp, "dw"), _o(db, h.f32, h.info.Cp, "db"),
                                     _o(lengths, h.i32, h.N, "lengths"), *_ws(ws), conv._stream(stream)), "seq_lnorm_bwd")


# ---------------------------------------------------------------------------- AdamW
def seq_adamw_create(sizes, dtype=SEQ_F32, bits=32, betas=(0.9, 0.999), eps=1e-8, decay=0.01) -> SeqPlan:
    """sizes: numbers of each tensor; dtype: of the gradients; bits: of the states, 32 or 8; decay: one for all tensors, or one for each."""
    import torch
    sizes = [int(n) for n in sizes]
    decays = [float(decay)] * len(sizes) if isinstance(decay, (int, float)) else [float(d) for d in decay]
    if len(decays) != len(sizes):
        raise ValueError("decay: one for each of %d tensors is wanted, not %d" % (len(sizes), len(decays)))
    a, b = (ctypes.c_int64 * len(sizes))(*sizes), (ctypes.c_double * len(sizes))(*decays)
    d = SeqAdamwDesc(sizes=ctypes.addressof(a), decays=ctypes.addressof(b), beta1=betas[0], beta2=betas[1], eps=eps, count=len(sizes), bits=bits, dtype=dtype)
    h = SeqPlan("seq_adamw_create", d, dtype, {"sizes": sizes, "bits": bits})
    h.state, h.scales = h.info.state_bytes * 8 // bits, h.info.scale_bytes // 4
    h.mdtype, h.vdtype = (torch.float32, torch.float32) if bits == 32 else (torch.int8, torch.uint8)
    h.bf16 = torch.bfloat16
    return h


def seq_adamw_states(h, device="cuda"):
    """Fresh states for a plan: m, v and, for 8 bits, their scales."""
    import torch
    _of(h, "seq_adamw")
    return (torch.zeros(h.state, dtype=h.mdtype, device=device), torch.zeros(h.state, dtype=h.vdtype, device=device),
            torch.zeros(h.scales, device=device) if h.bits == 8 else None)


class SeqAdamwTensors:
    """Parameters, their gradients and copies for a plan's calls, checked once.  Holds the memory that they have then."""

    def __init__(self, h, p, g, copies=None):
        _of(h, "seq_adamw")
        lists = [list(p), list(g), [None] * len(h.sizes) if copies is None else list(copies)]
        if any(len(x) != len(h.sizes) for x in lists):
            raise ValueError("lists of %d tensors are wanted, not of %s" % (len(h.sizes), ", ".join(str(len(x)) for x in lists)))
        tables = []
        for name, dtype, tensors in zip(("p", "g", "copies"), (h.f32, h.dtype, h.bf16), lists):
            if name == "p" and any(x is None for x in tensors):
                raise ValueError("p: a tensor is missing")
            for x, n in zip(tensors, h.sizes):
                if x is not None and x.numel() != n:
                    raise ValueError("%s: a tensor of %d numbers is wanted, not one of %s" % (name, n, tuple(x.shape)))
            tables.append((ctypes.c_void_p * len(tensors))(*(None if x is None else _t(x, dtype, n, name) for x, n in zip(tensors, h.sizes))))
        at = [x.data_ptr() for t in (lists[0], lists[2]) for x in t if x is not None and x.numel()]
        if len(set(at)) != len(at):
            raise ValueError("p, copies: a tensor stands there twice")
        _here(*(x for t in lists for x in t if x is not None and x.numel()))
        self.plan, self.tables = h, tables
        self.held = [x.detach() for t in lists for x in t if x is not None]  # (a tensor may get other memory later)
        self.first = next((x for x in self.held if x.numel()), None)


def seq_adamw_tensors(h, p, g, copies=None) -> SeqAdamwTensors:
    """p: fp32 tensors; g: gradients of the plan's type, None for tensors that stay as they are; copies: bf16 tensors that get p, or None."""
    return SeqAdamwTensors(h, p, g, copies)


def seq_adamw(h, tensors, m, v, now, scales=None, stream=None):
    """now: (rate, step from 1 on[, factor of the gradients]) as numbers, or the three as an fp32 tensor on the GPU."""
    if tensors.plan is not h:
        raise ValueError("tensors of this plan are wanted")
    on_gpu = hasattr(now, "data_ptr")
    _here(tensors.first, m, v, scales, now if on_gpu else None)
    p, g, copies = tensors.tables
    host = None if on_gpu else (ctypes.c_double * 3)(now[0], now[1], now[2] if len(now) > 2 else 1.0)
    conv._check(load().seq_adamw(_of(h, "seq_adamw"), p, g, copies, _t(m, h.mdtype, h.state, "m"), _t(v, h.vdtype, h.state, "v"),
                                 _o(scales, h.f32, h.scales, "scales"), host, _t(now, h.f32, 3, "now") if on_gpu else None, conv._stream(stream)), "seq_adamw")


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
