"""Host-side checks of the sequence operators: symbols, sizes, refusals before anything is launched, and the oracle's gradients
against differences of its forward passes."""
import ctypes
import os
import re

import numpy as np
import pytest

import seq_oracle as oracle
from paper_1808_05567_amd import conv, seq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_library_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "seq_mi355x.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(seq_[a-z_0-9]+)\s*\(", text))
    assert names == set(seq.EXPORTS)
    assert all(getattr(seq.load(), n) is not None for n in names)


def test_sizes():
    h = seq.seq_conv_create(3, 21, 100, 4, seq.SEQ_BF16, slots=5)
    assert (h.info.vlen, h.info.Cb, h.info.Cp, h.info.state_bytes) == (8, 3, 24, 3 * 3 * 16)
    assert "seq_conv" in seq.seq_describe(h)
    h = seq.seq_scan_create(3, 21, 100, 16, seq.SEQ_F32, slots=5)
    assert (h.info.vlen, h.info.Cb, h.info.Cp, h.info.state_bytes) == (4, 6, 24, 16 * 24 * 4)
    h = seq.seq_mv4_create(1, 200, 17, 64, seq.SEQ_I8)
    assert (h.info.wt_bytes, h.info.scale_bytes, h.info.Cp) == (2 * 32 * 64, 4 * 32 * 4, 208)


def status(f, *a, **k):
    with pytest.raises(conv.ConvError) as e:
        f(*a, **k)
    return e.value.status


def test_refused_problems():
    E, U = conv.CONV_EINVAL, conv.CONV_EUNSUPPORTED
    for bad in (dict(N=0), dict(C=0), dict(L=-1), dict(W=0), dict(dtype=7), dict(dtype=seq.SEQ_I8), dict(slots=-1)):
        assert status(seq.seq_conv_create, **{**dict(N=1, C=8, L=4, W=4), **bad}) == E, bad
    for bad in (dict(W=1), dict(W=9), dict(C=1 << 21), dict(N=1 << 20, L=1 << 12), dict(L=(1 << 30) + 1)):
        assert status(seq.seq_conv_create, **{**dict(N=1, C=8, L=4, W=4), **bad}) == U, bad
    for bad in (dict(S=0), dict(G=0), dict(G=3), dict(dtype=5)):
        assert status(seq.seq_scan_create, **{**dict(N=1, C=8, L=4, S=4), **bad}) == E, bad
    for bad in (dict(S=65), dict(G=4, C=8), dict(G=2048, C=8 * 2048, S=64)):
        assert status(seq.seq_scan_create, **{**dict(N=1, C=8, L=4, S=4), **bad}) == U, bad
    for eps in (-1.0, float("nan"), float("inf")):
        assert status(seq.seq_norm_create, 1, 8, 4, eps=eps) == E
    for bad in (dict(M=0), dict(group=48), dict(dtype=3), dict(dtype=-1)):
        assert status(seq.seq_mv4_create, **{**dict(M=1, C=8, K=8, group=32), **bad}) == E, bad
    assert status(seq.seq_mv4_create, (1 << 16) + 1, 8, 8, 32) == U
    # blocks or positions too far apart for the scan's tiles, and more work-items than a launch has
    assert status(seq.seq_scan_create, 1, 16, 1 << 23, 4) == U
    assert status(seq.seq_conv_create, 1 << 20, 1 << 12, 1, 4) == U and status(seq.seq_scan_create, 1 << 20, 1 << 13, 1, 4) == U
    assert status(seq.seq_mv4_create, 1 << 16, 8, 1 << 20, 32) == U


@pytest.mark.parametrize("strides,ok_in,ok_out", [
    ((0, 0, 0), True, True), ((96, 32, 8), True, True), ((96, 8, 24), True, True), ((96, 32, 4), False, False), ((96, -32, 8), False, False),
    ((0, 32, 8), True, False), ((88, 32, 8), True, False), ((1 << 41, 32, 8), False, False), ((96, 24, 16), True, False),
])
def test_views(strides, ok_in, ok_out):
    """N = 2, three blocks, L = 4 of bf16."""
    for name, ok in (("x", ok_in), ("y", ok_out)):
        d = seq.SeqConvDesc(N=2, C=24, L=4, W=4, dtype=seq.SEQ_BF16)
        setattr(d, name, seq.SeqView(*strides))
        h = ctypes.c_void_p()
        st = seq.load().seq_conv_create(ctypes.byref(d), ctypes.byref(h))
        assert (st == conv.CONV_OK) == ok, (name, st)
        if st == conv.CONV_OK:
            seq.load().seq_destroy(h)


def test_pointers_are_checked_before_any_launch():
    lib, E, WS = seq.load(), conv.CONV_EINVAL, conv.CONV_EWORKSPACE
    c = seq.seq_conv_create(1, 8, 4, 4, slots=1)
    s = seq.seq_scan_create(1, 8, 4, 4, slots=1)
    n = seq.seq_norm_create(1, 8, 4)
    m = seq.seq_mv4_create(1, 8, 8, 32, seq.SEQ_I8)
    no, p, odd = None, 16, 24
    assert lib.seq_conv_fwd(no, p, p, p, no, p, no, no, no, no) == E
    assert lib.seq_conv_fwd(s._h, p, p, p, no, p, no, no, no, no) == E  # (a plan of something else)
    assert lib.seq_conv_fwd(c._h, no, p, p, no, p, no, no, no, no) == E
    assert lib.seq_conv_fwd(c._h, p, p, odd, no, p, no, no, no, no) == E
    assert lib.seq_conv_fwd(c._h, p, p, p, no, p, no, 18, no, no) == E
    assert lib.seq_conv_step(c._h, p, p, p, no, p, no, no) == E
    assert lib.seq_conv_bwd(c._h, p, p, p, p, p, p, p, no, no, 0, no) == WS
    assert lib.seq_conv_bwd(c._h, p, p, p, p, p, p, p, no, p, c.info.workspace_bytes - 1, no) == WS
    assert lib.seq_scan_fwd(s._h, p, p, no, p, p, no, no, no, no, p, no, no, no, no, 0, no) == E
    assert lib.seq_scan_bwd(s._h, p, p, p, p, p, no, no, no, p, p, p, p, p, p, no, no, no, no, no, 0, no) == WS
    # a gate without its gradient, and the other way round
    assert lib.seq_scan_bwd(s._h, p, p, p, p, p, no, p, no, p, p, p, p, p, p, no, no, no, no, p, 1 << 30, no) == E
    assert lib.seq_scan_bwd(s._h, p, p, p, p, p, no, no, no, p, p, p, p, p, p, no, p, no, no, p, 1 << 30, no) == E
    # states without slots
    none, nos = seq.seq_conv_create(1, 8, 4, 4), seq.seq_scan_create(1, 8, 4, 4)
    assert lib.seq_conv_fwd(none._h, p, p, p, p, p, no, no, no, no) == E and lib.seq_conv_step(none._h, p, p, p, p, p, no, no) == E
    assert lib.seq_scan_fwd(nos._h, p, p, p, p, p, no, no, no, p, p, no, no, no, no, 0, no) == E
    assert lib.seq_scan_step(nos._h, p, p, p, p, p, no, no, no, p, p, no, no) == E
    # single positions by a plan of more
    assert lib.seq_conv_step(c._h, p, p, p, p, p, no, no) == E and lib.seq_scan_step(s._h, p, p, p, p, p, no, no, no, p, p, no, no) == E
    long = seq.seq_scan_create(1, 64, 4096, 16)
    assert lib.seq_scan_fwd(long._h, p, p, p, p, p, no, no, no, no, p, no, no, no, p, 16, no) == WS
    assert lib.seq_norm_fwd(n._h, p, no, no, no, p, no) == E
    assert lib.seq_norm_fwd_q8(n._h, p, no, p, no, p, no, no) == E
    assert lib.seq_norm_bwd(n._h, p, p, p, no, p, p, no, 0, no) == WS
    assert lib.seq_mv4(m._h, p, no, p, p, no, p, no) == E  # (8 bits without a scale)
    assert lib.seq_destroy(no) == E and lib.seq_query(c._h, no) == E


def test_binding_refuses_tensors_that_do_not_fit():
    import torch
    h = seq.seq_norm_create(1, 8, 4)
    x = torch.zeros(1, 2, 4, 4)
    with pytest.raises(ValueError):  # (not on the GPU)
        seq.seq_norm_fwd(h, x, None, torch.zeros(8), None, x)
    with pytest.raises(ValueError):
        seq.seq_norm_fwd(seq.seq_conv_create(1, 8, 4, 4), x, None, torch.zeros(8), None, x)
    for t in (torch.zeros(1, 2, 4, 8), torch.zeros(2, 4, 4), torch.zeros(1, 2, 4, 8)[..., ::2]):
        with pytest.raises(ValueError):
            seq.seq_norm_create(1, 8, 4, views={"x": t})


# ---------------------------------------------------------------------------- the oracle
def difference(f, x, at, h=1e-5):
    up, down = x.copy(), x.copy()
    up[at] += h
    down[at] -= h
    return (f(up) - f(down)) / (2 * h)


def places(rng, x, count=6):
    return [tuple(int(rng.integers(n)) for n in x.shape) for _ in range(count)]


@pytest.mark.parametrize("silu", [True, False])
def test_the_oracles_convolution_gradients_are_differences(silu):
    rng = np.random.default_rng(0)
    N, C, L, W = 2, 3, 7, 4
    x, w, b, dy = rng.standard_normal((N, L, C)), rng.standard_normal((W, C)), rng.standard_normal(C), rng.standard_normal((N, L, C))
    lengths = [L, 3]
    dy[1, 3:] = 0
    dx, dw, db = oracle.conv_bwd(x, w, b, dy, silu, lengths)
    loss = lambda x, w, b: float((oracle.conv(x, w, b, silu, None, lengths)[0] * dy).sum())  # noqa: E731
    for got, arg, f in ((dx, x, lambda v: loss(v, w, b)), (dw, w, lambda v: loss(x, v, b)), (db, b, lambda v: loss(x, w, v))):
        for at in places(rng, arg):
            assert abs(difference(f, arg, at) - got[at]) < 1e-7


@pytest.mark.parametrize("gate,G,sp", [(True, 1, True), (False, 2, True), (True, 2, False)])
def test_the_oracles_scan_gradients_are_differences(gate, G, sp):
    rng = np.random.default_rng(1)
    N, C, L, S = 2, 4, 6, 3
    p = {"x": rng.standard_normal((N, L, C)), "dt": rng.standard_normal((N, L, C)) * 0.3, "A": -np.exp(rng.standard_normal((S, C))),
         "B": rng.standard_normal((N, L, G * S)), "Cm": rng.standard_normal((N, L, G * S)), "D": rng.standard_normal(C),
         "z": rng.standard_normal((N, L, C)) if gate else None, "dt_bias": rng.standard_normal(C)}
    dy, lengths = rng.standard_normal((N, L, C)), [L, 2]
    g = oracle.scan_bwd(**p, dy=dy, G=G, use_softplus=sp, lengths=lengths)
    names = {"x": "dx", "dt": "ddt", "A": "dA", "B": "dB", "Cm": "dC", "D": "dD", "z": "dz", "dt_bias": "ddt_bias"}
    for k, name in names.items():
        if p[k] is None:
            continue
        f = lambda v: float((oracle.scan(**{**p, k: v}, G=G, use_softplus=sp, lengths=lengths)[0] * dy).sum())  # noqa: E731,B023
        for at in places(rng, p[k]):
            assert abs(difference(f, p[k], at) - g[name][at]) < 1e-6 * (1 + abs(g[name][at])), name


def test_the_oracles_norm_gradients_are_differences():
    rng = np.random.default_rng(2)
    r, w, dy, dr = rng.standard_normal((2, 3, 5)), rng.standard_normal(5), rng.standard_normal((2, 3, 5)), rng.standard_normal((2, 3, 5))
    dx, dw = oracle.norm_bwd(r, w, dy, dr, 1e-2)
    loss = lambda r, w: float((oracle.norm(r, w, 1e-2) * dy).sum() + (r * dr).sum())  # noqa: E731
    for at in places(rng, r):
        assert abs(difference(lambda v: loss(v, w), r, at) - dx[at]) < 1e-8
    for at in places(rng, w):
        assert abs(difference(lambda v: loss(r, v), w, at) - dw[at]) < 1e-8
