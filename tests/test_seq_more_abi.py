"""Host-side checks of the recurrence, the layer norm and AdamW: sizes, refusals before anything is launched, and the oracle's gradients against
differences of its forward passes."""
import ctypes
import functools

import numpy as np
import pytest
import torch

import seq_rec_oracle as oracle
from paper_1808_05567_amd import conv, seq
from test_seq_abi import difference, places, status
from test_seq_binding import calls, tensor  # noqa: F401


def test_sizes():
    h = seq.seq_rec_create(3, 21, 100, seq.SEQ_BF16, slots=5)
    assert (h.info.vlen, h.info.Cb, h.info.Cp, h.info.state_bytes) == (8, 3, 24, 24 * 4) and "seq_rec" in seq.seq_describe(h)
    h = seq.seq_lnorm_create(3, 21, 100, seq.SEQ_F32)
    assert (h.info.vlen, h.info.Cb, h.info.Cp) == (4, 6, 24) and "seq_lnorm" in seq.seq_describe(h)
    for bits, n in ((32, 4), (8, 1)):
        h = seq.seq_adamw_create([1, 0, 256, 257], bits=bits)
        assert h.info.state_bytes == 4 * 256 * n and h.info.scale_bytes == (4 * 8 if bits == 8 else 0) and h.info.workspace_bytes == 0
        assert (h.state, h.scales) == (1024, 8 if bits == 8 else 0) and "tensors=4" in seq.seq_describe(h)
    assert seq.seq_adamw_create([0, 0]).state == 0


def test_refused_problems():
    E, X = conv.CONV_EINVAL, conv.CONV_EUNSUPPORTED
    for bad in (dict(N=0), dict(C=0), dict(L=-1), dict(dtype=7), dict(dtype=seq.SEQ_I8), dict(slots=-1)):
        assert status(seq.seq_rec_create, **{**dict(N=1, C=8, L=4), **bad}) == E, bad
    for bad in (dict(C=1 << 21), dict(N=1 << 20, L=1 << 12), dict(L=(1 << 30) + 1), dict(N=1 << 20, C=1 << 13, L=1)):
        assert status(seq.seq_rec_create, **{**dict(N=1, C=8, L=4), **bad}) == X, bad
    for eps in (-1.0, float("nan"), float("inf")):
        assert status(seq.seq_lnorm_create, 1, 8, 4, eps=eps) == E
    inf, nan = float("inf"), float("nan")
    for bad in (dict(sizes=[]), dict(sizes=[4, -1]), dict(bits=16), dict(dtype=seq.SEQ_I8), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(betas=(nan, 0.9)),
                dict(eps=-1e-8), dict(eps=nan), dict(eps=inf), dict(decay=-0.1), dict(decay=nan), dict(decay=inf)):
        assert status(seq.seq_adamw_create, **{**dict(sizes=[4]), **bad}) == E, bad
    for sizes in ([1 << 36], [1 << 34, (1 << 34) + 1], [(1 << 62)] * 4, [(1 << 63) - 1]):
        assert status(seq.seq_adamw_create, sizes) == X, sizes
    with pytest.raises(ValueError):
        seq.seq_adamw_create([4, 4], decay=[0.1])


def test_pointers_are_checked_before_any_launch():
    lib, E, WS = seq.load(), conv.CONV_EINVAL, conv.CONV_EWORKSPACE
    r, n, rms = seq.seq_rec_create(1, 8, 4, slots=1), seq.seq_lnorm_create(1, 8, 4), seq.seq_norm_create(1, 8, 4)
    no, p, odd = None, 16, 24
    fwd = [p, p, p, p, no, no, no, no, p, no, no, no, no, 0, no]
    assert lib.seq_rec_fwd(no, *fwd) == E and lib.seq_rec_fwd(n._h, *fwd) == E
    for k in (0, 1, 2, 3, 8):
        assert lib.seq_rec_fwd(r._h, *fwd[:k], no, *fwd[k + 1:]) == E
    for k in (0, 1, 2, 3, 4, 5, 6, 7, 8, 9):
        assert lib.seq_rec_fwd(r._h, *fwd[:k], odd, *fwd[k + 1:]) == E
    assert lib.seq_rec_fwd(r._h, *fwd[:10], 18, *fwd[11:]) == E and lib.seq_rec_fwd(r._h, *fwd[:11], 18, *fwd[12:]) == E
    long = seq.seq_rec_create(1, 8, 1 << 14)  # (runs of a sequence: what they make of a state)
    assert lib.seq_rec_fwd(long._h, *fwd) == WS and lib.seq_rec_fwd(long._h, *fwd[:12], p, 16, no) == WS and lib.seq_rec_fwd(long._h, *fwd[:12], odd, 1 << 30, no) == E
    none = seq.seq_rec_create(1, 8, 4)
    assert lib.seq_rec_fwd(none._h, *fwd[:7], p, *fwd[8:]) == E and lib.seq_rec_fwd(none._h, *fwd[:9], p, *fwd[10:]) == E
    assert lib.seq_rec_step(r._h, p, p, p, p, no, no, no, p, p, no, no) == E  # (a plan of four positions)
    one = seq.seq_rec_create(1, 8, 1)
    assert lib.seq_rec_step(one._h, p, p, p, p, no, no, no, p, p, no, no) == E  # (without slots)
    bwd = [p, p, p, p, no, no, no, p, p, p, p, p, no, no, no, no]
    assert lib.seq_rec_bwd(r._h, *bwd, no, 0, no) == WS and lib.seq_rec_bwd(r._h, *bwd, p, r.info.workspace_bytes - 1, no) == WS
    for k in (4, 12):  # (a gate without its gradient, and the other way round)
        assert lib.seq_rec_bwd(r._h, *bwd[:k], p, *bwd[k + 1:], p, 1 << 20, no) == E
    assert lib.seq_lnorm_fwd(rms._h, p, no, p, no, no, p, no, no) == E and lib.seq_norm_fwd(n._h, p, no, p, no, p, no) == E
    assert lib.seq_lnorm_fwd(n._h, p, no, no, p, no, p, no, no) == E and lib.seq_lnorm_fwd(n._h, p, no, p, odd, no, p, no, no) == E
    assert lib.seq_lnorm_fwd(n._h, p, no, p, no, no, p, 18, no) == E and lib.seq_lnorm_fwd_q8(n._h, p, no, p, no, no, p, no, no, no) == E
    assert lib.seq_lnorm_bwd(n._h, p, p, p, no, p, p, p, no, no, 0, no) == WS
    assert lib.seq_lnorm_bwd(n._h, p, p, p, no, p, p, p, no, p, n.info.workspace_bytes - 1, no) == WS


def test_adamw_pointers_are_checked_before_any_launch():
    lib, E = seq.load(), conv.CONV_EINVAL
    table = lambda *x: (ctypes.c_void_p * len(x))(*x)  # noqa: E731
    now = (ctypes.c_double * 3)(1e-3, 1, 1)
    h32, h8 = seq.seq_adamw_create([4, 0]), seq.seq_adamw_create([4, 0], bits=8)
    ok = table(16, None)
    for p, g, copy, m, v, scales, host, gpu in (
            (None, ok, ok, 16, 16, None, now, None), (ok, None, ok, 16, 16, None, now, None), (ok, ok, ok, None, 16, None, now, None),
            (ok, ok, ok, 16, None, None, now, None), (ok, ok, ok, 16, 16, 16, now, None), (ok, ok, ok, 16, 16, None, None, None),
            (ok, ok, ok, 16, 16, None, now, 16), (ok, ok, ok, 16, 16, None, None, 18), (ok, ok, ok, 24, 16, None, now, None),
            (table(24, None), ok, ok, 16, 16, None, now, None), (ok, table(24, None), ok, 16, 16, None, now, None), (ok, ok, table(24, None), 16, 16, None, now, None),
            (table(None, None), ok, ok, 16, 16, None, now, None)):
        assert lib.seq_adamw(h32._h, p, g, copy, m, v, scales, host, gpu, None) == E
    assert lib.seq_adamw(h8._h, ok, ok, ok, 16, 16, None, now, None, None) == E
    for step in (0, -1, float("nan")):
        assert lib.seq_adamw(h32._h, ok, ok, ok, 16, 16, None, (ctypes.c_double * 3)(1e-3, step, 1), None, None) == E
    # nothing to do: no launch
    nothing = table(None, None)
    assert lib.seq_adamw(h32._h, nothing, nothing, None, 16, 16, None, now, None, None) == conv.CONV_OK
    empty = seq.seq_adamw_create([0])
    assert lib.seq_adamw(empty._h, table(None), table(16), None, None, None, None, now, None, None) == conv.CONV_OK


def test_adamw_tensors_are_checked(calls):  # noqa: F811
    f = torch.float32
    h = seq.seq_adamw_create([4, 6], seq.SEQ_BF16)
    p, g, c = [tensor(4, dtype=f), tensor(2, 3, dtype=f)], [tensor(4), tensor(6)], [tensor(4), None]
    good = seq.seq_adamw_tensors(h, p, g, c)
    m, v = tensor(512, dtype=f), tensor(512, dtype=f)
    seq.seq_adamw(h, good, m, v, (1e-3, 1), stream=0)
    seq.seq_adamw(h, seq.seq_adamw_tensors(h, p, [None, g[1]]), m, v, tensor(3, dtype=f), stream=0)
    assert calls == ["seq_adamw"] * 2
    for bad in ((p[:1], g), (p, g[:1]), (p, g, c[:1]), ([p[0], None], g), ([p[0], tensor(6)], g), (p, [g[0], tensor(6, dtype=f)]), (p, g, [tensor(4, dtype=f), None]),
                ([p[0], tensor(7, dtype=f)], g), ([p[0], tensor(12, dtype=f)[::2]], g), ([p[0], torch.zeros(6)], g), (p, g, [c[0], tensor(5)])):
        with pytest.raises(ValueError):
            seq.seq_adamw_tensors(h, *bad)
    twice = seq.seq_adamw_create([4, 4], seq.SEQ_BF16)
    with pytest.raises(ValueError):
        seq.seq_adamw_tensors(twice, [p[0], p[0]], [g[0], g[0]])
    with pytest.raises(ValueError):
        seq.seq_adamw_tensors(twice, [p[0], tensor(4, dtype=f)], [g[0], g[0]], [c[0], c[0]])
    seq.seq_adamw_tensors(twice, [p[0], tensor(4, dtype=f)], [g[0], g[0]])  # (gradients may be one)
    for args in ((twice, good, m, v, (1e-3, 1)), (h, good, m[:256], v, (1e-3, 1)), (h, good, m, tensor(512), (1e-3, 1)), (h, good, m, v, tensor(2, dtype=f)),
                 (h, good, m, v, tensor(3))):
        with pytest.raises(ValueError):
            seq.seq_adamw(*args, stream=0)
    assert calls == ["seq_adamw"] * 2


class Elsewhere(torch.Tensor):
    """A tensor in host memory that says it is on the second of several GPUs."""
    is_cuda = True

    def get_device(self):
        return 1


def test_tensors_of_two_devices_are_refused(calls):  # noqa: F811
    f = torch.float32
    h = seq.seq_lnorm_create(1, 8, 4, seq.SEQ_BF16)
    x, w = tensor(1, 1, 4, 8), tensor(8, dtype=f)
    seq.seq_lnorm_fwd(h, x, None, w, None, None, x, stream=0)
    assert calls == ["seq_lnorm_fwd"]
    far = torch.zeros(1, 1, 4, 8, dtype=torch.bfloat16).as_subclass(Elsewhere)
    with pytest.raises(ValueError):
        seq.seq_lnorm_fwd(h, far, None, w, None, None, x, stream=0)
    r = seq.seq_rec_create(1, 8, 4, seq.SEQ_BF16)
    with pytest.raises(ValueError):
        seq.seq_rec_fwd(r, x, x, far, w, x, stream=0)
    assert calls == ["seq_lnorm_fwd"]


def test_views_and_extents_of_the_recurrence(calls):  # noqa: F811
    N, L, w = 2, 4, tensor(16, dtype=torch.float32)
    wide = tensor(N, 8, L, 8)
    parts = [wide[:, 2 * k:2 * k + 2] for k in range(4)]
    h = seq.seq_rec_create(N, 16, L, seq.SEQ_BF16, views=dict(zip("xfiz", parts)))
    y = tensor(N, 2, L, 8)
    seq.seq_rec_fwd(h, *parts[:3], w, y, z=parts[3], stream=0)
    for k in range(3):
        bad = parts[:3]
        bad[k] = y
        with pytest.raises(ValueError):
            seq.seq_rec_fwd(h, *bad, w, y, stream=0)
    with pytest.raises(ValueError):
        seq.seq_rec_fwd(h, *parts[:3], w[:8], y, stream=0)
    assert calls == ["seq_rec_fwd"]


def test_distances_that_the_recurrence_refuses():
    """Positions more than 2^20 elements apart and, where x has its blocks nearer than its positions, blocks more than 2^24."""
    def at(c, l):
        return torch.empty_strided((2, 3, 5, 8), (1 << 40, c, l, 1), dtype=torch.bfloat16, device="meta")
    far, near = 1 << 20, 64
    plan = functools.partial(seq.seq_rec_create, 2, 24, 5, seq.SEQ_BF16)
    for name in ("x", "f", "i", "z", "y", "dy", "dx", "df", "di", "dz"):
        rows = {"x": at(8, near)}
        for views in ({name: at(8, far)}, rows | {name: at(1 << 24, near)}, {name: at(1 << 36, near)}):
            plan(views=views)
        for views in ({name: at(8, far + 8)}, rows | {name: at((1 << 24) + 8, near)}):
            if name != "x" or views["x"].stride(1) == 8:  # (with its blocks further apart x is not such a tensor)
                assert status(plan, views=views) == conv.CONV_EUNSUPPORTED


# ---------------------------------------------------------------------------- the oracle
@pytest.mark.parametrize("gate", [True, False])
def test_the_oracles_recurrence_gradients_are_differences(gate):
    rng = np.random.default_rng(1)
    N, C, L = 2, 4, 6
    p = {k: rng.standard_normal((N, L, C)) for k in ("x", "f", "i")}
    p.update(A=-np.exp(rng.uniform(-3, 1, C)), f_bias=rng.standard_normal(C), i_bias=rng.standard_normal(C), z=rng.standard_normal((N, L, C)) if gate else None)
    dy, lengths = rng.standard_normal((N, L, C)), [L, 2]
    g, _ = oracle.rec_bwd(**p, dy=dy, lengths=lengths)
    for k, name in {"x": "dx", "f": "df", "i": "di", "A": "dA", "z": "dz", "f_bias": "df_bias", "i_bias": "di_bias"}.items():
        if p[k] is None:
            continue
        f = lambda v: float((oracle.rec(**{**p, k: v}, lengths=lengths)[0][0] * dy).sum())  # noqa: E731,B023
        for at in places(rng, p[k]):
            assert abs(difference(f, p[k], at) - g[name][at]) < 1e-6 * (1 + abs(g[name][at])), name


def test_the_oracles_layer_norm_gradients_are_differences():
    rng = np.random.default_rng(2)
    r, w, b, dy, dr = rng.standard_normal((2, 3, 5)), rng.standard_normal(5), rng.standard_normal(5), rng.standard_normal((2, 3, 5)), rng.standard_normal((2, 3, 5))
    (dx, dw, db), _ = oracle.lnorm_bwd(r, w, dy, dr, 1e-2)
    loss = lambda r, w, b: float((oracle.lnorm(r, w, b, 1e-2)[0] * dy).sum() + (r * dr).sum())  # noqa: E731
    for x, got, f in ((r, dx, lambda v: loss(v, w, b)), (w, dw, lambda v: loss(r, v, b)), (b, db, lambda v: loss(r, w, v))):
        for at in places(rng, x):
            assert abs(difference(f, x, at) - got[at]) < 1e-7
