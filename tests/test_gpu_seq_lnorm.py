"""Layer norm against its definition in 64 bits."""
import numpy as np
import pytest
import torch

import seq_rec_oracle as oracle
from seq_util import DTYPES, Seq, close, ints, lengths_of, nans, rounded, spoil, vector, vlen
from paper_1808_05567_amd import seq

pytestmark = pytest.mark.gpu
U, EPS = 2.0 ** -24, 1e-5

CASES = [  # N, C, L, residual, bias, lengths, layout.  (Some are more than a workgroup holds at once; one channel is no variance at all.)
    (1, 8, 1, True, True, "none", "dense"), (2, 5, 3, False, False, "none", "slice"), (3, 40, 17, True, True, "ragged", "rows"),
    (1, 130, 65, True, False, "none", "dense"), (16, 4096, 1, True, True, "none", "dense"), (2, 2048, 9, True, True, "clamped", "dense"),
    (1, 1000, 7, True, True, "none", "slice"), (1, 8200, 3, True, True, "none", "rows"), (1, 8201, 9, False, True, "none", "dense"),
    (2, 20001, 5, True, True, "ragged", "dense"), (3, 34003, 2, True, False, "ragged", "rows"), (700, 17, 1, True, True, "none", "dense"),
    (3, 520, 1500, True, True, "ragged", "rows"), (1, 45, 4200, False, True, "none", "rows"), (5, 1100, 900, True, True, "ragged", "rows"),
    (2, 136, 4100, True, True, "ragged", "dense"), (2, 1, 6, True, True, "none", "dense"), (4, 2047, 40, True, True, "none", "dense"),
]


def inputs(rng, N, C, L, dtype, shift):
    return rounded((rng.standard_normal((N, L, C)) + shift).astype(np.float32), dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,C,L,residual,bias,kind,layout", CASES)
def test_forward(N, C, L, residual, bias, kind, layout, dtype):
    rng = np.random.default_rng(C + L)
    x, res = inputs(rng, N, C, L, dtype, 0.5), inputs(rng, N, C, L, dtype, 4.0 if C % 2 else 0.0)
    w, b = (rng.standard_normal(C).astype(np.float32).astype(np.float64) for _ in range(2))
    x[0, 0] = res[0, 0] = 0
    lengths = lengths_of(kind, N, L, rng)
    X, RES = (Seq(N, C, L, dtype, layout, spoil(t, lengths)) for t in (x, res))
    Y, R, Q = Seq(N, C, L, dtype, layout), Seq(N, C, L, dtype, layout), Seq(N, C, L, dtype, layout, v=16, torch_type=torch.int8)
    scale = nans(N, L)
    h = seq.seq_lnorm_create(N, C, L, dtype, EPS, views={"x": X.t, "res": RES.t, "r": R.t, "y": Y.t, "q": Q.t})
    wv, bv = vector(w, vlen(dtype)), vector(b, vlen(dtype)) if bias else None
    seq.seq_lnorm_fwd(h, X.t, RES.t if residual else None, wv, bv, R.t if residual else None, Y.t, lengths=ints(lengths))
    live = np.ones((N, L, 1))
    for n, end in enumerate(lengths if lengths is not None else []):
        live[n, max(int(end), 0):] = 0
    r = x * live
    if residual:
        r = R.get()
        close(r, (x + res) * live, U * np.abs(x + res), dtype == seq.SEQ_BF16, "r")
    y, ey = oracle.lnorm(r, w, b if bias else None, EPS)
    y, ey = y * live, ey * live
    close(Y.get(), y, ey, dtype == seq.SEQ_BF16, "y")
    # 8 bits; r into the residual's place this time, for some
    inplace = residual and N % 2 == 1
    if inplace:
        h = seq.seq_lnorm_create(N, C, L, dtype, EPS, views={"x": X.t, "res": RES.t, "r": RES.t, "y": Y.t, "q": Q.t})
    seq.seq_lnorm_fwd_q8(h, X.t, RES.t if residual else None, wv, bv, (RES.t if inplace else R.t) if residual else None, Q.t, scale, lengths=ints(lengths))
    got, s = Q.get(), scale.double().cpu().numpy()
    if inplace:
        np.testing.assert_array_equal(RES.get(), r)
    want = np.abs(y).max(-1) / 127
    close(s, want, ey.max(-1) / 127 + 2 * U * want, False, "scale")
    # the nearest whole number, but for quotients that rounding takes across a half: off by y's error and the scale's 127 times its own share, and by 4 U of 127
    step = np.where(s > 0, s, 1)[..., None]
    assert np.all(np.abs(got - y / step) <= 0.5 + 2 * ey.max(-1, keepdims=True) / step + 127 * 4 * U)
    assert np.all(np.abs(got).max(-1)[s > 0] == 127) and not got[s == 0].any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,C,L,residual,bias,kind,layout", CASES)
def test_gradients(N, C, L, residual, bias, kind, layout, dtype):
    rng = np.random.default_rng(C + L + 1)
    r, dy, dr = inputs(rng, N, C, L, dtype, 3.0 if C % 2 else 0.25), inputs(rng, N, C, L, dtype, 0), inputs(rng, N, C, L, dtype, 0)
    w = rng.standard_normal(C).astype(np.float32).astype(np.float64)
    lengths = lengths_of(kind, N, L, rng)
    R, DY, DR = (Seq(N, C, L, dtype, layout, spoil(t, lengths)) for t in (r, dy, dr))
    DX = Seq(N, C, L, dtype, layout)
    h = seq.seq_lnorm_create(N, C, L, dtype, EPS, views={"r": R.t, "dy": DY.t, "dx": DX.t, "dr": DR.t})
    dw, db, ws = nans(h.info.Cp), nans(h.info.Cp) if bias else None, seq.seq_workspace(h).fill_(0xFF)

    def call():
        seq.seq_lnorm_bwd(h, R.t, vector(w, vlen(dtype)), DY.t, DR.t if residual else None, DX.t, dw, db, ws, lengths=ints(lengths))
    call()
    inside = np.concatenate([np.arange(n * L, n * L + min(max(int(e), 0), L)) for n, e in enumerate([L] * N if lengths is None else lengths)])
    flat = lambda t: t.reshape(N * L, C)[inside]  # noqa: E731
    want, err = oracle.lnorm_bwd(flat(r), w, flat(dy), flat(dr) if residual else None, EPS)
    got = DX.get().reshape(N * L, C)
    close(got[inside], want[0], err[0], dtype == seq.SEQ_BF16, "dx")
    assert not np.delete(got, inside, axis=0).any()
    close(dw.double().cpu().numpy()[:C], want[1], err[1], False, "dw")
    assert not dw[C:].any()
    if bias:
        close(db.double().cpu().numpy()[:C], want[2], err[2], False, "db")
        assert not db[C:].any()
    first = dw.clone(), DX.t.clone()
    ws.fill_(0xFF)
    call()
    assert torch.equal(first[0], dw) and torch.equal(first[1], DX.t)


@pytest.mark.parametrize("C", [64, 61])
def test_no_numbers_stay_visible(C):
    """NaN and infinity in one position make its scale NaN, and leave the others alone; slots beyond C stay zero."""
    N, L, dtype = 1, 4, seq.SEQ_F32
    x = np.random.default_rng(0).standard_normal((N, L, C))
    x[0, 1, 3], x[0, 2, 60] = np.nan, np.inf
    X, Y, Q, scale = Seq(N, C, L, dtype, "dense", x), Seq(N, C, L, dtype), Seq(N, C, L, dtype, v=16, torch_type=torch.int8), nans(N, L)
    h = seq.seq_lnorm_create(N, C, L, dtype, EPS)
    ones = vector(np.ones(C), 4)
    seq.seq_lnorm_fwd(h, X.t, None, ones, None, None, Y.t)
    seq.seq_lnorm_fwd_q8(h, X.t, None, ones, None, None, Q.t, scale)
    s = scale.cpu().numpy()[0]
    assert np.isnan(s[1]) and np.isnan(s[2]) and np.isfinite(s[[0, 3]]).all()
    y = Y.get()[0]
    assert np.isnan(y[1]).all() and np.isnan(y[2]).all() and np.isfinite(y[[0, 3]]).all()
    R, DY, DX = Seq(N, C, L, dtype, "dense", x), Seq(N, C, L, dtype, "dense", np.ones((N, L, C))), Seq(N, C, L, dtype)
    seq.seq_lnorm_bwd(h, R.t, ones, DY.t, None, DX.t, nans(h.info.Cp), None, seq.seq_workspace(h))
    d = DX.get()[0]
    assert np.isnan(d[1]).all() and np.isnan(d[2]).all() and np.isfinite(d[[0, 3]]).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["dense", "rows"])
def test_more_than_16_megabytes(layout, dtype):
    """Results past the caches, one position and sixteen at a time."""
    N, C, L = 4, 1044, 2100
    rng = np.random.default_rng(2)
    x, res = (inputs(rng, N, C, L, dtype, 0.3) for _ in range(2))
    w, b = (np.float64(np.float32(rng.standard_normal(C))) for _ in range(2))
    X, RES, R, Y = (Seq(N, C, L, dtype, layout, a) for a in (x, res, None, None))
    h = seq.seq_lnorm_create(N, C, L, dtype, EPS, views={"x": X.t, "res": RES.t, "r": R.t, "y": Y.t})
    seq.seq_lnorm_fwd(h, X.t, RES.t, vector(w, vlen(dtype)), vector(b, vlen(dtype)), R.t, Y.t)
    r = R.get()
    close(r, x + res, U * np.abs(x + res), dtype == seq.SEQ_BF16, "r")
    y, ey = oracle.lnorm(r, w, b, EPS)
    close(Y.get(), y, ey, dtype == seq.SEQ_BF16, "y")


def test_a_mean_far_from_zero():
    """Differences of some units of 4096 in fp32: the variance is that of the numbers as they are stored."""
    N, C, L, dtype = 2, 600, 5, seq.SEQ_F32
    rng = np.random.default_rng(1)
    x = np.float64(np.float32(4096 + rng.standard_normal((N, L, C))))
    X, Y = Seq(N, C, L, dtype, "dense", x), Seq(N, C, L, dtype)
    h = seq.seq_lnorm_create(N, C, L, dtype, EPS)
    w = np.ones(C)
    seq.seq_lnorm_fwd(h, X.t, None, vector(w, 4), None, None, Y.t)
    y, ey = oracle.lnorm(x, w, None, EPS)
    assert ey.max() < 0.02  # (74 units of 4096: what the mean itself may be off)
    close(Y.get(), y, ey, False, "y")
