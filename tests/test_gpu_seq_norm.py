"""Root-mean-square norm against its definition in 64 bits."""
import numpy as np
import pytest
import torch

import seq_oracle as oracle
from seq_util import DTYPES, Seq, close, nans, rounded, vector, vlen
from paper_1808_05567_amd import seq

pytestmark = pytest.mark.gpu
U, EPS = 2.0 ** -24, 1e-5

CASES = [  # N, C, L, residual, layout.  (The last ones: more than a workgroup holds at once.)
    (1, 8, 1, True, "dense"), (2, 5, 3, False, "slice"), (3, 40, 17, True, "rows"), (1, 130, 65, True, "dense"), (16, 4096, 1, True, "dense"),
    (2, 2048, 9, True, "dense"), (1, 1000, 7, True, "slice"), (1, 8200, 3, True, "rows"), (1, 8200, 9, False, "dense"), (2, 20000, 5, True, "dense"),
    (3, 34000, 2, True, "rows"), (700, 16, 1, True, "dense"), (3, 520, 1500, True, "rows"), (1, 40, 4200, False, "rows"), (5, 1100, 900, True, "rows"), (2, 136, 4100, True, "dense"),
]


def forward_bound(C):
    # the sum of squares (at most log2 of the threads and 16 terms in turn: C units are far more), its root, a quotient, two products
    return (8 + min(C, 64)) * U


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,C,L,residual,layout", CASES)
def test_forward(N, C, L, residual, layout, dtype):
    rng = np.random.default_rng(C + L)
    x, res = rounded(rng.standard_normal((N, L, C)), dtype), rounded(rng.standard_normal((N, L, C)), dtype)
    w = rng.standard_normal(C).astype(np.float32).astype(np.float64)
    x[0, 0] = 0
    res[0, 0] = 0
    X, RES, Y, R = Seq(N, C, L, dtype, layout, x), Seq(N, C, L, dtype, layout, res), Seq(N, C, L, dtype, layout), Seq(N, C, L, dtype, layout)
    Q = Seq(N, C, L, dtype, layout, v=16, torch_type=torch.int8)
    scale = nans(N, L)
    h = seq.seq_norm_create(N, C, L, dtype, EPS, views={"x": X.t, "res": RES.t, "r": R.t, "y": Y.t, "q": Q.t})
    wv = vector(w, vlen(dtype))
    seq.seq_norm_fwd(h, X.t, RES.t if residual else None, wv, R.t if residual else None, Y.t)
    r = x
    if residual:
        r = R.get()
        close(r, x + res, U * np.abs(x + res), dtype == seq.SEQ_BF16, "r")
    y = oracle.norm(r, w, EPS)
    close(Y.get(), y, forward_bound(C) * np.abs(y), dtype == seq.SEQ_BF16, "y")
    # 8 bits; r into the residual's place this time, for some
    inplace = residual and N % 2 == 1
    if inplace:
        h = seq.seq_norm_create(N, C, L, dtype, EPS, views={"x": X.t, "res": RES.t, "r": RES.t, "y": Y.t, "q": Q.t})
    seq.seq_norm_fwd_q8(h, X.t, RES.t if residual else None, wv, (RES.t if inplace else R.t) if residual else None, Q.t, scale)
    got, s = Q.get(), scale.double().cpu().numpy()
    if inplace:
        np.testing.assert_array_equal(RES.get(), r)
    want = np.abs(y).max(-1) / 127
    close(s, want, 2 * forward_bound(C) * want, False, "scale")
    # the nearest whole number, but for quotients that rounding takes across a half
    assert np.all(np.abs(got - y / np.where(s > 0, s, 1)[..., None]) <= 0.5 + 127 * 4 * forward_bound(C))
    assert not got[0, 0].any() and s[0, 0] == 0
    assert np.all(np.abs(got).max(-1)[s > 0] == 127)


def test_no_numbers_stay_visible():
    """NaN and infinity in one position make its scale NaN, and leave the others alone."""
    N, C, L, dtype = 1, 64, 4, seq.SEQ_F32
    x = np.random.default_rng(0).standard_normal((N, L, C))
    x[0, 1, 3], x[0, 2, 60] = np.nan, np.inf
    X, Y, Q, scale = Seq(N, C, L, dtype, "dense", x), Seq(N, C, L, dtype), Seq(N, C, L, dtype, v=16, torch_type=torch.int8), nans(N, L)
    h = seq.seq_norm_create(N, C, L, dtype, EPS)
    seq.seq_norm_fwd(h, X.t, None, vector(np.ones(C), 4), None, Y.t)
    seq.seq_norm_fwd_q8(h, X.t, None, vector(np.ones(C), 4), None, Q.t, scale)
    s = scale.cpu().numpy()[0]
    assert np.isnan(s[1]) and np.isnan(s[2]) and np.isfinite(s[[0, 3]]).all()
    y = Y.get()[0]
    assert np.isnan(y[1]).all() and np.isnan(y[2, 60]) and np.isfinite(y[[0, 3]]).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,C,L,residual,layout", CASES)
def test_gradients(N, C, L, residual, layout, dtype):
    rng = np.random.default_rng(C + L + 1)
    f = lambda: rounded(rng.standard_normal((N, L, C)), dtype)  # noqa: E731
    r, dy, dr = f(), f(), f() if residual else None
    w = rng.standard_normal(C).astype(np.float32).astype(np.float64)
    R, DY, DX = Seq(N, C, L, dtype, layout, r), Seq(N, C, L, dtype, layout, dy), Seq(N, C, L, dtype, layout)
    DR = Seq(N, C, L, dtype, layout, dr) if residual else None
    h = seq.seq_norm_create(N, C, L, dtype, EPS, views={"r": R.t, "dy": DY.t, "dx": DX.t, "dr": DR.t if residual else None})
    dw, ws = nans(h.info.Cp), seq.seq_workspace(h).fill_(0xFF)
    seq.seq_norm_bwd(h, R.t, vector(w, vlen(dtype)), DY.t, DR.t if residual else None, DX.t, dw, ws)
    ref, mag = oracle.norm_bwd(r, w, dy, dr, EPS), oracle.norm_bwd(r, w, dy, dr, EPS, mag=True)
    close(DX.get(), ref[0], 3 * forward_bound(C) * mag[0], dtype == seq.SEQ_BF16, "dx")
    got = dw.double().cpu().numpy()
    assert not got[C:].any()
    close(got[:C], ref[1], (forward_bound(C) + N * L * U) * mag[1], False, "dw")
    first = dw.clone()
    ws.fill_(0xFF)
    seq.seq_norm_bwd(h, R.t, vector(w, vlen(dtype)), DY.t, DR.t if residual else None, DX.t, dw, ws)
    assert torch.equal(first, dw)
