"""The sequence operators at sizes that reach their other loops: many workgroups' shares of the channels, results past the caches, states of a gigabyte."""
import numpy as np
import pytest
import torch

import seq_oracle as oracle
from seq_util import DTYPES, Seq, close, ints, nans, rounded, spoil, vector, vlen
from test_gpu_seq_norm import EPS, forward_bound
from test_gpu_seq_scan import bound, data, tensors
from paper_1808_05567_amd import seq

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,C,S", [(512, 8192, 64), (700, 6000, 33)])
def test_steps_of_a_gigabyte_of_states(N, C, S, dtype):
    """Compared at every 397th channel of some sequences."""
    rng, slots, v = np.random.default_rng(4), N + 1, vlen(dtype)
    f = lambda c: rounded(rng.standard_normal((N, 1, c)).astype(np.float32), dtype)  # noqa: E731
    x, dt, z, B, Cm = f(C), 0.5 * f(C), f(C), f(S), f(S)
    A, bias = np.float64(np.float32(-np.exp(rng.uniform(-3, 2, (S, C))))), np.float64(np.float32(rng.uniform(-6, 0.5, C)))
    X, DT, Z, BT, CT, Y = (Seq(N, n, 1, dtype, "dense", t) for n, t in ((C, x), (C, dt), (C, z), (S, B), (S, Cm), (C, None)))
    h = seq.seq_scan_create(N, C, 1, S, dtype, slots=slots)
    state = torch.randn(slots, S, h.info.Cp, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    state[..., C:] = 0
    where, n, c = rng.permutation(slots)[:N], np.array([0, 1, N // 2, N - 1]), np.arange(0, C, 397)
    pick = lambda: state[torch.from_numpy(where[n]).cuda()][..., torch.from_numpy(c).cuda()].double().cpu().numpy()  # noqa: E731
    spare, old = state[np.setdiff1d(np.arange(slots), where)[0]].clone(), pick()
    seq.seq_scan_step(h, X.t, DT.t, vector(A, v), BT.t, CT.t, state, Y.t, z=Z.t, dt_bias=vector(bias, v), slots=ints(where))
    args = (x[n][..., c], dt[n][..., c], A[:, c], B[n], Cm[n])
    opt = dict(z=z[n][..., c], dt_bias=bias[c], state=old)
    (y, after), (my, ma) = oracle.scan(*args, **opt), oracle.scan(*args, **opt, mag=True)
    close(Y.get()[n][..., c], y, bound(1) * my, dtype == seq.SEQ_BF16, "y")
    close(pick(), after, bound(1) * ma, False, "state")
    assert torch.equal(spare, state[np.setdiff1d(np.arange(slots), where)[0]])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,C,L,S,G", [(2, 1160, 20, 16, 1), (1, 300, 20, 64, 1), (2, 1040, 9, 8, 2), (1, 2304, 17, 33, 2)])
def test_scan_gradients_from_many_shares_of_the_channels(N, C, L, S, G, dtype):
    """Eight workgroups and more (here 10, 10, 3 and 36) each leave a part of dB and dC."""
    rng, p = data(N, C, L, S, G, dtype, C)
    lengths, bf16 = np.array([L, L - 4][:N]), dtype == seq.SEQ_BF16
    t, opt, A, ref = tensors(p, N, C, L, S, G, True, True, lengths, "dense", dtype)
    DY = Seq(N, C, L, dtype, "dense", spoil(p["dy"], lengths))
    out = {k: Seq(N, c, L, dtype) for k, c in (("dx", C), ("ddt", C), ("dz", C), ("dB", G * S), ("dC", G * S))}
    h = seq.seq_scan_create(N, C, L, S, dtype, G=G)
    dA, dD, db = nans(S, h.info.Cp), nans(h.info.Cp), nans(h.info.Cp)
    seq.seq_scan_bwd(h, t["x"].t, t["dt"].t, A, t["B"].t, t["C"].t, DY.t, out["dx"].t, out["ddt"].t, dA, out["dB"].t, out["dC"].t,
                     seq.seq_workspace(h).fill_(0xFF), z=t["z"].t, dD=dD, dz=out["dz"].t, ddt_bias=db, lengths=ints(lengths), **opt)
    args = (p["x"], p["dt"], p["A"], p["B"], p["Cm"], p["dy"])
    r, m = oracle.scan_bwd(*args, **ref), oracle.scan_bwd(*args, **ref, mag=True)
    for k, q in out.items():
        close(q.get(), r[k], (2 * bound(L) + C * U) * m[k], bf16, k)
    for k, got in (("dA", dA), ("dD", dD), ("ddt_bias", db)):
        close(got.double().cpu().numpy()[..., :C], r[k], (2 * bound(L) + N * L * U) * m[k], False, k)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["dense", "rows"])
def test_convolution_of_more_than_16_megabytes(layout, dtype):
    """Results past the caches, compared at every 97th channel."""
    N, C, W = 2, 1028, 4
    L = 2100 if dtype == seq.SEQ_F32 else 4200
    rng = np.random.default_rng(1)
    x = rounded(rng.standard_normal((N, L, C)).astype(np.float32), dtype)
    w, bias = (np.float64(np.float32(0.5 * rng.standard_normal(s))) for s in ((W, C), (C,)))
    lengths, v = np.array([L - 5, L]), vlen(dtype)
    X, Y = Seq(N, C, L, dtype, layout, spoil(x, lengths)), Seq(N, C, L, dtype, layout)
    h = seq.seq_conv_create(N, C, L, W, dtype, views={"x": X.t, "y": Y.t})
    seq.seq_conv_fwd(h, X.t, vector(w, v), vector(bias, v), Y.t, lengths=ints(lengths))
    some = np.arange(0, C, 97)
    args = (x[..., some], w[:, some], bias[some], True, None, lengths)
    close(Y.get()[..., some], oracle.conv(*args)[0], 16 * U * oracle.conv(*args, mag=True)[0], dtype == seq.SEQ_BF16, "y")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["dense", "rows"])
def test_norm_of_more_than_16_megabytes(layout, dtype):
    """Results past the caches, one position and sixteen at a time."""
    N, C, L = 4, 1044, 2100
    rng = np.random.default_rng(2)
    x, res = (rounded(rng.standard_normal((N, L, C)).astype(np.float32), dtype) for _ in range(2))
    w = np.float64(np.float32(rng.standard_normal(C)))
    X, RES, R, Y = (Seq(N, C, L, dtype, layout, a) for a in (x, res, None, None))
    h = seq.seq_norm_create(N, C, L, dtype, EPS, views={"x": X.t, "res": RES.t, "r": R.t, "y": Y.t})
    seq.seq_norm_fwd(h, X.t, RES.t, vector(w, vlen(dtype)), R.t, Y.t)
    r = R.get()
    close(r, x + res, U * np.abs(x + res), dtype == seq.SEQ_BF16, "r")
    y = oracle.norm(r, w, EPS)
    close(Y.get(), y, forward_bound(C) * np.abs(y), dtype == seq.SEQ_BF16, "y")
