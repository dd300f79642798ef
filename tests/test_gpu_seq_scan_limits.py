"""The selective scan at the ends of what its parameters may be."""
import numpy as np
import pytest
import torch

import seq_oracle as oracle
from seq_util import DTYPES, Seq, close, ints, nans, spoil, vector, vlen
from test_gpu_seq_scan import bound, data, tensors
from paper_1808_05567_amd import seq

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("L", [1, 5, 16, 300])
def test_states_that_keep_nothing(L, dtype):
    """A of minus infinity: exp(d A) = 0, so that such a state is the position's own d B x, whatever positions the kernels add to fill their eights
    and runs, and whatever sequences end inside."""
    N, C, S, slots = 4, 72, 5, 6
    rng, p = data(N, C, L, S, 1, dtype, L)
    p["A"][1], p["A"][4, ::3] = -np.inf, -np.inf
    lengths = np.array([L, 0, min(1, L), max(1, L - 3)])
    t, opt, A, ref = tensors(p, N, C, L, S, 1, True, True, lengths, "dense", dtype)
    Y, old, where = Seq(N, C, L, dtype), rng.standard_normal((slots, S, C)).astype(np.float32), np.array([3, 0, 5, 1])
    st = vector(old, vlen(dtype))
    h = seq.seq_scan_create(N, C, L, S, dtype, slots=slots)
    ws = seq.seq_workspace(h).fill_(0xFF)
    seq.seq_scan_fwd(h, t["x"].t, t["dt"].t, A, t["B"].t, t["C"].t, Y.t, ws, z=t["z"].t, state_in=st, state_out=st, slots=ints(where), lengths=ints(lengths), **opt)
    args, ref = (p["x"], p["dt"], p["A"], p["B"], p["Cm"]), dict(ref, state=old[where])
    (y, after), (my, ma) = oracle.scan(*args, **ref), oracle.scan(*args, **ref, mag=True)
    close(Y.get(), y, bound(L) * my, dtype == seq.SEQ_BF16, "y")
    close(st.double().cpu().numpy()[where, :, :C], after, bound(L) * ma, False, "state")
    # backwards: all gradients that such a state has (that of dt is none: 0 times infinity)
    DY = Seq(N, C, L, dtype, "dense", spoil(p["dy"], lengths))
    out = {k: Seq(N, c, L, dtype) for k, c in (("dx", C), ("ddt", C), ("dz", C), ("dB", S), ("dC", S))}
    dA = nans(S, h.info.Cp)
    ws.fill_(0xFF)
    seq.seq_scan_bwd(h, t["x"].t, t["dt"].t, A, t["B"].t, t["C"].t, DY.t, out["dx"].t, out["ddt"].t, dA, out["dB"].t, out["dC"].t, ws,
                     z=t["z"].t, dz=out["dz"].t, lengths=ints(lengths), **opt)
    del ref["state"]
    with np.errstate(invalid="ignore"):
        r, m = oracle.scan_bwd(*args, p["dy"], **ref), oracle.scan_bwd(*args, p["dy"], **ref, mag=True)
    for k in ("dx", "dB", "dC", "dz"):
        close(out[k].get(), r[k], (2 * bound(L) + C * U) * m[k], dtype == seq.SEQ_BF16, k)
    close(dA.double().cpu().numpy()[:, :C], r["dA"], (2 * bound(L) + N * L * U) * m["dA"], False, "dA")


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_step_of_states_that_keep_nothing(dtype):
    N, C, S = 2, 24, 3
    rng, p = data(N, C, 1, S, 1, dtype, 3)
    p["A"][1] = -np.inf
    t, opt, A, ref = tensors(p, N, C, 1, S, 1, False, True, None, "dense", dtype)
    Y, old = Seq(N, C, 1, dtype), rng.standard_normal((N, S, C)).astype(np.float32)
    st = vector(old, vlen(dtype))
    h = seq.seq_scan_create(N, C, 1, S, dtype, slots=N)
    seq.seq_scan_step(h, t["x"].t, t["dt"].t, A, t["B"].t, t["C"].t, st, Y.t, **opt)
    args, ref = (p["x"], p["dt"], p["A"], p["B"], p["Cm"]), dict(ref, state=old)
    (y, after), (my, ma) = oracle.scan(*args, **ref), oracle.scan(*args, **ref, mag=True)
    close(Y.get(), y, bound(1) * my, dtype == seq.SEQ_BF16, "y")
    close(st.double().cpu().numpy()[..., :C], after, bound(1) * ma, False, "state")


@pytest.mark.parametrize("dtype", DTYPES)
def test_states_of_zero_that_would_grow(dtype):
    """A above zero: what a run of positions multiplies a state with passes 2^128, and the state is zero until the last positions."""
    N, C, L, S = 2, 72, 300, 5
    rng, p = data(N, C, L, S, 1, dtype, 8)
    p["A"] = np.float64(np.float32(rng.uniform(0.9, 1.1, (S, C))))
    p["dt"] = np.full_like(p["dt"], 8.0)
    p["x"][:, :L - 4] = 0
    t, opt, A, ref = tensors(p, N, C, L, S, 1, True, False, None, "dense", dtype)
    Y, DY = Seq(N, C, L, dtype), Seq(N, C, L, dtype, "dense", p["dy"])
    h = seq.seq_scan_create(N, C, L, S, dtype, slots=N)
    st = torch.zeros(N, S, h.info.Cp, device="cuda")
    ws = seq.seq_workspace(h).fill_(0xFF)
    seq.seq_scan_fwd(h, t["x"].t, t["dt"].t, A, t["B"].t, t["C"].t, Y.t, ws, z=t["z"].t, state_in=st, state_out=st, **opt)
    args = (p["x"], p["dt"], p["A"], p["B"], p["Cm"])
    (y, after), (my, ma) = oracle.scan(*args, **ref), oracle.scan(*args, **ref, mag=True)
    # (an exponent of 13 binary places, off by its step's two units, its factor's and its product's: 36 units a position, of which there are three)
    close(Y.get(), y, (bound(4) + 128 * U) * my, dtype == seq.SEQ_BF16, "y")
    close(st.double().cpu().numpy()[..., :C], after, (bound(4) + 128 * U) * ma, False, "state")
