"""Selective scan against its definition in 64 bits."""
import numpy as np
import pytest
import torch

import seq_oracle as oracle
from seq_util import DTYPES, Seq, close, ints, lengths_of, nans, rounded, spoil, vector, vlen
from paper_1808_05567_amd import seq

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
# A position multiplies the state by an exponential (its argument, scaled once, and the instruction: 3 units and one a unit of the exponent, that
# is at most 8 here) and adds a product of three (3 units): 12 units a position on the way from an input to a result, some 32 for the
# sums over at most 64 states, the step's softplus and the gate.
STEP, REST = 12, 48


def bound(L):
    return (STEP * L + REST) * U


def data(N, C, L, S, G, dtype, seed):
    rng = np.random.default_rng(seed)
    f = lambda *s: rng.standard_normal(s)  # noqa: E731
    p = {k: rounded(f(N, L, C), dtype) for k in ("x", "z", "dy")}
    p["dt"] = rounded(0.5 * f(N, L, C), dtype)
    p["B"], p["Cm"] = rounded(f(N, L, G * S), dtype), rounded(f(N, L, G * S), dtype)
    f32 = lambda x: x.astype(np.float32).astype(np.float64)  # noqa: E731
    p["A"] = f32(-np.exp(rng.uniform(-3, 2, (S, C))))
    p["D"], p["dt_bias"] = f32(f(C)), f32(rng.uniform(-6, 0.5, C))
    return rng, p


CASES = [  # N, C, L, S, G, z, D and bias, softplus, lengths, state, layout
    (1, 64, 1, 16, 1, True, True, True, "none", True, "dense"), (2, 5, 7, 4, 1, False, False, True, "none", True, "slice"),
    (3, 40, 33, 16, 1, True, True, True, "ragged", True, "rows"), (1, 130, 65, 16, 1, True, True, True, "none", False, "dense"),
    (2, 144, 129, 8, 2, False, True, True, "ragged", True, "slice"), (4, 32, 64, 24, 4, True, True, True, "clamped", True, "dense"),
    (1, 72, 200, 64, 1, True, False, True, "none", True, "rows"), (2, 16, 300, 1, 2, True, True, False, "ragged", True, "dense"),
    (5, 200, 12, 17, 1, False, True, True, "ragged", True, "dense"), (1, 96, 513, 12, 3, True, True, True, "none", True, "slice"),
    (3, 8, 70, 33, 1, True, True, False, "ragged", False, "rows"),
]


def tensors(p, N, C, L, S, G, gate, extra, lengths, layout, dtype):
    make = lambda k, c=C: Seq(N, c, L, dtype, layout, spoil(p[k], lengths))  # noqa: E731
    t = {"x": make("x"), "dt": make("dt"), "B": make("B", G * S), "C": make("Cm", G * S), "z": make("z") if gate else None}
    v = vlen(dtype)
    opt = {"D": vector(p["D"], v) if extra else None, "dt_bias": vector(p["dt_bias"], v) if extra else None}
    ref = dict(D=p["D"] if extra else None, dt_bias=p["dt_bias"] if extra else None, z=p["z"] if gate else None, G=G, lengths=lengths)
    return t, opt, vector(p["A"], v), ref


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,C,L,S,G,gate,extra,sp,kind,with_state,layout", CASES)
def test_forward(N, C, L, S, G, gate, extra, sp, kind, with_state, layout, dtype):
    rng, p = data(N, C, L, S, G, dtype, N + C + L)
    if not sp:
        p["dt"] = rounded(np.abs(p["dt"]) * 0.1, dtype)
        p["dt_bias"] = np.abs(p["dt_bias"])
    v, lengths = vlen(dtype), lengths_of(kind, N, L, rng)
    t, opt, A, ref = tensors(p, N, C, L, S, G, gate, extra, lengths, layout, dtype)
    Y, slots = Seq(N, C, L, dtype, layout), N + 2
    where = rng.permutation(slots)[:N]
    old = rng.standard_normal((slots, S, C)).astype(np.float32)
    st = vector(old, v) if with_state else None
    h = seq.seq_scan_create(N, C, L, S, dtype, G=G, softplus=sp, slots=slots, views={k: q.t for k, q in t.items() if q} | {"y": Y.t})
    ws = seq.seq_workspace(h)
    if ws is not None:
        ws.fill_(0xFF)
    z = t["z"].t if gate else None
    seq.seq_scan_fwd(h, t["x"].t, t["dt"].t, A, t["B"].t, t["C"].t, Y.t, ws, z=z, state_in=st, state_out=st, slots=ints(where), lengths=ints(lengths), **opt)
    torch.cuda.synchronize()
    args = (p["x"], p["dt"], p["A"], p["B"], p["Cm"])
    ref.update(use_softplus=sp, state=old[where] if with_state else None)
    y, after = oracle.scan(*args, **ref)
    my, ma = oracle.scan(*args, **ref, mag=True)
    close(Y.get(), y, bound(L) * my, dtype == seq.SEQ_BF16, "y")
    if with_state:
        got = st.double().cpu().numpy()[..., :C]
        close(got[where], after, bound(L) * ma, False, "state")
        others = np.setdiff1d(np.arange(slots), where)
        np.testing.assert_array_equal(got[others], old[others].astype(np.float64))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,C,S,G,gate,layout", [(1, 64, 16, 1, True, "dense"), (3, 21, 5, 1, False, "rows"), (4, 160, 64, 2, True, "slice"), (2, 48, 1, 3, True, "dense")])
def test_steps_follow_the_forward_pass(N, C, S, G, gate, layout, dtype):
    L, v = 6, vlen(dtype)
    rng, p = data(N, C, L, S, G, dtype, C + S)
    t, opt, A, ref = tensors(p, N, C, L, S, G, gate, True, None, "dense", dtype)
    slots = N + 1
    where = np.arange(N)[::-1].copy()
    old = rng.standard_normal((slots, S, C)).astype(np.float32)
    st = vector(old, v)
    one = {k: Seq(N, q.C, 1, dtype, layout, np.zeros((N, 1, q.C))) if q else None for k, q in t.items()}
    Y = Seq(N, C, 1, dtype, layout)
    h = seq.seq_scan_create(N, C, 1, S, dtype, G=G, slots=slots, views={k: q.t for k, q in one.items() if q} | {"y": Y.t})
    args = (p["x"], p["dt"], p["A"], p["B"], p["Cm"])
    ref["state"] = old[where]
    y, after = oracle.scan(*args, **ref)
    my, ma = oracle.scan(*args, **ref, mag=True)
    for l in range(L):
        for k, q in t.items():
            if q:
                one[k].t.copy_(q.t[:, :, l:l + 1])
        seq.seq_scan_step(h, one["x"].t, one["dt"].t, A, one["B"].t, one["C"].t, st, Y.t, z=one["z"].t if gate else None, slots=ints(where), **opt)
        close(Y.get()[:, 0], y[:, l], bound(L) * my[:, l], dtype == seq.SEQ_BF16, "y at %d" % l)
    got = st.double().cpu().numpy()[..., :C]
    close(got[where], after, bound(L) * ma, False, "state")
    np.testing.assert_array_equal(got[N], old[N].astype(np.float64))
    # a row without a slot: zeros, and no state changes
    keep = st.clone()
    seq.seq_scan_step(h, one["x"].t, one["dt"].t, A, one["B"].t, one["C"].t, st, Y.t, slots=ints([-1] * (N - 1) + [slots]), **opt)
    assert torch.equal(keep, st) and not Y.get().any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,C,L,S,G,gate,extra,sp,kind,_,layout", CASES)
def test_gradients(N, C, L, S, G, gate, extra, sp, kind, _, layout, dtype):
    rng, p = data(N, C, L, S, G, dtype, 2 * N + C + L)
    if not sp:
        p["dt"] = rounded(np.abs(p["dt"]) * 0.1, dtype)
        p["dt_bias"] = np.abs(p["dt_bias"])
    v, lengths, bf16 = vlen(dtype), lengths_of(kind, N, L, rng), dtype == seq.SEQ_BF16
    t, opt, A, ref = tensors(p, N, C, L, S, G, gate, extra, lengths, layout, dtype)
    DY = Seq(N, C, L, dtype, layout, spoil(p["dy"], lengths))
    out = {k: Seq(N, c, L, dtype, layout) for k, c in (("dx", C), ("ddt", C), ("dB", G * S), ("dC", G * S))}
    out["dz"] = Seq(N, C, L, dtype, layout) if gate else None
    h = seq.seq_scan_create(N, C, L, S, dtype, G=G, softplus=sp, views={k: q.t for k, q in {**t, **out, "dy": DY}.items() if q})
    Cp = h.info.Cp
    dA, dD, db = nans(S, Cp), nans(Cp), nans(Cp)
    ws = seq.seq_workspace(h).fill_(0xFF)

    def call():
        seq.seq_scan_bwd(h, t["x"].t, t["dt"].t, A, t["B"].t, t["C"].t, DY.t, out["dx"].t, out["ddt"].t, dA, out["dB"].t, out["dC"].t, ws,
                         z=t["z"].t if gate else None, dD=dD, dz=out["dz"].t if gate else None, ddt_bias=db, lengths=ints(lengths), **opt)
    call()
    torch.cuda.synchronize()
    args = (p["x"], p["dt"], p["A"], p["B"], p["Cm"], p["dy"])
    r = oracle.scan_bwd(*args, use_softplus=sp, **ref)
    m = oracle.scan_bwd(*args, use_softplus=sp, **ref, mag=True)
    for k in ("dx", "ddt", "dB", "dC", "dz"):
        if out[k] is not None:
            # (there and back, and a sum over channels)
            close(out[k].get(), r[k], (2 * bound(L) + C * U) * m[k], bf16, k)
    for k, got in (("dA", dA), ("dD", dD), ("ddt_bias", db)):
        got = got.double().cpu().numpy()
        assert not got[..., C:].any()
        close(got[..., :C], r[k], (2 * bound(L) + N * L * U) * m[k], False, k)
    first = [dA.clone()] + [q.t.clone() for q in out.values() if q]
    ws.fill_(0xFF)
    call()
    assert all(torch.equal(a, b) for a, b in zip(first, [dA] + [q.t for q in out.values() if q]))


@pytest.mark.parametrize("axis", ["n", "c", "l"])
def test_distances_beyond_32_bits(axis):
    """A tensor's elements pass 2^32 by each distance of a view alone: sequences far apart, many blocks or positions as far as they may be."""
    dtype, S, far = seq.SEQ_BF16, 5, 1 << 24
    N, C, L = {"n": (2, 16, 12), "c": (1, 260 * 8, 2), "l": (1, 8, 260)}[axis]
    shape = {"n": ((1 << 32) + 64, 96, 8), "c": (0, far, 8), "l": (0, 8, far)}[axis]
    need = {"n": (1 << 32) + 512, "c": 260 * far, "l": 260 * far}[axis]
    rng, p = data(N, C, L, S, 1, dtype, 5)
    base, offsets = torch.empty(need + 16384, dtype=torch.bfloat16, device="cuda"), iter(range(0, 16384, 1024))

    def tensor(data=None, channels=C):
        t = base.as_strided((N, channels // 8, L, 8), shape + (1,), next(offsets))
        if data is not None:
            t.copy_(torch.from_numpy(data).view(N, L, channels // 8, 8).permute(0, 2, 1, 3))
        return t
    x, dt, dy = (tensor(p[k]) for k in ("x", "dt", "dy"))
    y, ddt = tensor(), tensor()
    B, Cm = (Seq(N, S, L, dtype, "dense", p[k]).t for k in ("B", "Cm"))
    dB, dC = Seq(N, S, L, dtype), Seq(N, S, L, dtype)
    h = seq.seq_scan_create(N, C, L, S, dtype, views={"x": x, "dt": dt, "y": y, "dy": dy, "dx": y, "ddt": ddt})
    back = lambda t: t.permute(0, 2, 1, 3).reshape(N, L, C).double().cpu().numpy()  # noqa: E731
    ws, A = seq.seq_workspace(h), vector(p["A"], 8)
    seq.seq_scan_fwd(h, x, dt, A, B, Cm, y, ws)
    args = (p["x"], p["dt"], p["A"], p["B"], p["Cm"])
    close(back(y), oracle.scan(*args)[0], bound(L) * oracle.scan(*args, mag=True)[0], True)
    seq.seq_scan_bwd(h, x, dt, A, B, Cm, dy, y, ddt, nans(S, C), dB.t, dC.t, ws)
    r, m = oracle.scan_bwd(*args, p["dy"]), oracle.scan_bwd(*args, p["dy"], mag=True)
    for k, got in (("dx", back(y)), ("ddt", back(ddt)), ("dB", dB.get()), ("dC", dC.get())):
        close(got, r[k], (2 * bound(L) + C * U) * m[k], True, k)


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_runs(dtype):
    """Sequences in more runs than 16 waves take at once, in both directions; the second one ends early."""
    N, C, L, S = 2, 8, 20011, 3
    rng, p = data(N, C, L, S, 1, dtype, 6)
    p["A"] = np.float64(np.float32(-np.logspace(-4, 0, S)[:, None] * np.ones((1, C))))
    lengths = np.array([L, L - 7000])
    t, opt, A, ref = tensors(p, N, C, L, S, 1, True, True, lengths, "dense", dtype)
    Y, DY = Seq(N, C, L, dtype), Seq(N, C, L, dtype, "dense", spoil(p["dy"], lengths))
    out = {k: Seq(N, c, L, dtype) for k, c in (("dx", C), ("ddt", C), ("dz", C), ("dB", S), ("dC", S))}
    h = seq.seq_scan_create(N, C, L, S, dtype)
    ws = seq.seq_workspace(h).fill_(0xFF)
    seq.seq_scan_fwd(h, t["x"].t, t["dt"].t, A, t["B"].t, t["C"].t, Y.t, ws, z=t["z"].t, lengths=ints(lengths), **opt)
    args = (p["x"], p["dt"], p["A"], p["B"], p["Cm"])
    close(Y.get(), oracle.scan(*args, **ref)[0], bound(L) * oracle.scan(*args, **ref, mag=True)[0], dtype == seq.SEQ_BF16, "y")
    dA, dD, db = nans(S, h.info.Cp), nans(h.info.Cp), nans(h.info.Cp)
    seq.seq_scan_bwd(h, t["x"].t, t["dt"].t, A, t["B"].t, t["C"].t, DY.t, out["dx"].t, out["ddt"].t, dA, out["dB"].t, out["dC"].t, ws,
                     z=t["z"].t, dD=dD, dz=out["dz"].t, ddt_bias=db, lengths=ints(lengths), **opt)
    r, m = oracle.scan_bwd(*args, p["dy"], **ref), oracle.scan_bwd(*args, p["dy"], **ref, mag=True)
    for k, q in out.items():
        close(q.get(), r[k], (2 * bound(L) + C * U) * m[k], dtype == seq.SEQ_BF16, k)
    for k, got in (("dA", dA), ("dD", dD), ("ddt_bias", db)):
        close(got.double().cpu().numpy()[..., :C], r[k], (2 * bound(L) + N * L * U) * m[k], False, k)


def test_long_decays_and_large_steps():
    """States that nothing leaves and steps that leave nothing of a state: exp(d A) from 1 - 1e-6 to 0."""
    N, C, L, S, dtype = 1, 64, 700, 16, seq.SEQ_F32
    rng, p = data(N, C, L, S, 1, dtype, 1)
    p["A"] = np.float64(np.float32(-np.logspace(-5, 4, S)[:, None] * np.ones((1, C))))
    t, opt, A, ref = tensors(p, N, C, L, S, 1, True, True, None, "dense", dtype)
    Y = Seq(N, C, L, dtype)
    h = seq.seq_scan_create(N, C, L, S, dtype)
    seq.seq_scan_fwd(h, t["x"].t, t["dt"].t, A, t["B"].t, t["C"].t, Y.t, seq.seq_workspace(h), z=t["z"].t, **opt)
    args = (p["x"], p["dt"], p["A"], p["B"], p["Cm"])
    close(Y.get(), oracle.scan(*args, **ref)[0], bound(L) * oracle.scan(*args, **ref, mag=True)[0], False)


@pytest.mark.parametrize("dtype", DTYPES)
def test_another_stream_and_a_graph(dtype):
    """On a stream of its own, then recorded: replays give what the calls give, whatever ran between."""
    N, C, L, S = 2, 72, 150, 16
    rng, p = data(N, C, L, S, 1, dtype, 9)
    t, opt, A, ref = tensors(p, N, C, L, S, 1, True, True, None, "dense", dtype)
    Y = Seq(N, C, L, dtype)
    h = seq.seq_scan_create(N, C, L, S, dtype)
    ws = seq.seq_workspace(h)

    def call():
        seq.seq_scan_fwd(h, t["x"].t, t["dt"].t, A, t["B"].t, t["C"].t, Y.t, ws, z=t["z"].t, **opt)
    call()
    want = Y.t.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        Y.t.zero_()
        call()
        assert torch.equal(Y.t, want)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        Y.t.zero_()
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y.t, want)
