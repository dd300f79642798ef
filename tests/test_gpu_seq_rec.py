"""Gated linear recurrence against its definition in 64 bits."""
import numpy as np
import pytest
import torch

import seq_rec_oracle as oracle
from seq_util import DTYPES, Seq, close, ints, lengths_of, nans, rounded, spoil, vector, vlen
from paper_1808_05567_amd import seq

pytestmark = pytest.mark.gpu


def data(N, C, L, dtype, seed):
    rng = np.random.default_rng(seed)
    p = {k: rounded(rng.standard_normal((N, L, C)).astype(np.float32), dtype) for k in ("x", "f", "i", "z", "dy")}
    f32 = lambda x: x.astype(np.float32).astype(np.float64)  # noqa: E731
    # decays from 1 - 1e-4 to e^-4 a position
    p["A"] = f32(-np.exp(rng.uniform(-9, 1.5, C)))
    p["f_bias"], p["i_bias"] = f32(rng.standard_normal(C)), f32(rng.standard_normal(C))
    return rng, p


CASES = [  # N, C, L, z, biases, lengths, state, layout
    (1, 64, 1, True, True, "none", True, "dense"), (2, 5, 7, False, False, "none", True, "slice"), (3, 40, 33, True, True, "ragged", True, "rows"),
    (1, 130, 65, True, True, "none", False, "dense"), (2, 144, 129, False, True, "ragged", True, "slice"), (4, 32, 64, True, False, "clamped", True, "dense"),
    (1, 72, 200, True, True, "none", True, "rows"), (2, 16, 31, True, True, "ragged", False, "dense"), (5, 200, 12, False, True, "ragged", True, "dense"),
    # several rounds of a workgroup's positions, and sequences shared by several workgroups
    (2, 24, 1537, True, True, "ragged", True, "dense"), (1, 40, 512, False, True, "none", True, "dense"), (1, 9, 513, True, True, "none", True, "slice"),
    (2, 72, 300, True, True, "ragged", True, "rows"), (4100, 8, 70, True, False, "ragged", True, "dense"), (4100, 4, 37, True, True, "ragged", True, "rows"),
    (2, 12, 5000, True, True, "ragged", True, "dense"), (3, 100, 1300, True, True, "ragged", True, "rows"), (1, 8, 9001, False, False, "none", True, "slice"),
    (40, 136, 600, True, True, "ragged", True, "dense"),
]


def scratch(h):
    """A workspace of whatever, which no result may show."""
    ws = seq.seq_workspace(h)
    return None if ws is None else ws.fill_(0xFF)


def tensors(p, N, C, L, gate, biases, lengths, layout, dtype):
    t = {k: Seq(N, C, L, dtype, layout, spoil(p[k], lengths)) for k in ("x", "f", "i", "z")}
    v = vlen(dtype)
    opt = {k: vector(p[k], v) if biases else None for k in ("f_bias", "i_bias")}
    ref = dict(z=p["z"] if gate else None, lengths=lengths, **{k: p[k] if biases else None for k in opt})
    return t, opt, vector(p["A"], v), ref


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,C,L,gate,biases,kind,with_state,layout", CASES)
def test_forward(N, C, L, gate, biases, kind, with_state, layout, dtype):
    rng, p = data(N, C, L, dtype, N + C + L)
    lengths = lengths_of(kind, N, L, rng)
    t, opt, A, ref = tensors(p, N, C, L, gate, biases, lengths, layout, dtype)
    Y, slots = Seq(N, C, L, dtype, layout), N + 2
    where = rng.permutation(slots)[:N]
    old = rng.standard_normal((slots, C)).astype(np.float32)
    st = vector(old, vlen(dtype)) if with_state else None
    h = seq.seq_rec_create(N, C, L, dtype, slots=slots, views={k: q.t for k, q in t.items()} | {"y": Y.t})
    seq.seq_rec_fwd(h, t["x"].t, t["f"].t, t["i"].t, A, Y.t, scratch(h), z=t["z"].t if gate else None, state_in=st, state_out=st, slots=ints(where),
                    lengths=ints(lengths), **opt)
    torch.cuda.synchronize()
    (y, after), (ey, ea) = oracle.rec(p["x"], p["f"], p["i"], p["A"], state=old[where] if with_state else None, **ref)
    close(Y.get(), y, ey, dtype == seq.SEQ_BF16, "y")
    if with_state:
        got = st.double().cpu().numpy()[:, :C]
        close(got[where], after, ea, False, "state")
        others = np.setdiff1d(np.arange(slots), where)
        np.testing.assert_array_equal(got[others], old[others].astype(np.float64))
        assert not st[:, C:].any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,C,gate,layout", [(1, 64, True, "dense"), (3, 21, False, "rows"), (4, 160, True, "slice"), (70, 1000, True, "dense")])
def test_steps_follow_the_forward_pass(N, C, gate, layout, dtype):
    L, v = 5, vlen(dtype)
    rng, p = data(N, C, L, dtype, C)
    t, opt, A, ref = tensors(p, N, C, L, gate, True, None, "dense", dtype)
    slots, where = N + 1, np.arange(N)[::-1].copy()
    old = rng.standard_normal((slots, C)).astype(np.float32)
    st = vector(old, v)
    one = {k: Seq(N, C, 1, dtype, layout, np.zeros((N, 1, C))) for k in t}
    Y = Seq(N, C, 1, dtype, layout)
    h = seq.seq_rec_create(N, C, 1, dtype, slots=slots, views={k: q.t for k, q in one.items()} | {"y": Y.t})
    (y, after), (ey, ea) = oracle.rec(p["x"], p["f"], p["i"], p["A"], state=old[where], **ref)
    for l in range(L):
        for k, q in t.items():
            one[k].t.copy_(q.t[:, :, l:l + 1])
        seq.seq_rec_step(h, one["x"].t, one["f"].t, one["i"].t, A, st, Y.t, z=one["z"].t if gate else None, slots=ints(where), **opt)
        close(Y.get()[:, 0], y[:, l], ey[:, l], dtype == seq.SEQ_BF16, "y at %d" % l)
    got = st.double().cpu().numpy()[:, :C]
    close(got[where], after, ea, False, "state")
    np.testing.assert_array_equal(got[N], old[N].astype(np.float64))
    # a row without a slot: zeros, and no state changes
    keep = st.clone()
    seq.seq_rec_step(h, one["x"].t, one["f"].t, one["i"].t, A, st, Y.t, slots=ints([-1] * (N - 1) + [slots]), **opt)
    assert torch.equal(keep, st) and not Y.get().any()


@pytest.mark.parametrize("dtype", DTYPES)
def test_sequences_without_a_slot(dtype):
    """They start from zeros and store nothing; a prompt in two parts is the prompt."""
    N, C, L, first, slots = 3, 40, 50, 21, 4
    rng, p = data(N, C, L, dtype, 5)
    t, opt, A, ref = tensors(p, N, C, L, True, True, None, "dense", dtype)
    where, old = np.array([2, -1, 4]), rng.standard_normal((slots, C)).astype(np.float32)
    st = vector(old, vlen(dtype))
    h = seq.seq_rec_create(N, C, first, dtype, slots=slots, views={k: t["x"].t[:, :, :first] for k in ("x", "f", "i", "z", "y")})
    rest = seq.seq_rec_create(N, C, L - first, dtype, slots=slots, views={k: t["x"].t[:, :, first:] for k in ("x", "f", "i", "z", "y")})
    Y = Seq(N, C, L, dtype)
    for plan, part in ((h, slice(0, first)), (rest, slice(first, L))):
        a = {k: q.t[:, :, part] for k, q in t.items()}
        seq.seq_rec_fwd(plan, a["x"], a["f"], a["i"], A, Y.t[:, :, part], scratch(plan), z=a["z"], state_in=st, state_out=st, slots=ints(where), **opt)
    begin = np.zeros((N, C))
    begin[0] = old[2]
    (y, after), (ey, ea) = oracle.rec(p["x"], p["f"], p["i"], p["A"], state=begin, **ref)
    got = Y.get()
    close(got[0], y[0], ey[0], dtype == seq.SEQ_BF16, "y")
    close(got[1:, :first], y[1:, :first], ey[1:, :first], dtype == seq.SEQ_BF16, "y without a slot")
    s = st.double().cpu().numpy()[:, :C]
    close(s[2], after[0], ea[0], False, "state")
    np.testing.assert_array_equal(s[[0, 1, 3]], old[[0, 1, 3]].astype(np.float64))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,C,L,gate,biases,kind,_,layout", CASES)
def test_gradients(N, C, L, gate, biases, kind, _, layout, dtype):
    rng, p = data(N, C, L, dtype, 2 * N + C + L)
    lengths = lengths_of(kind, N, L, rng)
    t, opt, A, ref = tensors(p, N, C, L, gate, biases, lengths, layout, dtype)
    DY = Seq(N, C, L, dtype, layout, spoil(p["dy"], lengths))
    out = {k: Seq(N, C, L, dtype, layout) for k in ("dx", "df", "di", "dz")}
    h = seq.seq_rec_create(N, C, L, dtype, views={k: q.t for k, q in (t | out).items()} | {"dy": DY.t})
    g = {k: nans(h.info.Cp) for k in ("dA", "df_bias", "di_bias")}
    ws = seq.seq_workspace(h).fill_(0xFF)

    def call():
        seq.seq_rec_bwd(h, t["x"].t, t["f"].t, t["i"].t, A, DY.t, out["dx"].t, out["df"].t, out["di"].t, g["dA"], ws, z=t["z"].t if gate else None,
                        dz=out["dz"].t if gate else None, df_bias=g["df_bias"] if biases else None, di_bias=g["di_bias"] if biases else None,
                        lengths=ints(lengths), **opt)
    call()
    torch.cuda.synchronize()
    want, err = oracle.rec_bwd(p["x"], p["f"], p["i"], p["A"], p["dy"], **ref)
    for k, q in out.items():
        if k in want:
            close(q.get(), want[k], err[k], dtype == seq.SEQ_BF16, k)
    for k, q in g.items():
        if k == "dA" or biases:
            got = q.double().cpu().numpy()
            assert not got[C:].any()
            close(got[:C], want[k], err[k], False, k)
    first = [q.clone() for q in g.values()] + [q.t.clone() for q in out.values()]
    ws.fill_(0xFF)
    call()
    assert all(torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0)) for a, b in zip(first, [q for q in g.values()] + [q.t for q in out.values()]))


@pytest.mark.parametrize("dtype", DTYPES)
def test_the_ends_of_what_parameters_may_be(dtype):
    """A of zero and above (the state stays, nothing comes in), of minus infinity, -1e30 and -1e-30; gates that are shut and open."""
    N, C, L = 2, 48, 40
    rng, p = data(N, C, L, dtype, 3)
    p["A"][:6] = [0, 3.5, -np.inf, np.float32(-1e30), np.float32(-1e-30), np.inf]
    p["f"][0, 3:9], p["f"][1, 5:7], p["i"][0, 10:12], p["i"][1, 20:22] = -80, 80, -80, 80
    p["f"][:, :, 4] = 0.5  # (a gate that is shut times -1e-30 is less than fp32 holds)
    t, opt, A, ref = tensors(p, N, C, L, True, False, None, "dense", dtype)
    Y, DY = Seq(N, C, L, dtype), Seq(N, C, L, dtype, "dense", p["dy"])
    out = {k: Seq(N, C, L, dtype) for k in ("dx", "df", "di", "dz")}
    old = rng.standard_normal((N, C)).astype(np.float32)
    st = vector(old, vlen(dtype))
    h = seq.seq_rec_create(N, C, L, dtype, slots=N)
    dA = nans(h.info.Cp)
    seq.seq_rec_fwd(h, t["x"].t, t["f"].t, t["i"].t, A, Y.t, scratch(h), z=t["z"].t, state_in=st, state_out=st)
    (y, after), (ey, ea) = oracle.rec(p["x"], p["f"], p["i"], p["A"], state=old, **ref)
    close(Y.get(), y, ey, dtype == seq.SEQ_BF16, "y")
    close(st.double().cpu().numpy()[:, :C], after, ea, False, "state")
    np.testing.assert_array_equal(st.cpu().numpy()[:, [0, 1, 5]], old[:, [0, 1, 5]])
    seq.seq_rec_bwd(h, t["x"].t, t["f"].t, t["i"].t, A, DY.t, out["dx"].t, out["df"].t, out["di"].t, dA, seq.seq_workspace(h), z=t["z"].t, dz=out["dz"].t)
    want, err = oracle.rec_bwd(p["x"], p["f"], p["i"], p["A"], p["dy"], **ref)
    for k, q in out.items():
        close(q.get(), want[k], err[k], dtype == seq.SEQ_BF16, k)
    close(dA.double().cpu().numpy()[:C], want["dA"], err["dA"], False, "dA")


def test_an_infinity_stays_in_its_sequence_and_channel():
    N, C, L, dtype = 2, 16, 60, seq.SEQ_F32
    _, p = data(N, C, L, dtype, 4)
    p["x"][0, 20, 3], p["f"][1, 30, 5] = np.inf, np.nan
    t, opt, A, ref = tensors(p, N, C, L, True, True, None, "dense", dtype)
    Y = Seq(N, C, L, dtype)
    h = seq.seq_rec_create(N, C, L, dtype)
    seq.seq_rec_fwd(h, t["x"].t, t["f"].t, t["i"].t, A, Y.t, scratch(h), z=t["z"].t, **opt)
    got = Y.get()
    assert np.isfinite(got[0, :20]).all() and not np.isfinite(got[0, 20, 3]) and not np.isfinite(got[1, 30:, 5]).any()
    got[0, 20:, 3] = got[1, 30:, 5] = 0
    assert np.isfinite(got).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_captured_and_replayed_beside_another_graph(dtype):
    """Forward and backward on a side stream, two graphs with workspaces of their own, replayed in turn with eager work between."""
    N, C, L = 2, 40, 2100
    runs = []
    for seed in (1, 2):
        _, p = data(N, C, L, dtype, seed)
        lengths = np.array([L, 1333])
        t, opt, A, ref = tensors(p, N, C, L, True, True, lengths, "dense", dtype)
        Y, DY = Seq(N, C, L, dtype), Seq(N, C, L, dtype, "dense", spoil(p["dy"], lengths))
        out = {k: Seq(N, C, L, dtype) for k in ("dx", "df", "di", "dz")}
        h = seq.seq_rec_create(N, C, L, dtype, slots=N)
        g = {k: nans(h.info.Cp) for k in ("dA", "df_bias", "di_bias")}
        ws, n, st = seq.seq_workspace(h), ints(lengths), torch.zeros(N, h.info.Cp, device="cuda")

        def call(h=h, t=t, A=A, Y=Y, DY=DY, out=out, g=g, ws=ws, n=n, st=st, opt=opt):
            seq.seq_rec_fwd(h, t["x"].t, t["f"].t, t["i"].t, A, Y.t, ws, z=t["z"].t, state_out=st, lengths=n, **opt)
            seq.seq_rec_bwd(h, t["x"].t, t["f"].t, t["i"].t, A, DY.t, out["dx"].t, out["df"].t, out["di"].t, g["dA"], ws, z=t["z"].t, dz=out["dz"].t,
                            df_bias=g["df_bias"], di_bias=g["di_bias"], lengths=n, **opt)
        results = [Y.t, st] + [q.t for q in out.values()] + list(g.values())
        call()
        torch.cuda.synchronize()
        want = [q.clone() for q in results]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        runs.append((graph, results, want, call))
    for k in range(6):
        graph, results, want, call = runs[k % 2]
        for q in results:
            q.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, want)), k
        runs[1 - k % 2][3]()
        torch.cuda.synchronize()
