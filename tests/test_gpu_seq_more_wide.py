"""The recurrence, the layer norm and AdamW where tensors are large or far apart, in other layouts side by side, and on other streams."""
import numpy as np
import pytest
import torch

import seq_rec_oracle as oracle
from seq_util import DTYPES, TORCH, Seq, close, ints, nans, rounded, spoil, vector, vlen
from test_gpu_seq_adamw import BLOCK
from test_gpu_seq_rec import data, scratch, tensors
from paper_1808_05567_amd import seq

pytestmark = pytest.mark.gpu
U, EPS = 2.0 ** -24, 1e-5
INPUTS, GRADS = ("x", "f", "i", "z"), ("dx", "df", "di", "dz")


def run_rec(p, t, Y, DY, out, N, C, L, dtype, lengths, some, opt, A, ref):
    """Forward and gradients against the oracle at the channels `some`."""
    h = seq.seq_rec_create(N, C, L, dtype, slots=N, views={k: q.t for k, q in (t | out).items()} | {"y": Y.t, "dy": DY.t})
    ws, n, bf16 = scratch(h), ints(lengths), dtype == seq.SEQ_BF16
    g = {k: nans(h.info.Cp) for k in ("dA", "df_bias", "di_bias")}
    st = torch.zeros(N, h.info.Cp, device="cuda")
    seq.seq_rec_fwd(h, t["x"].t, t["f"].t, t["i"].t, A, Y.t, ws, z=t["z"].t, state_out=st, lengths=n, **opt)
    seq.seq_rec_bwd(h, t["x"].t, t["f"].t, t["i"].t, A, DY.t, out["dx"].t, out["df"].t, out["di"].t, g["dA"], ws, z=t["z"].t, dz=out["dz"].t,
                    df_bias=g["df_bias"], di_bias=g["di_bias"], lengths=n, **opt)
    torch.cuda.synchronize()
    pick = {k: q[..., some] for k, q in p.items()}
    ref = dict(z=pick["z"], lengths=lengths, f_bias=pick["f_bias"], i_bias=pick["i_bias"])
    args = [pick[k] for k in ("x", "f", "i", "A")]
    (y, after), (ey, ea) = oracle.rec(*args, **ref)
    close(Y.get()[..., some], y, ey, bf16, "y")
    close(st.double().cpu().numpy()[:, some], after, ea, False, "state")
    want, err = oracle.rec_bwd(*args, pick["dy"], **ref)
    for k, q in out.items():
        close(q.get()[..., some], want[k], err[k], bf16, k)
    for k, q in g.items():
        close(q.double().cpu().numpy()[some], want[k], err[k], False, k)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["dense", "rows"])
def test_recurrence_of_more_than_16_megabytes(layout, dtype):
    """Results past the caches, compared at every 97th channel."""
    N, C, L = 3, 1044, 2900
    _, p = data(N, C, L, dtype, 1)
    lengths = np.array([L, L - 7, 5])
    t, opt, A, ref = tensors(p, N, C, L, True, True, lengths, layout, dtype)
    Y, DY = Seq(N, C, L, dtype, layout), Seq(N, C, L, dtype, layout, spoil(p["dy"], lengths))
    out = {k: Seq(N, C, L, dtype, layout) for k in GRADS}
    run_rec(p, t, Y, DY, out, N, C, L, dtype, lengths, np.arange(0, C, 97), opt, A, ref)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout,N,blocks,L", [("dense", 24, 8, 1100), ("dense", 256, 1, 700), ("dense", 257, 1, 150), ("rows", 200, 6, 300), ("rows", 191, 8, 100)])
def test_recurrence_of_about_as_many_workgroups_as_compute_units(layout, N, blocks, L, dtype):
    """Backwards in workgroups of more waves, and one workgroup beside where that ends."""
    C = blocks * vlen(dtype) - 1
    rng, p = data(N, C, L, dtype, N)
    lengths = rng.integers(0, L + 1, N)
    lengths[:3] = L, 0, 1
    t, opt, A, ref = tensors(p, N, C, L, True, True, lengths, layout, dtype)
    Y, DY = Seq(N, C, L, dtype, layout), Seq(N, C, L, dtype, layout, spoil(p["dy"], lengths))
    run_rec(p, t, Y, DY, {k: Seq(N, C, L, dtype, layout) for k in GRADS}, N, C, L, dtype, lengths, np.arange(C), opt, A, ref)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("first", ["dense", "rows", "slice"])
def test_recurrence_of_tensors_in_different_layouts(first, dtype):
    """x decides how lanes are laid out; the others lie as they may."""
    N, C, L = 2, 92, 333
    _, p = data(N, C, L, dtype, 2)
    lengths, others = np.array([L, 200]), {"dense": "rows", "rows": "slice", "slice": "rows"}[first]
    t = {k: Seq(N, C, L, dtype, first if k == "x" else others, spoil(p[k], lengths)) for k in INPUTS}
    _, opt, A, ref = tensors(p, N, C, L, True, True, lengths, "dense", dtype)
    Y, DY = Seq(N, C, L, dtype, others), Seq(N, C, L, dtype, "dense", spoil(p["dy"], lengths))
    out = {k: Seq(N, C, L, dtype, "slice" if k == "df" else first) for k in GRADS}
    run_rec(p, t, Y, DY, out, N, C, L, dtype, lengths, np.arange(C), opt, A, ref)


@pytest.mark.parametrize("dtype", DTYPES)
def test_recurrence_of_one_gate_for_all_positions(dtype):
    """f expanded over positions, i over sequences: distances of zero."""
    N, C, L = 2, 40, 130
    _, p = data(N, C, L, dtype, 3)
    p["f"][:], p["i"][:] = p["f"][:, :1], p["i"][:1]
    t, opt, A, ref = tensors(p, N, C, L, True, True, None, "dense", dtype)
    t["f"].t, t["i"].t = t["f"].t[:, :, :1].expand_as(t["f"].t), t["i"].t[:1].expand_as(t["i"].t)
    Y, DY = Seq(N, C, L, dtype), Seq(N, C, L, dtype, "dense", p["dy"])
    run_rec(p, t, Y, DY, {k: Seq(N, C, L, dtype) for k in GRADS}, N, C, L, dtype, None, np.arange(C), opt, A, ref)


class Far:
    """[N, Cb, L, v] in a large memory: places that are more than 2^32 bytes apart."""
    base = None

    def __init__(self, at, N, C, L, strides, data=None):
        self.C, self.t = C, Far.base[at:].as_strided((N, -(-C // 8), L, 8), (*strides, 1))
        if data is None:
            self.t.fill_(float("nan"))
        else:
            full = np.zeros((N, L, self.t.shape[1] * 8))
            full[..., :C] = data
            self.t.copy_(torch.from_numpy(full).view(N, L, -1, 8).permute(0, 2, 1, 3))

    def get(self):
        N, Cb, L, v = self.t.shape
        return self.t.permute(0, 2, 1, 3).reshape(N, L, Cb * v).double().cpu().numpy()[..., :self.C]


@pytest.mark.parametrize("strides", [((1 << 31) + 4096, 8 << 10, 8), (1 << 15, 1 << 13, 1 << 20), (1 << 15, 1 << 10, 1 << 20)], ids=["sequences", "positions", "rows"])
def test_places_that_32_bits_do_not_reach(strides):
    """The recurrence and the layer norm in bf16: sequences 2^31 numbers apart, and 2200 positions 2^20."""
    N, C, L, dtype = 2, 24, 2200 if strides[2] > 8 else 600, seq.SEQ_BF16
    Far.base = torch.empty((1 << 31) + (1 << 29), dtype=torch.bfloat16, device="cuda")
    _, p = data(N, C, L, dtype, 4)
    lengths, at = np.array([L - 3, L]), iter(range(0, 10 << 16, 1 << 16))
    t = {k: Far(next(at), N, C, L, strides, p[k]) for k in INPUTS}
    Y, DY, out = Far(next(at), N, C, L, strides), Far(next(at), N, C, L, strides, p["dy"]), {k: Far(next(at), N, C, L, strides) for k in GRADS}
    _, opt, A, ref = tensors(p, N, C, L, True, True, lengths, "dense", dtype)
    run_rec(p, t, Y, DY, out, N, C, L, dtype, lengths, np.arange(C), opt, A, ref)
    h = seq.seq_lnorm_create(N, C, L, dtype, EPS, views={"x": t["x"].t, "y": Y.t, "r": t["x"].t, "dy": DY.t, "dx": out["dx"].t})
    w, wv = np.float64(np.float32(np.random.default_rng(1).standard_normal(C))), None
    wv = vector(w, 8)
    Y.t.fill_(float("nan"))
    seq.seq_lnorm_fwd(h, t["x"].t, None, wv, None, None, Y.t)
    y, ey = oracle.lnorm(p["x"], w, None, EPS)
    close(Y.get(), y, ey, True, "lnorm")
    dw = nans(h.info.Cp)
    seq.seq_lnorm_bwd(h, t["x"].t, wv, DY.t, None, out["dx"].t, dw, None, scratch(h))
    want, err = oracle.lnorm_bwd(p["x"], w, p["dy"], None, EPS)
    close(out["dx"].get(), want[0], err[0], True, "dx")
    close(dw.double().cpu().numpy(), want[1], err[1], False, "dw")
    Far.base = None


def test_a_tensor_of_more_than_4_gigabytes():
    """AdamW in 8 bits, its numbers compared where 32 bits of bytes and of numbers end, and against a small tensor of the same numbers."""
    n = (1 << 30) + 700
    h = seq.seq_adamw_create([5, n], seq.SEQ_BF16, 8, decay=[0.0, 0.1])
    p, g = torch.full((n,), 0.5, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    where = [0, (1 << 29) - 256, (1 << 30) - 512, n - 188 - 256, n - 188]  # (blocks, the last one a part of one)
    gen = torch.Generator("cuda").manual_seed(1)
    for a in where:
        g[a:a + 256] = torch.randn(min(256, n - a), device="cuda", generator=gen).to(torch.bfloat16)
    m, v, scales = seq.seq_adamw_states(h)
    first = torch.ones(5, device="cuda"), torch.ones(5, device="cuda", dtype=torch.bfloat16)
    seq.seq_adamw(h, seq.seq_adamw_tensors(h, [first[0], p], [first[1], g]), m, v, (1e-2, 3), scales=scales)
    for a in where:
        size = min(256, n - a)
        one = seq.seq_adamw_create([size], seq.SEQ_BF16, 8, decay=0.1)
        q = torch.full((size,), 0.5, device="cuda")
        sm, sv, ss = seq.seq_adamw_states(one)
        seq.seq_adamw(one, seq.seq_adamw_tensors(one, [q], [g[a:a + size].clone()]), sm, sv, (1e-2, 3), scales=ss)
        b = 1 + a // BLOCK
        assert torch.equal(p[a:a + size], q) and torch.equal(m[b * BLOCK:][:256], sm) and torch.equal(v[b * BLOCK:][:256], sv)
        assert torch.equal(scales.view(2, -1)[:, b], ss.view(2)) and float(ss.min()) > 0
    assert bool((p[1000:2000] == 0.5 - torch.tensor(1e-2, device="cuda") * torch.tensor(0.1, device="cuda") * 0.5).all())


def test_calls_at_once_on_other_streams():
    """Two plans of each operator on two streams, each with its own tensors and workspace: what they give one after the other."""
    N, C, L, dtype = 2, 136, 1500, seq.SEQ_BF16
    jobs = []
    for seed in (1, 2):
        _, p = data(N, C, L, dtype, seed)
        t, opt, A, _ = tensors(p, N, C, L, True, True, None, "dense", dtype)
        Y, DY, out = Seq(N, C, L, dtype), Seq(N, C, L, dtype, "dense", p["dy"]), {k: Seq(N, C, L, dtype) for k in GRADS}
        h, norm = seq.seq_rec_create(N, C, L, dtype, slots=N), seq.seq_lnorm_create(N, C, L, dtype, EPS)
        adam = seq.seq_adamw_create([3000, 7], dtype, 8)
        g, w = {k: nans(h.info.Cp) for k in ("dA", "df_bias", "di_bias", "dw", "db")}, torch.ones(h.info.Cp, device="cuda")
        ws, nws, U1, D1 = scratch(h), scratch(norm), Seq(N, C, L, dtype), Seq(N, C, L, dtype)
        gen = torch.Generator("cuda").manual_seed(seed)
        ps = [torch.randn(n, device="cuda", generator=gen) for n in (3000, 7)]
        gs = [torch.randn(n, device="cuda", generator=gen).to(TORCH[dtype]) for n in (3000, 7)]
        states = seq.seq_adamw_states(adam)
        start = [q.clone() for q in ps] + [q.clone() for q in states]

        def call(stream, h=h, norm=norm, adam=adam, t=t, A=A, Y=Y, DY=DY, out=out, g=g, w=w, ws=ws, nws=nws, U1=U1, D1=D1, ps=ps, gs=gs, states=states, opt=opt, start=start):
            with torch.cuda.stream(stream):
                for q, s in zip(ps + list(states), start):
                    q.copy_(s)
                for _ in range(5):
                    seq.seq_lnorm_fwd(norm, t["x"].t, t["z"].t, w, None, U1.t, Y.t)
                    seq.seq_rec_fwd(h, t["x"].t, t["f"].t, t["i"].t, A, Y.t, ws, z=t["z"].t, **opt)
                    seq.seq_rec_bwd(h, t["x"].t, t["f"].t, t["i"].t, A, DY.t, out["dx"].t, out["df"].t, out["di"].t, g["dA"], ws, z=t["z"].t, dz=out["dz"].t,
                                    df_bias=g["df_bias"], di_bias=g["di_bias"], **opt)
                    seq.seq_lnorm_bwd(norm, U1.t, w, DY.t, None, D1.t, g["dw"], g["db"], nws)
                    seq.seq_adamw(adam, seq.seq_adamw_tensors(adam, ps, gs), states[0], states[1], (1e-3, 1), scales=states[2])
        jobs.append((call, [Y.t, U1.t, D1.t] + [q.t for q in out.values()] + list(g.values()) + ps + list(states)))
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    want = []
    for call, results in jobs:
        call(torch.cuda.current_stream())
        torch.cuda.synchronize()
        want.append([q.clone() for q in results])
    for _, results in jobs:
        for q in results:
            if q.is_floating_point():
                q.fill_(0.25)
    torch.cuda.synchronize()
    for (call, _), s in zip(jobs, streams):
        call(s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for (_, results), w in zip(jobs, want) for a, b in zip(results, w))


def test_a_gradient_that_is_not_finite():
    """In 32 bits it spoils its own number; in 8 the states of the 256 numbers that share its scale, from the next step on."""
    n, at = 700, 300
    for bits in (32, 8):
        for what in (float("inf"), float("-inf"), float("nan")):
            h = seq.seq_adamw_create([n], seq.SEQ_F32, bits, decay=0.1)
            gen = torch.Generator("cuda").manual_seed(1)
            p, g = torch.randn(n, device="cuda", generator=gen), torch.randn(n, device="cuda", generator=gen)
            runs = []
            for spoilt in (False, True):
                q, d = p.clone(), g.clone()
                if spoilt:
                    d[at] = what
                m, v, scales = seq.seq_adamw_states(h)
                seq.seq_adamw(h, seq.seq_adamw_tensors(h, [q], [d]), m, v, (1e-2, 1), scales=scales)
                first = q.clone()
                seq.seq_adamw(h, seq.seq_adamw_tensors(h, [q], [g]), m, v, (1e-2, 2), scales=scales)
                runs.append((first, q))
            (a, b), (c, d) = runs
            others = torch.arange(n, device="cuda") != at
            assert torch.equal(a[others], c[others]) and not c[at].isfinite() and not d[at].isfinite()
            far = others if bits == 32 else (torch.arange(n, device="cuda") < 256) | (torch.arange(n, device="cuda") >= 512)
            assert torch.equal(b[far], d[far]) and (bits == 32 or bool(d[256:512].isnan().all()))


def test_tensors_whose_memory_is_replaced_stay_where_they_were():
    h = seq.seq_adamw_create([300], seq.SEQ_F32)
    p, g = torch.ones(300, device="cuda"), torch.ones(300, device="cuda")
    tensors, (m, v, _) = seq.seq_adamw_tensors(h, [p], [g]), seq.seq_adamw_states(h)
    old = p.detach()
    p.data = torch.zeros(300, device="cuda")
    seq.seq_adamw(h, tensors, m, v, (1e-2, 1))
    assert not p.any() and bool((old < 1).all())


@pytest.mark.parametrize("N,C,L,layout,dtype", [
    (9, 1100, 1000, "rows", seq.SEQ_BF16), (9, 700, 1000, "rows", seq.SEQ_F32), (33, 20, 1000, "rows", seq.SEQ_BF16), (33, 300, 1000, "slice", seq.SEQ_F32),
    (9, 2900, 1001, "rows", seq.SEQ_BF16), (4, 1500, 2200, "dense", seq.SEQ_F32), (40, 4, 900, "dense", seq.SEQ_F32)])
def test_layer_norm_of_many_positions(N, C, L, layout, dtype):
    """Gradients in more workgroups, inputs past the caches."""
    bf16, v = dtype == seq.SEQ_BF16, vlen(dtype)
    rng = np.random.default_rng(N + C)
    x, dy = rounded(rng.standard_normal((N, L, C)), dtype), rounded(rng.standard_normal((N, L, C)), dtype)
    w, b = (np.float32(rng.standard_normal(C)).astype(np.float64) for _ in range(2))
    lengths = rng.integers(0, L + 1, N)
    inside = (np.arange(L) < lengths[:, None])[..., None]
    X, DY, Y, DX = Seq(N, C, L, dtype, layout, spoil(x, lengths)), Seq(N, C, L, dtype, layout, spoil(dy, lengths)), Seq(N, C, L, dtype, layout), Seq(N, C, L, dtype, layout)
    h = seq.seq_lnorm_create(N, C, L, dtype, EPS, views={"x": X.t, "y": Y.t, "r": X.t, "dy": DY.t, "dx": DX.t})
    dw, db, n, ws = nans(h.info.Cp), nans(h.info.Cp), ints(lengths), scratch(h)
    seq.seq_lnorm_fwd(h, X.t, None, vector(w, v), vector(b, v), None, Y.t, lengths=n)
    seq.seq_lnorm_bwd(h, X.t, vector(w, v), DY.t, None, DX.t, dw, db, ws, lengths=n)
    y, ey = oracle.lnorm(x, w, b, EPS)
    close(Y.get(), y * inside, ey * inside, bf16, "y")
    (dx, *want), (edx, *err) = oracle.lnorm_bwd(x, w, dy * inside, None, EPS)
    close(DX.get(), dx * inside, edx * inside, bf16, "dx")
    for name, got, a, e in zip(("dw", "db"), (dw, db), want, err):
        close(got.double().cpu().numpy()[:C], a, e, False, name)


@pytest.mark.parametrize("dtype", DTYPES)
def test_eight_bits_hold_what_the_operations_one_after_the_other_give(dtype):
    """The states' codes and scales after each of several steps, in every bit: fp32 operations rounded one by one, the nearest whole number of the rounded quotient.
    (A code that goes to the other side of a half moves the number by a step, and with it the scale of the steps behind.)"""
    f = np.float32
    n, beta1, beta2, rate, factor = 3000 * 256, 0.9, 0.95, 1e-3, 0.7
    h = seq.seq_adamw_create([n], dtype, 8, betas=(beta1, beta2))
    rng = np.random.default_rng(1)
    p, m, v = torch.zeros(n, device="cuda"), np.zeros(n, f), np.zeros(n, f)
    gm, gv, scales = seq.seq_adamw_states(h)
    for step in range(1, 5):
        g = torch.from_numpy((rng.standard_normal(n) * np.exp(rng.standard_normal((n // 256, 1)) - 6).repeat(256, 1).reshape(-1)).astype(f)).to(TORCH[dtype])
        seq.seq_adamw(h, seq.seq_adamw_tensors(h, [p], [g.cuda()]), gm, gv, (rate, step, factor), scales=scales)
        s = g.float().numpy() * f(factor)
        m, v = m * f(beta1) + s * f(1 - beta1), v * f(beta2) + s * s * f(1 - beta2)
        a, b = np.sqrt(np.abs(m)).reshape(-1, 256), np.sqrt(np.sqrt(v)).reshape(-1, 256)
        sa, sb = a.max(1, keepdims=True) * (f(1) / f(127)), b.max(1, keepdims=True) * (f(1) / f(255))
        qa, qb = np.rint(a / sa) * np.sign(m).reshape(a.shape), np.maximum(np.rint(b / sb), b > 0)
        assert a.dtype == b.dtype == sa.dtype == f
        got = scales.cpu().numpy().reshape(2, -1)
        assert np.array_equal(got[0], sa[:, 0]) and np.array_equal(got[1], sb[:, 0])
        assert np.array_equal(gm.cpu().numpy().reshape(a.shape), qa) and np.array_equal(gv.cpu().numpy().reshape(a.shape), qb)
        a, b = qa * sa, qb * sb
        m, v = (a * np.abs(a)).reshape(-1).astype(f), np.square(b * b).reshape(-1).astype(f)
