"""The recurrence, the layer norm and AdamW as a model has them: a training step of a recurrent block, its single tokens, and the state space block's own steps."""
import numpy as np
import pytest
import torch

import seq_rec_oracle as oracle
from seq_oracle import sigmoid
from seq_util import Seq, rounded, vector, vlen
from paper_1808_05567_amd import seq, seq_block

pytestmark = pytest.mark.gpu
EPS = 1e-5
NAMES = ("x", "f", "i", "z")


def parameters(C, Ci, seed):
    rng = np.random.default_rng(seed)
    f = lambda *s, k=1.0: (k * rng.standard_normal(s)).astype(np.float32)  # noqa: E731
    return {"w": 1 + f(C, k=0.1), "b": f(C, k=0.1), "w_in": f(4 * Ci, C, k=C ** -0.5), "A": -np.exp(f(Ci, k=0.5) - 2), "f_bias": f(Ci, k=0.5),
            "i_bias": f(Ci, k=0.5), "w_out": f(C, Ci, k=Ci ** -0.5)}


class Block:
    """r = x + res, u = lnorm(r), (x f i z) = W_in u, s = rec(x, f, i, z), out = W_out s, and the way back, by the library's operators."""

    def __init__(self, N, L, C, Ci, dtype, slots=0):
        assert C % vlen(dtype) == Ci % vlen(dtype) == 0
        self.dims, self.v = (N, L, C, Ci), vlen(dtype)
        self.w_in, self.w_out = seq_block._Projection(N, L, C, 4 * Ci, dtype, "cuda"), seq_block._Projection(N, L, Ci, C, dtype, "cuda")
        T = lambda c: torch.zeros(N, c // self.v, L, self.v, dtype=self.w_in.wt.dtype, device="cuda")  # noqa: E731
        self.r, self.u, self.p, self.s, self.out = T(C), T(C), T(4 * Ci), T(Ci), T(C)
        self.du, self.dp, self.ds, self.dx = T(C), T(4 * Ci), T(Ci), T(C)
        parts = lambda t: [t[:, k * (Ci // self.v):(k + 1) * (Ci // self.v)] for k in range(4)]  # noqa: E731
        self.parts, self.dparts = parts(self.p), parts(self.dp)
        self.norm = seq.seq_lnorm_create(N, C, L, dtype, EPS)
        self.rec = seq.seq_rec_create(N, Ci, L, dtype, slots=slots, views=dict(zip(NAMES, self.parts)) | dict(zip(("dx", "df", "di", "dz"), self.dparts)))
        self.ws = torch.empty(max(self.norm.info.workspace_bytes, self.rec.info.workspace_bytes, 16), dtype=torch.uint8, device="cuda")

    def load(self, t):
        self.t = t
        self.w_in.set(t["w_in"])
        self.w_out.set(t["w_out"])

    def forward(self, x, res, state=None, lengths=None):
        t, (px, pf, pi, pz) = self.t, self.parts
        seq.seq_lnorm_fwd(self.norm, x, res, t["w"], t["b"], self.r, self.u, lengths=lengths)
        self.w_in.fwd(self.u, self.p)
        seq.seq_rec_fwd(self.rec, px, pf, pi, t["A"], self.s, self.ws, z=pz, f_bias=t["f_bias"], i_bias=t["i_bias"], state_in=state, state_out=state, lengths=lengths)
        self.w_out.fwd(self.s, self.out)
        return self.out, self.r

    def backward(self, dout, dr, lengths=None):
        t, (px, pf, pi, pz), d = self.t, self.parts, self.dparts
        g = {k: torch.empty_like(t[k]) for k in ("w", "b", "A", "f_bias", "i_bias")}
        self.w_out.bwd(dout, self.ds)
        g["w_out"] = self.w_out.upd(self.s, dout)
        seq.seq_rec_bwd(self.rec, px, pf, pi, t["A"], self.ds, d[0], d[1], d[2], g["A"], self.ws, z=pz, f_bias=t["f_bias"], i_bias=t["i_bias"], dz=d[3],
                        df_bias=g["f_bias"], di_bias=g["i_bias"], lengths=lengths)
        g["w_in"] = self.w_in.upd(self.u, self.dp)
        self.w_in.bwd(self.dp, self.du)
        seq.seq_lnorm_bwd(self.norm, self.r, t["w"], self.du, dr, self.dx, g["w"], g["b"], self.ws, lengths=lengths)
        return self.dx, g


def reference(p, x, res, dout, dr):
    """out, r, dx and the parameters' gradients of one sequence in 64 bits."""
    Ci = len(p["A"])
    r = x + res
    u, _ = oracle.lnorm(r, p["w"], p["b"], EPS)
    q = dict(zip(NAMES, np.split(u @ p["w_in"].T, 4, axis=-1)))
    args = dict(q, A=p["A"], f_bias=p["f_bias"], i_bias=p["i_bias"])
    (s, _), _ = oracle.rec(**args)
    ds = dout @ p["w_out"]
    d, _ = oracle.rec_bwd(**args, dy=ds)
    dq = np.concatenate([d["dx"], d["df"], d["di"], d["dz"]], -1)
    (dx, dw, db), _ = oracle.lnorm_bwd(r, p["w"], dq @ p["w_in"], dr, EPS)
    flat = lambda t: t.reshape(-1, t.shape[-1])  # noqa: E731
    g = {"w": dw, "b": db, "A": d["dA"], "f_bias": d["df_bias"], "i_bias": d["di_bias"], "w_in": flat(dq).T @ flat(u), "w_out": flat(dout).T @ flat(s)}
    assert q["x"].shape[-1] == Ci
    return s @ p["w_out"].T, r, dx, g


@pytest.mark.parametrize("bits", [32, 8])
def test_a_training_step(bits):
    """In fp32, sequences that end early, against the sequences one by one; the bound is that of the whole step (five operators, each good to some 1e-6 of its
    magnitudes).  Then AdamW with these gradients."""
    N, L, C, Ci, dtype = 4, 70, 24, 40, seq.SEQ_F32
    ends = [L, 0, 1, 33]
    params = parameters(C, Ci, 3)
    p = {k: t.astype(np.float64) for k, t in params.items()}
    t = {k: torch.from_numpy(q).cuda() for k, q in params.items()}
    rng = np.random.default_rng(1)
    x, res, dout, dr = (np.float64(np.float32(rng.standard_normal((N, L, C)))) for _ in range(4))
    for n, end in enumerate(ends):
        dout[n, end:] = 0  # (the projections' weights are summed over all positions)
    X, RES, DOUT, DR = (Seq(N, C, L, dtype, "dense", a).t.contiguous() for a in (x, res, dout, dr))
    lengths = torch.tensor(ends, dtype=torch.int32, device="cuda")
    block = Block(N, L, C, Ci, dtype)
    block.load(t)
    back = lambda q: q.permute(0, 2, 1, 3).reshape(N, L, -1).double().cpu().numpy()  # noqa: E731
    out, r = (back(q) for q in block.forward(X, RES, lengths=lengths))
    dx, g = block.backward(DOUT, DR, lengths=lengths)
    dx, want, wr, wx, wg = back(dx), np.zeros_like(out), np.zeros_like(r), np.zeros_like(out), None
    for n, end in enumerate(ends):
        if end:
            want[n, :end], wr[n, :end], wx[n, :end], one = (q if isinstance(q, dict) else q[0] for q in reference(p, *(a[n:n + 1, :end] for a in (x, res, dout, dr))))
            wg = one if wg is None else {k: wg[k] + one[k] for k in wg}
    for got, ref, name in [(out, want, "out"), (r, wr, "r"), (dx, wx, "dx")] + [(g[k].double().cpu().numpy(), wg[k], k) for k in wg]:
        assert np.linalg.norm(got - ref) <= 1e-5 * np.linalg.norm(ref), name
    names = list(t)
    h = seq.seq_adamw_create([t[k].numel() for k in names], dtype, bits, decay=[0.1 if k.startswith("w_") else 0.0 for k in names])
    m, v, scales = seq.seq_adamw_states(h)
    seq.seq_adamw(h, seq.seq_adamw_tensors(h, [t[k] for k in names], [g[k] for k in names]), m, v, (1e-2, 1), scales=scales)
    for k in names:
        (p1, _, _), (ep, _, _) = oracle.adamw(p[k], g[k].double().cpu().numpy(), 0, 0, 1e-2, 1, 1.0, 0.9, 0.999, 1e-8, 0.1 if k.startswith("w_") else 0.0)
        assert np.all(np.abs(t[k].double().cpu().numpy() - p1) <= ep), k


def test_single_tokens():
    """A prompt, then its tokens one by one with 4-bit projections that hold what they stand for: the prompt's own pass over all of them, within what 8 bits of the
    norm and bf16 make of each (some 2^-7 an operator and position); captured, the same again."""
    N, L, more, C, Ci, dtype = 3, 20, 4, 64, 128, seq.SEQ_BF16
    params = parameters(C, Ci, 5)
    t = {k: torch.from_numpy(q).cuda() for k, q in params.items()}
    plans = {"w_in": seq.seq_mv4_create(N, C, 4 * Ci, 64, seq.SEQ_I8), "w_out": seq.seq_mv4_create(N, Ci, C, 64, dtype)}
    packed = {}
    for k, h in plans.items():  # (the prompt runs with the numbers that the 4 bits stand for)
        wt, scale = torch.empty(h.info.wt_bytes, dtype=torch.uint8, device="cuda"), torch.empty(h.info.scale_bytes // 4, device="cuda")
        seq.seq_mv4_quant(h, t[k], wt, scale)
        seq.seq_mv4_unquant(h, wt, scale, t[k])
        packed[k] = wt, scale
    rng = np.random.default_rng(2)
    x, res = (rounded(rng.standard_normal((N, L + more, C)), dtype) for _ in range(2))
    whole, part = Block(N, L + more, C, Ci, dtype), Block(N, L, C, Ci, dtype, slots=N)
    X, RES = (Seq(N, C, L + more, dtype, "dense", a).t.contiguous() for a in (x, res))
    for b in (whole, part):
        b.load(t)
    want = whole.forward(X, RES)[0].clone()
    state = torch.zeros(N, part.rec.info.Cp, device="cuda")
    part.forward(X[:, :, :L].contiguous(), RES[:, :, :L].contiguous(), state=state)
    T = lambda c, v=8, d=torch.bfloat16: torch.zeros(N, c // v, 1, v, dtype=d, device="cuda")  # noqa: E731
    x1, res1, r1, u1, p1, s1, out1, scale = T(C), T(C), T(C), T(C, 16, torch.int8), T(4 * Ci), T(Ci), T(C), torch.zeros(N, 1, device="cuda")
    parts = [p1[:, k * (Ci // 8):(k + 1) * (Ci // 8)] for k in range(4)]
    norm, rec = seq.seq_lnorm_create(N, C, 1, dtype, EPS), seq.seq_rec_create(N, Ci, 1, dtype, slots=N, views=dict(zip(NAMES, parts)))

    def token():
        seq.seq_lnorm_fwd_q8(norm, x1, res1, t["w"], t["b"], r1, u1, scale)
        seq.seq_mv4(plans["w_in"], u1, *packed["w_in"], p1, xscale=scale)
        seq.seq_rec_step(rec, *parts[:3], t["A"], state, s1, z=parts[3], f_bias=t["f_bias"], i_bias=t["i_bias"])
        seq.seq_mv4(plans["w_out"], s1, *packed["w_out"], out1)

    def serve(call):
        got = []
        for l in range(L, L + more):
            x1.copy_(X[:, :, l:l + 1])
            res1.copy_(RES[:, :, l:l + 1])
            call()
            torch.cuda.synchronize()
            got.append(out1.clone())
        return torch.cat(got, 2)
    begin = state.clone()
    eager = serve(token)
    ref = want[:, :, L:].double()
    assert (eager.double() - ref).norm() <= 5 * 2.0 ** -7 * ref.norm()
    after = state.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        token()
    state.copy_(begin)
    assert torch.equal(serve(graph.replay), eager) and torch.equal(state, after)


@pytest.mark.parametrize("bits", [32, 8])
def test_the_state_space_block_trains(bits):
    """SeqBlockAdamW: the block's numbers are those of the formula, its projections and steps have them, and an odd inner width is no matter."""
    N, L, C, Ci, S, W = 2, 20, 40, 50, 5, 4
    block = seq_block.SeqBlock(N, L, C, Ci, S, W, seq_block.init(C, Ci, S, W, seed=1), slots=N)
    served = seq_block.SeqBlockStep(block, N)
    adamw = seq_block.SeqBlockAdamW(block, bits=bits)
    x, res, dout, dr = (torch.randn(N, C // 8, L, 8, device="cuda").to(torch.bfloat16) for _ in range(4))
    before = {k: t.double().cpu().numpy() for k, t in block.params.items()}
    block.forward(x, res)
    _, g = block.backward(dout, dr)
    adamw.step(g, 1e-2, 0.5)
    for k, t in block.params.items():
        decay = 0.1 if k.startswith("w_") else 0.0
        (p1, _, _), (ep, _, _) = oracle.adamw(before[k], g[k].double().cpu().numpy(), 0, 0, 1e-2, 1, 0.5, 0.9, 0.95, 1e-8, decay)
        assert np.all(np.abs(t.double().cpu().numpy() - p1) <= ep), k
    other = seq_block.SeqBlock(N, L, C, Ci, S, W, {k: t.clone() for k, t in block.params.items()}, slots=N)
    assert all(torch.equal(a, b) for a, b in zip(block.forward(x, res), other.forward(x, res)))
    one = [t[:, :, :1].contiguous() for t in (x, res)]
    assert all(torch.equal(a, b) for a, b in zip(served(*one, block.states()), seq_block.SeqBlockStep(other, N)(*one, other.states())))
    adamw.step(g, 1e-2)
    assert adamw.t == 2 and all(t.isfinite().all() for t in block.params.values())
