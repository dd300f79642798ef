"""The operators together: a block's training step against its definition in 64 bits, prompts against single tokens."""
import numpy as np
import pytest
import torch

import seq_oracle as oracle
from paper_1808_05567_amd import seq, seq_block
from seq_util import Seq

pytestmark = pytest.mark.gpu
EPS = 1e-5


def reference(p, x, res, S):
    """Everything the backward pass needs, [N, L, .]."""
    r = x + res
    u = oracle.norm(r, p["norm"], EPS)
    Ci = p["taps"].shape[1]
    pp = u @ p["w_in"].T
    px, pz = pp[..., :Ci], pp[..., Ci:]
    c, _ = oracle.conv(px, p["taps"], p["bias"])
    dt, B, Cm = c @ p["w_dt"].T, c @ p["w_B"].T, c @ p["w_C"].T
    s, _ = oracle.scan(c, dt, p["A"], B, Cm, D=p["D"], z=pz, dt_bias=p["dt_bias"])
    return r, u, px, pz, c, dt, B, Cm, s, s @ p["w_out"].T


def reference_bwd(p, x, res, dout, dr, S):
    r, u, px, pz, c, dt, B, Cm, s, _ = reference(p, x, res, S)
    flat = lambda t: t.reshape(-1, t.shape[-1])  # noqa: E731
    outer = lambda a, b: flat(a).T @ flat(b)  # noqa: E731
    g = {"w_out": outer(dout, s)}
    b = oracle.scan_bwd(c, dt, p["A"], B, Cm, dout @ p["w_out"], D=p["D"], z=pz, dt_bias=p["dt_bias"])
    g.update(A=b["dA"], D=b["dD"], dt_bias=b["ddt_bias"], w_dt=outer(b["ddt"], c), w_B=outer(b["dB"], c), w_C=outer(b["dC"], c))
    dc = b["dx"] + b["ddt"] @ p["w_dt"] + b["dB"] @ p["w_B"] + b["dC"] @ p["w_C"]
    dpx, g["taps"], g["bias"] = oracle.conv_bwd(px, p["taps"], p["bias"], dc)
    dp = np.concatenate([dpx, b["dz"]], -1)
    g["w_in"] = outer(dp, u)
    dx, g["norm"] = oracle.norm_bwd(r, p["norm"], dp @ p["w_in"], dr, EPS)
    return dx, g


@pytest.mark.parametrize("N,L,C,Ci,S", [(2, 37, 24, 40, 16), (1, 70, 20, 30, 5)])
def test_a_training_step(N, L, C, Ci, S):
    """In fp32: each operator is good to some 1e-6 of its magnitudes, the chain of seven to 1e-4 of the results' size."""
    W, dtype = 4, seq.SEQ_F32
    rng = np.random.default_rng(C)
    params = seq_block.init(C, Ci, S, W, seed=1)
    p = {k: t.double().cpu().numpy() for k, t in params.items()}
    x, res, dout, dr = (np.float64(np.float32(rng.standard_normal((N, L, C)))) for _ in range(4))
    block = seq_block.SeqBlock(N, L, C, Ci, S, W, params, dtype)
    X, RES, DOUT, DR = (Seq(N, C, L, dtype, "dense", a) for a in (x, res, dout, dr))
    out, r = block.forward(X.t.contiguous(), RES.t.contiguous())
    back = lambda t, n: t.permute(0, 2, 1, 3).reshape(N, L, -1)[..., :n].double().cpu().numpy()  # noqa: E731

    def near(got, want, name):
        assert np.linalg.norm(got - want) <= 1e-4 * np.linalg.norm(want), name
    near(back(out, C), reference(p, x, res, S)[-1], "out")
    near(back(r, C), x + res, "r")
    dx, g = block.backward(DOUT.t.contiguous(), DR.t.contiguous())
    want, wg = reference_bwd(p, x, res, dout, dr, S)
    near(back(dx, C), want, "dx")
    assert set(g) == set(wg)
    for k in wg:
        near(g[k].double().cpu().numpy(), wg[k], k)


def test_single_tokens_continue_prompts():
    """A prompt, then tokens one by one, against the prompt with the tokens behind it.  The weights are whole numbers of -7 ... 7 times a power of two,
    which 4 bits and bf16 both hold; what differs is the norm's result in 8 bits (half a step of 1/127 of the largest of its numbers, about
    3 of their standard deviations: 0.7 % of them) and bf16 roundings (0.2 % each) of seven operators: 5 % is some four times what they add up to."""
    N, L, extra, C, Ci, S, W = 3, 20, 4, 128, 192, 16, 4
    rng = np.random.default_rng(0)
    params = seq_block.init(C, Ci, S, W, seed=2)
    for k in ("w_in", "w_dt", "w_B", "w_C", "w_out"):
        q = torch.from_numpy(rng.integers(-7, 8, tuple(params[k].shape))).float()
        q[:, ::64] = 7  # (each group of 64 has the largest)
        params[k] = (q * 2.0 ** -6 * (0.25 if k == "w_dt" else 1)).cuda()
    make = lambda L: seq_block.SeqBlock(N, L, C, Ci, S, W, params, slots=N + 1)  # noqa: E731
    at = torch.tensor([2, 0, 3], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([L, L - 7, 1], dtype=torch.int32, device="cuda")
    x, res = (torch.randn(N, C // 8, L + extra, 8, device="cuda", generator=torch.Generator("cuda").manual_seed(3)).to(torch.bfloat16) for _ in range(2))
    whole = make(L + extra)
    # (the tokens follow each prompt's own end)
    xs, rs = x.clone(), res.clone()
    prompt = make(L)
    states = prompt.states()
    prompt.forward(x[:, :, :L].contiguous(), res[:, :, :L].contiguous(), states, at, lengths)
    step = seq_block.SeqBlockStep(prompt, N)
    tokens = []
    for t in range(extra):
        x1, r1 = (torch.stack([a[n, :, L + t] for n in range(N)]).unsqueeze(2).contiguous() for a in (x, res))
        for n, end in enumerate(lengths.tolist()):
            xs[n, :, end + t], rs[n, :, end + t] = x[n, :, L + t], res[n, :, L + t]
        out, r = step(x1, r1, states, at)
        tokens.append(out.clone())
    want, _ = whole.forward(xs, rs, lengths=(lengths + extra).to(torch.int32))
    for n, end in enumerate(lengths.tolist()):
        w = want[n, :, end:end + extra].float()
        got = torch.stack([t[n, :, 0] for t in tokens], 1).float()
        assert (got - w).norm() <= 0.05 * w.norm(), (n, float((got - w).norm() / w.norm()))


def test_captured_tokens():
    """Single tokens recorded once: every replay leaves the output and the states that a call leaves."""
    N, C, Ci, S, W = 5, 136, 200, 16, 4
    block = seq_block.SeqBlock(N, 8, C, Ci, S, W, seq_block.init(C, Ci, S, W, seed=4), slots=N + 2)
    g = torch.Generator("cuda").manual_seed(5)
    tokens = [[torch.randn(N, C // 8, 1, 8, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2)] for _ in range(4)]
    at = torch.tensor([4, 0, 6, 1, -1], dtype=torch.int32, device="cuda")
    step = seq_block.SeqBlockStep(block, N)
    states, want = block.states(), []
    for x, r in tokens:
        out, after = step(x, r, states, at)
        want.append([t.clone() for t in (out, after, *states)])
    x, r, again = *(torch.empty_like(t) for t in tokens[0]), block.states()
    x.copy_(tokens[0][0])
    r.copy_(tokens[0][1])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out, after = step(x, r, again, at)
    for t in again:
        t.zero_()
    for token, w in zip(tokens, want):
        x.copy_(token[0])
        r.copy_(token[1])
        graph.replay()
        torch.cuda.synchronize()
        for got, t in zip((out, after, *again), w):
            assert torch.equal(got, t)
