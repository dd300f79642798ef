"""The sequence operators of ``paper_1808_05567_amd.seq`` as cases that can be timed and checked.

A case is one pass through one of them, as a program that trains or serves a language model of
short convolutions and state spaces calls it:

  conv   a short causal convolution of every channel with SiLU: over prompts ("fwd"), its
         gradients ("bwd"), over one new token a sequence ("step")
  scan   a selective state space scan, the same three
  norm   a root-mean-square norm with the residual's addition: training forward and backward,
         and with an output in 8 bits for the products that follow ("q8")
  mv4    a projection of a few tokens with weights of 4 bits and scales for groups of channels

Tensors of sequences have the library's blocked form, [N][Cb][L][v] with v channels in 16 bytes,
dense ("blocked") or with a position's channels side by side ("rows").  Sums, states and
parameters are fp32.
"""
import math

import torch
import torch.nn.functional as F

own = False

_T = {"f32": torch.float32, "bf16": torch.bfloat16, "i8": torch.int8}
EPS = 1e-5


# ---------------------------------------------------------------------------- cases
def listed():
    return [
        # one new token of one sequence: latency
        {"name": "conv_step_b1_bf16", "op": "conv", "pass": "step", "dtype": "bf16", "layout": "blocked",
         "N": 1, "C": 2048, "L": 1, "W": 4, "slots": 8},
        # five prompts of different lengths, one of them none, states carried in and out
        {"name": "conv_prompt_b5_bf16", "op": "conv", "pass": "fwd", "dtype": "bf16", "layout": "blocked",
         "N": 5, "C": 2048, "L": 1021, "W": 4, "slots": 8, "ragged": True},
        # the gradients of a training step
        {"name": "conv_train_bwd_bf16", "op": "conv", "pass": "bwd", "dtype": "bf16", "layout": "blocked",
         "N": 8, "C": 2048, "L": 2048, "W": 4, "ragged": False},
        # one new token of each of 64 sequences: the states are what is read and written
        {"name": "scan_step_b64_bf16", "op": "scan", "pass": "step", "dtype": "bf16", "layout": "blocked",
         "N": 64, "C": 4096, "L": 1, "S": 16, "G": 1, "gate": True, "slots": 80},
        # one long prompt
        {"name": "scan_prompt_b1_bf16", "op": "scan", "pass": "fwd", "dtype": "bf16", "layout": "blocked",
         "N": 1, "C": 2048, "L": 4096, "S": 16, "G": 1, "gate": True, "slots": 4, "ragged": False},
        # short sequences of different lengths in full precision, four groups of channels
        {"name": "scan_ragged_b3_f32", "op": "scan", "pass": "fwd", "dtype": "f32", "layout": "rows",
         "N": 3, "C": 768, "L": 333, "S": 16, "G": 4, "gate": False, "slots": 3, "ragged": True},
        # the gradients of a training step
        {"name": "scan_train_bwd_bf16", "op": "scan", "pass": "bwd", "dtype": "bf16", "layout": "blocked",
         "N": 2, "C": 2048, "L": 2048, "S": 16, "G": 1, "gate": True, "ragged": False},
        # where two blocks of a training step meet
        {"name": "norm_train_fwd_bf16", "op": "norm", "pass": "fwd", "dtype": "bf16", "layout": "blocked",
         "N": 8, "C": 2048, "L": 2048, "residual": True},
        # its gradients, in full precision
        {"name": "norm_train_bwd_f32", "op": "norm", "pass": "bwd", "dtype": "f32", "layout": "blocked",
         "N": 2, "C": 2048, "L": 1024, "residual": True},
        # before the projections of one new token of each of 16 sequences
        {"name": "norm_q8_b16_bf16", "op": "norm", "pass": "q8", "dtype": "bf16", "layout": "blocked",
         "N": 16, "C": 4096, "L": 1, "residual": True},
        # a projection of one token that the norm has left in 8 bits
        {"name": "mv4_b1_i8", "op": "mv4", "pass": "fwd", "dtype": "i8", "M": 1, "C": 4096, "K": 8192, "group": 128},
        # a projection of a batch of tokens
        {"name": "mv4_b24_bf16", "op": "mv4", "pass": "fwd", "dtype": "bf16", "M": 24, "C": 2048, "K": 4100, "group": 64},
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _channels(rng, lo, hi):
    """Mostly multiples of 64, as models have them; odd ones too."""
    while True:
        c = _log(rng, lo, hi)
        c = c if rng.random() < 0.35 else max(64, c // 64 * 64)
        if c != 3072:  # (no size of ours)
            return c


def draw(rng):
    op, what = rng.choice((("conv", "fwd"), ("conv", "bwd"), ("conv", "step"), ("scan", "fwd"), ("scan", "fwd"), ("scan", "bwd"),
                           ("scan", "step"), ("norm", "fwd"), ("norm", "bwd"), ("norm", "q8"), ("mv4", "fwd"), ("mv4", "fwd")))
    c = {"op": op, "pass": what, "dtype": rng.choice(("bf16", "bf16", "f32")), "layout": rng.choice(("blocked", "blocked", "rows"))}
    if op == "mv4":
        del c["layout"]
        c["dtype"] = rng.choice(("bf16", "i8", "f32"))
        c["M"] = _log(rng, 1, 48)
        c["group"] = rng.choice((32, 64, 128))
        c["C"] = rng.choice((1, 2, 3, 5, 8, 11, 16, 24, 32)) * 128 + rng.choice((0, 0, 0, 32, 72))
        c["K"] = _channels(rng, 64, 8192)
        return c
    step = what == "step"
    if op == "conv":
        c["C"], c["W"] = _channels(rng, 40, 4096), rng.choice((2, 3, 4, 4, 4))
        c["N"] = _log(rng, 1, 128 if step else 16)
        most = (1 << 25) // (c["N"] * c["C"]) // (2 if c["dtype"] == "f32" else 1)
        c["L"] = 1 if step else _log(rng, 1, max(1, min(8192, most)))
    elif op == "scan":
        c["S"], c["G"], c["gate"] = rng.choice((4, 8, 16, 16, 16, 32)), rng.choice((1, 1, 2)), rng.random() < 0.6
        c["C"] = _channels(rng, 40, 4096)
        if c["G"] > 1:
            c["C"] = max(16, c["C"] // 16 * 16)
        c["N"] = _log(rng, 1, 64 if step else 8)
        most = (1 << 26) // (c["N"] * c["C"] * c["S"])
        c["L"] = 1 if step else _log(rng, 1, max(1, min(8192, most)))
        if step:
            c["S"] = min(c["S"], max(4, (1 << 22) // (c["N"] * c["C"])))
    else:
        c["C"], c["N"], c["residual"] = _channels(rng, 40, 8192), _log(rng, 1, 16), rng.random() < 0.8
        most = (1 << 25) // (c["N"] * c["C"]) // (2 if c["dtype"] == "f32" else 1)
        c["L"] = _log(rng, 1, max(1, min(64 if what == "q8" else 8192, most)))
        return c
    if what != "bwd":
        c["slots"] = c["N"] + rng.randrange(4)
    if not step:
        c["ragged"] = rng.random() < 0.5
    return c


def work(case):
    if case["op"] == "mv4":
        M, C, K = case["M"], case["C"], case["K"]
        e = _T[case["dtype"]].itemsize
        return {"bytes": K * C // 2 + 4 * K * -(-C // case["group"]) + M * C * e + M * K * (4 if case["dtype"] == "f32" else 2), "flops": 2 * M * K * C}
    N, C, L, what, e = case["N"], case["C"], case["L"], case["pass"], _T[case["dtype"]].itemsize
    n = N * C * L
    if case["op"] == "conv":
        W = case["W"]
        if what == "bwd":
            return {"bytes": 3 * e * n + 8 * C * (W + 1), "flops": n * (6 * W + 14)}
        return {"bytes": 2 * e * n + 4 * C * (W + 1) + 2 * e * N * C * (W - 1), "flops": n * (2 * W + 6)}
    if case["op"] == "scan":
        S, G, gate = case["S"], case["G"], 1 if case["gate"] else 0
        bc, par = 2 * e * N * L * G * S, 4 * C * (S + 2)
        if what == "bwd":
            return {"bytes": e * n * (5 + 2 * gate) + 2 * bc + 2 * par, "flops": n * S * 24}
        return {"bytes": e * n * (3 + gate) + bc + par + 8 * N * S * C, "flops": n * S * 8}
    res = 1 if case["residual"] else 0
    if what == "q8":
        return {"bytes": n * (e * (1 + 2 * res) + 1) + 4 * N * L + 4 * C, "flops": n * 8}
    if what == "bwd":
        return {"bytes": n * e * (3 + res) + 8 * C, "flops": n * 10}
    return {"bytes": n * e * (2 + 2 * res) + 4 * C, "flops": n * 5}


# ---------------------------------------------------------------------------- inputs
def _vlen(case):
    return 16 // _T[case["dtype"]].itemsize


def _blocks(case, N, Cb, L, v=None, dtype=None, fill=None):
    """A tensor [N][Cb][L][v] in the case's layout; `fill(shape)` gives the numbers, [N, L, Cb * v] in fp32."""
    v, dtype = v or _vlen(case), dtype or _T[case["dtype"]]
    shape = (N, Cb, L, v) if case["layout"] == "blocked" else (N, L, Cb, v)
    t = torch.zeros(shape, dtype=dtype, device="cuda")
    if case["layout"] != "blocked":
        t = t.permute(0, 2, 1, 3)
    if fill is not None:
        t.copy_(fill((N, L, Cb * v)).view(N, L, Cb, v).permute(0, 2, 1, 3))
    return t


def _random(case, g, C, N, L, scale=1.0, count=1):
    """`count` tensors of C channels side by side in one, as one projection leaves them."""
    v = _vlen(case)
    Cb = -(-C // v)

    def fill(shape):
        x = torch.randn(shape, generator=g, device="cuda") * scale
        return (x.view(N, L, count, Cb * v) * (torch.arange(Cb * v, device="cuda") < C)).view(shape)
    t = _blocks(case, N, Cb * count, L, fill=fill)
    return [t[:, i * Cb:(i + 1) * Cb] for i in range(count)]


def _lengths(case, g):
    if not case.get("ragged"):
        return None
    n = torch.randint(0, case["L"] + 1, (case["N"],), generator=g, device="cuda", dtype=torch.int32)
    n[0] = case["L"]
    if case["N"] > 2:
        n[1] = 0
    return n


def _slots(case, g):
    return torch.randperm(case["slots"], generator=g, device="cuda")[:case["N"]].to(torch.int32)


def _padded(x, C, Cp):
    return F.pad(x, (0, Cp - C)).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    st = {"case": case}
    if case["op"] == "mv4":
        _prepare_mv4(case, g, st)
    else:
        N, C, L, v, what = case["N"], case["C"], case["L"], _vlen(case), case["pass"]
        Cb = -(-C // v)
        Cp = Cb * v
        {"conv": _prepare_conv, "scan": _prepare_scan, "norm": _prepare_norm}[case["op"]](case, g, st, N, C, L, Cb, Cp, what)
    st["plan"], st["ws"] = _plan(case, st)
    return st


def _prepare_conv(case, g, st, N, C, L, Cb, Cp, what):
    W = case["W"]
    # (the first half of a projection's output; the second is the gate)
    st["x"] = _random(case, g, C, N, L, count=2)[0]
    st["w"] = _padded(torch.randn(W, C, generator=g, device="cuda") * W ** -0.5, C, Cp)
    st["bias"] = _padded(torch.randn(C, generator=g, device="cuda") * 0.2, C, Cp)
    if what == "bwd":
        st["dy"], = _random(case, g, C, N, L)
        st["dx"] = _blocks(case, N, 2 * Cb, L)[:, :Cb]
        st["dw"], st["dbias"] = torch.zeros_like(st["w"]), torch.zeros_like(st["bias"])
    else:
        st["y"] = _blocks(case, N, Cb, L)
        st["state"] = torch.zeros(case["slots"], Cb, W - 1, Cp // Cb, device="cuda", dtype=_T[case["dtype"]])
        st["state"].copy_(torch.randn(st["state"].shape, generator=g, device="cuda"))
        st["state"].mul_((torch.arange(Cp, device="cuda") < C).view(Cb, 1, -1))  # (zeros beyond C)
        st["slots"] = _slots(case, g)
    st["lengths"] = _lengths(case, g)


def _prepare_scan(case, g, st, N, C, L, Cb, Cp, what):
    S, G = case["S"], case["G"]
    xz = _random(case, g, C, N, L, count=2)
    st["x"], st["z"] = xz[0], xz[1] if case["gate"] else None
    st["dt"], = _random(case, g, C, N, L, 0.5)
    st["B"], st["C"] = _random(case, g, G * S, N, L, count=2)
    A = -(torch.arange(1, S + 1, device="cuda").float().view(S, 1) * (0.8 + 0.4 * torch.rand(S, C, generator=g, device="cuda")))
    st["A"] = _padded(A, C, Cp)
    st["D"] = _padded(1 + 0.1 * torch.randn(C, generator=g, device="cuda"), C, Cp)
    step = torch.exp(torch.empty(C, device="cuda").uniform_(math.log(1e-3), math.log(1e-1), generator=g))
    st["dt_bias"] = _padded(step + torch.log(-torch.expm1(-step)), C, Cp)  # (softplus of it is the step)
    if what == "bwd":
        st["dy"], = _random(case, g, C, N, L)
        dxz = _blocks(case, N, 2 * Cb, L)
        st["dx"], st["dz"] = dxz[:, :Cb], dxz[:, Cb:] if case["gate"] else None
        st["ddt"] = _blocks(case, N, Cb, L)
        Sb = st["B"].shape[1]
        dbc = _blocks(case, N, 2 * Sb, L)
        st["dB"], st["dC"] = dbc[:, :Sb], dbc[:, Sb:]
        st["dA"], st["dD"], st["ddt_bias"] = torch.zeros_like(st["A"]), torch.zeros_like(st["D"]), torch.zeros_like(st["D"])
    else:
        st["y"] = _blocks(case, N, Cb, L)
        st["state"] = _padded(torch.randn(case["slots"], S, C, generator=g, device="cuda") * 0.3, C, Cp)
        st["slots"] = _slots(case, g)
    st["lengths"] = _lengths(case, g)


def _prepare_norm(case, g, st, N, C, L, Cb, Cp, what):
    st["w"] = _padded(1 + 0.2 * torch.randn(C, generator=g, device="cuda"), C, Cp)
    if what == "bwd":
        st["r"], = _random(case, g, C, N, L, 1.5)
        st["dy"], = _random(case, g, C, N, L)
        st["dr"] = _random(case, g, C, N, L)[0] if case["residual"] else None
        st["dx"] = _blocks(case, N, Cb, L)
        st["dw"] = torch.zeros_like(st["w"])
        return
    st["x"], = _random(case, g, C, N, L)
    st["res"] = _random(case, g, C, N, L, 1.2)[0] if case["residual"] else None
    st["r"] = _blocks(case, N, Cb, L) if case["residual"] else None
    if what == "q8":
        st["q"] = _blocks(case, N, -(-C // 16), L, v=16, dtype=torch.int8)
        st["scale"] = torch.zeros(N, L, device="cuda")
        st["stands_for"] = torch.empty_like(st["q"], dtype=torch.bfloat16)
    else:
        st["y"] = _blocks(case, N, Cb, L)


def _prepare_mv4(case, g, st):
    M, C, K, group = case["M"], case["C"], case["K"], case["group"]
    Kp, Cw = -(-K // 16) * 16, -(-C // 128) * 128
    q = torch.randint(-8, 8, (K, C), generator=g, device="cuda", dtype=torch.int32)
    st["wq"] = _pack4(q, K, C, Kp, Cw)
    st["wscale"] = F.pad(torch.rand(-(-C // group), K, generator=g, device="cuda") * 0.02 + 0.005, (0, Kp - K)).contiguous()
    if case["dtype"] == "i8":
        Cx = -(-C // 16) * 16
        x = torch.randint(-127, 128, (M, C), generator=g, device="cuda", dtype=torch.int32)
        st["xscale"] = torch.rand(M, generator=g, device="cuda") * 0.02 + 0.01
    else:
        Cx = -(-C // _vlen(case)) * _vlen(case)
        x = torch.randn(M, C, generator=g, device="cuda")
        st["xscale"] = None
    st["x"] = F.pad(x, (0, Cx - C)).to(_T[case["dtype"]]).contiguous()
    if case["dtype"] == "f32":
        st["y"] = torch.zeros(M, -(-K // 4) * 4, device="cuda")
    else:
        st["y"] = torch.zeros(M, -(-K // 8) * 8, device="cuda", dtype=torch.bfloat16)


def _pack4(q, K, C, Kp, Cw):
    """The library's layout of 4-bit weights, [Cw/128][Kp][4][4][8 x 4 bits]: word i of 16-byte lane j of a row holds the
    channels 32 i + 8 j .. + 7 of its 128, the first in the lowest bits, in two's complement."""
    q = F.pad(q, (0, Cw - C, 0, Kp - K)) & 15
    q = q.view(Kp, Cw // 128, 4, 4, 8).permute(1, 0, 3, 2, 4)  # [Cw/128][Kp][j][i][8]
    return (q[..., 0::2] | (q[..., 1::2] << 4)).to(torch.uint8).contiguous()


def _plan(case, st):
    """The framework's plan for these tensors, and its workspace."""
    if not own:
        return None, None
    from paper_1808_05567_amd import seq
    views = {k: t for k, t in st.items() if isinstance(t, torch.Tensor) and t.dim() == 4 and k not in ("state", "wq", "stands_for")}
    code = {"f32": seq.SEQ_F32, "bf16": seq.SEQ_BF16, "i8": seq.SEQ_I8}[case["dtype"]]
    if case["op"] == "conv":
        h = seq.seq_conv_create(case["N"], case["C"], case["L"], case["W"], code, silu=True, slots=case.get("slots", 0), views=views)
    elif case["op"] == "scan":
        h = seq.seq_scan_create(case["N"], case["C"], case["L"], case["S"], code, G=case["G"], softplus=True,
                                slots=case.get("slots", 0), views=views)
    elif case["op"] == "norm":
        h = seq.seq_norm_create(case["N"], case["C"], case["L"], code, EPS, views=views)
    else:
        h = seq.seq_mv4_create(case["M"], case["C"], case["K"], case["group"], code)
    return h, seq.seq_workspace(h)


# ---------------------------------------------------------------------------- one pass
def run(st):
    case = st["case"]
    key = (case["op"], case["pass"])
    outputs = {("conv", "fwd"): ("y", "state"), ("conv", "step"): ("y", "state"), ("conv", "bwd"): ("dx", "dw", "dbias"),
               ("scan", "fwd"): ("y", "state"), ("scan", "step"): ("y", "state"),
               ("scan", "bwd"): ("dx", "ddt", "dA", "dB", "dC", "dD", "dz", "ddt_bias"),
               ("norm", "fwd"): ("r", "y"), ("norm", "q8"): ("r", "q", "scale"), ("norm", "bwd"): ("dx", "dw"), ("mv4", "fwd"): ("y",)}[key]
    if own:
        _call(key, st)
    else:
        _PLAIN[key](st, case)
    out = {k: st[k] for k in outputs if st[k] is not None}
    if key == ("norm", "q8"):  # (what the 8 bits stand for)
        out["y"] = torch.mul(out.pop("q"), st["scale"].view(case["N"], 1, case["L"], 1), out=st["stands_for"])
    return out


def _call(key, s):
    from paper_1808_05567_amd import seq
    h = s["plan"]
    if key == ("conv", "fwd"):
        seq.seq_conv_fwd(h, s["x"], s["w"], s["bias"], s["y"], state_in=s["state"], state_out=s["state"], slots=s["slots"], lengths=s["lengths"])
    elif key == ("conv", "step"):
        seq.seq_conv_step(h, s["x"], s["w"], s["bias"], s["state"], s["y"], slots=s["slots"])
    elif key == ("conv", "bwd"):
        seq.seq_conv_bwd(h, s["x"], s["w"], s["bias"], s["dy"], s["dx"], s["dw"], s["dbias"], s["ws"], lengths=s["lengths"])
    elif key == ("scan", "fwd"):
        seq.seq_scan_fwd(h, s["x"], s["dt"], s["A"], s["B"], s["C"], s["y"], s["ws"], D=s["D"], z=s["z"], dt_bias=s["dt_bias"],
                         state_in=s["state"], state_out=s["state"], slots=s["slots"], lengths=s["lengths"])
    elif key == ("scan", "step"):
        seq.seq_scan_step(h, s["x"], s["dt"], s["A"], s["B"], s["C"], s["state"], s["y"], D=s["D"], z=s["z"], dt_bias=s["dt_bias"], slots=s["slots"])
    elif key == ("scan", "bwd"):
        seq.seq_scan_bwd(h, s["x"], s["dt"], s["A"], s["B"], s["C"], s["dy"], s["dx"], s["ddt"], s["dA"], s["dB"], s["dC"], s["ws"],
                         D=s["D"], z=s["z"], dt_bias=s["dt_bias"], dD=s["dD"], dz=s["dz"], ddt_bias=s["ddt_bias"], lengths=s["lengths"])
    elif key == ("norm", "fwd"):
        seq.seq_norm_fwd(h, s["x"], s["res"], s["w"], s["r"], s["y"])
    elif key == ("norm", "q8"):
        seq.seq_norm_fwd_q8(h, s["x"], s["res"], s["w"], s["r"], s["q"], s["scale"])
    elif key == ("norm", "bwd"):
        seq.seq_norm_bwd(h, s["r"], s["w"], s["dy"], s["dr"], s["dx"], s["dw"], s["ws"])
    else:
        seq.seq_mv4(h, s["x"], s["wq"], s["wscale"], s["y"], xscale=s["xscale"])


# ---------------------------------------------------------------------------- plain forms, fp32
def _rows(t, C):
    """[N][Cb][L][v] -> [N, L, C] in fp32."""
    N, Cb, L, v = t.shape
    return t.permute(0, 2, 1, 3).reshape(N, L, Cb * v)[..., :C].float()


def _store(t, x):
    """[N, L, C] in fp32 -> the blocked tensor t, rounded once, zeros beyond C."""
    N, Cb, L, v = t.shape
    t.copy_(F.pad(x, (0, Cb * v - x.shape[-1])).view(N, L, Cb, v).permute(0, 2, 1, 3))


def _inside(st, N, L):
    """[N, L, 1]: whether a position is inside its sequence; None where all are."""
    if st["lengths"] is None:
        return None
    return (torch.arange(L, device="cuda") < st["lengths"].view(N, 1)).unsqueeze(-1)


def _sigmoid(x):
    return 1 / (1 + torch.exp(-x))


def _plain_conv_fwd(st, case):
    N, C, L, W = case["N"], case["C"], case["L"], case["W"]
    at = st["slots"].long()
    before = _rows(st["state"][at], C)
    xe = torch.cat((before, _rows(st["x"], C)), 1)
    s = (xe.unfold(1, W, 1) * st["w"][:, :C].t()).sum(-1) + st["bias"][:C]
    y = s * _sigmoid(s)
    inside = _inside(st, N, L)
    _store(st["y"], y if inside is None else torch.where(inside, y, 0.0))
    n = st["lengths"].long() if inside is not None else torch.full((N,), L, device="cuda")
    last = torch.gather(xe, 1, (n.view(N, 1, 1) + torch.arange(W - 1, device="cuda").view(1, W - 1, 1)).expand(N, W - 1, C))
    new = torch.empty_like(st["state"][:N])
    _store(new, last)
    st["state"][at] = new


def _plain_conv_bwd(st, case):
    N, C, L, W = case["N"], case["C"], case["L"], case["W"]
    w = st["w"][:, :C]
    x, dy = _rows(st["x"], C), _rows(st["dy"], C)
    inside = _inside(st, N, L)
    if inside is not None:
        x, dy = torch.where(inside, x, 0.0), torch.where(inside, dy, 0.0)
    xw = F.pad(x, (0, 0, W - 1, 0)).unfold(1, W, 1)  # [N, L, C, W]
    s = (xw * w.t()).sum(-1) + st["bias"][:C]
    p = _sigmoid(s)
    ds = dy * p * (1 + s * (1 - p))
    dx = (F.pad(ds, (0, 0, 0, W - 1)).unfold(1, W, 1) * w.flip(0).t()).sum(-1)
    _store(st["dx"], dx if inside is None else torch.where(inside, dx, 0.0))
    st["dw"][:, :C] = (xw * ds.unsqueeze(-1)).sum((0, 1)).t()
    st["dbias"][:C] = ds.sum((0, 1))


def _scan(a, b):
    """h[l] = a[l] h[l-1] + b[l] along dimension 1 from h[-1] = 0, by doubling; a and b are used up."""
    s = 1
    while s < a.shape[1]:
        b[:, s:] += a[:, s:] * b[:, :-s]
        a[:, s:] = a[:, s:] * a[:, :-s]
        s *= 2
    return b


def _scan_inputs(st, case):
    N, C, L, S, G = case["N"], case["C"], case["L"], case["S"], case["G"]
    x, raw = _rows(st["x"], C), _rows(st["dt"], C) + st["dt_bias"][:C]
    d = torch.where(raw > 20, raw, torch.log1p(torch.exp(raw.clamp(max=20))))
    inside = _inside(st, N, L)
    if inside is not None:
        x, d = torch.where(inside, x, 0.0), torch.where(inside, d, 0.0)
    A = st["A"][:, :C].t()
    B = _rows(st["B"], G * S).view(N, L, G, 1, S)
    Cm = _rows(st["C"], G * S).view(N, L, G, 1, S)
    return x, raw, d, A, B, Cm, inside


def _plain_scan_fwd(st, case):
    N, C, L, S, G = case["N"], case["C"], case["L"], case["S"], case["G"]
    x, raw, d, A, B, Cm, inside = _scan_inputs(st, case)
    at = st["slots"].long()
    a = torch.exp(d.unsqueeze(-1) * A)
    h = ((d * x).view(N, L, G, C // G, 1) * B).view(N, L, C, S)
    h[:, 0] += a[:, 0] * st["state"][at][..., :C].transpose(1, 2)
    h = _scan(a, h)
    y = (h.view(N, L, G, C // G, S) * Cm).sum(-1).view(N, L, C) + st["D"][:C] * x
    if st["z"] is not None:
        z = _rows(st["z"], C)
        y = y * z * _sigmoid(z)
    _store(st["y"], y if inside is None else torch.where(inside, y, 0.0))
    new = F.pad(h[:, -1].transpose(1, 2), (0, st["state"].shape[-1] - C))
    st["state"][at] = new


def _plain_scan_bwd(st, case):
    N, C, L, S, G = case["N"], case["C"], case["L"], case["S"], case["G"]
    x, raw, d, A, B, Cm, inside = _scan_inputs(st, case)
    dy = _rows(st["dy"], C)
    if inside is not None:
        dy = torch.where(inside, dy, 0.0)
    a = torch.exp(d.unsqueeze(-1) * A)
    h = _scan(a.clone(), ((d * x).view(N, L, G, C // G, 1) * B).view(N, L, C, S))
    hg = h.view(N, L, G, C // G, S)
    if st["z"] is not None:
        z = _rows(st["z"], C)
        p = _sigmoid(z)
        y = (hg * Cm).sum(-1).view(N, L, C) + st["D"][:C] * x
        dz = dy * y * p * (1 + z * (1 - p))
        _store(st["dz"], dz if inside is None else torch.where(inside, dz, 0.0))
        dy = dy * z * p if inside is None else torch.where(inside, dy * z * p, 0.0)
    dyg = dy.view(N, L, G, C // G, 1)
    after = torch.cat((a[:, 1:], torch.zeros_like(a[:, :1])), 1)
    g = _scan(after.flip(1), (dyg * Cm).view(N, L, C, S).flip(1)).flip(1)
    gg = g.view(N, L, G, C // G, S)
    _store(st["dC"], (dyg * hg).sum(3).view(N, L, G * S))
    _store(st["dB"], (gg * (d * x).view(N, L, G, C // G, 1)).sum(3).view(N, L, G * S))
    gB = (gg * B).sum(-1).view(N, L, C)
    _store(st["dx"], st["D"][:C] * dy + d * gB)
    t = g * a * torch.cat((torch.zeros_like(h[:, :1]), h[:, :-1]), 1)
    dd = (t * A).sum(-1) + x * gB
    ddt = dd * _sigmoid(raw)
    ddt = ddt if inside is None else torch.where(inside, ddt, 0.0)
    _store(st["ddt"], ddt)
    st["dA"][:, :C] = (t * d.unsqueeze(-1)).sum((0, 1)).t()
    st["dD"][:C] = (dy * x).sum((0, 1))
    st["ddt_bias"][:C] = ddt.sum((0, 1))


def _plain_norm(st, case):
    C = case["C"]
    r = _rows(st["x"], C)
    if st["res"] is not None:
        _store(st["r"], r + _rows(st["res"], C))
        r = _rows(st["r"], C)  # (the norm is of what is stored)
    return r / torch.sqrt((r * r).mean(-1, keepdim=True) + EPS) * st["w"][:C]


def _plain_norm_fwd(st, case):
    _store(st["y"], _plain_norm(st, case))


def _plain_norm_q8(st, case):
    y = _plain_norm(st, case)
    scale = y.abs().amax(-1) / 127
    st["scale"].copy_(scale)
    scale = torch.where(scale > 0, scale, 1.0)
    _store(st["q"], torch.round(y / scale.unsqueeze(-1)))


def _plain_norm_bwd(st, case):
    C = case["C"]
    r, dy, w = _rows(st["r"], C), _rows(st["dy"], C), st["w"][:C]
    rstd = 1 / torch.sqrt((r * r).mean(-1, keepdim=True) + EPS)
    wdy = w * dy
    dx = rstd * (wdy - r * rstd * rstd * (wdy * r).mean(-1, keepdim=True))
    _store(st["dx"], dx if st["dr"] is None else dx + _rows(st["dr"], C))
    st["dw"][:C] = (dy * r * rstd).sum((0, 1))


def _unpack4(wq, K, C):
    Cs, Kp = wq.shape[:2]
    b = wq.int()
    q = torch.stack((b & 15, b >> 4), -1).view(Cs, Kp, 4, 4, 8)
    q = q.permute(1, 0, 3, 2, 4).reshape(Kp, Cs * 128)[:K, :C]
    return q - 16 * (q > 7)


def _plain_mv4(st, case):
    M, C, K, group = case["M"], case["C"], case["K"], case["group"]
    scale = st["wscale"][:, :K].t().repeat_interleave(group, 1)[:, :C]
    y = st["x"][:, :C].float() @ (_unpack4(st["wq"], K, C).float() * scale).t()
    if st["xscale"] is not None:
        y = y * st["xscale"].unsqueeze(-1)
    st["y"][:, :K] = y


_PLAIN = {("conv", "fwd"): _plain_conv_fwd, ("conv", "step"): _plain_conv_fwd, ("conv", "bwd"): _plain_conv_bwd,
          ("scan", "fwd"): _plain_scan_fwd, ("scan", "step"): _plain_scan_fwd, ("scan", "bwd"): _plain_scan_bwd,
          ("norm", "fwd"): _plain_norm_fwd, ("norm", "q8"): _plain_norm_q8, ("norm", "bwd"): _plain_norm_bwd, ("mv4", "fwd"): _plain_mv4}


# ---------------------------------------------------------------------------- from the definitions, 64 bits
def exact(case, seed):
    """One position after the other, as the definitions have it."""
    st = prepare(case, seed)
    return {"conv": _exact_conv, "scan": _exact_scan, "norm": _exact_norm, "mv4": _exact_mv4}[case["op"]](case, st)


def _wide(t, C):
    """[N][Cb][L][v] -> [N, L, C] in 64 bits."""
    return t.double().transpose(1, 2).flatten(2)[:, :, :C]


def _like(t, x):
    """Back to the form of t."""
    full = torch.zeros(t.shape[0], t.shape[2], t.shape[1] * t.shape[3], dtype=torch.float64, device="cuda")
    full[:, :, :x.shape[2]] = x
    return full.unflatten(2, (t.shape[1], t.shape[3])).transpose(1, 2)


def _vector(t, x):
    full = torch.zeros(t.shape, dtype=torch.float64, device="cuda")
    full[..., :x.shape[-1]] = x
    return full


def _ends(case, st):
    return [case["L"]] * case["N"] if st["lengths"] is None else st["lengths"].tolist()


def _exact_conv(case, st):
    N, C, L, W = case["N"], case["C"], case["L"], case["W"]
    w, bias = st["w"][:, :C].double(), st["bias"][:C].double()
    x, ends = _wide(st["x"], C), _ends(case, st)
    if case["pass"] == "bwd":
        dy = _wide(st["dy"], C)
        dx, dw, db = torch.zeros_like(x), torch.zeros_like(w), torch.zeros_like(bias)
        for n, end in enumerate(ends):
            s = bias.expand(end, C).clone()
            for k in range(min(W, end)):  # k positions back
                s[k:] += w[W - 1 - k] * x[n, :end - k]
            e = torch.exp(-s)
            ds = dy[n, :end] * (1 + e + s * e) / (1 + e) ** 2
            db += ds.sum(0)
            for k in range(min(W, end)):
                dx[n, :end - k] += w[W - 1 - k] * ds[k:]
                dw[W - 1 - k] += (ds[k:] * x[n, :end - k]).sum(0)
        return {"dx": _like(st["dx"], dx), "dw": _vector(st["dw"], dw), "dbias": _vector(st["dbias"], db)}
    state, y = st["state"].double(), torch.zeros_like(x)
    for n, (end, at) in enumerate(zip(ends, st["slots"].tolist())):
        line = torch.cat((_wide(st["state"][at:at + 1], C)[0], x[n, :end]))
        s = bias.expand(end, C).clone()
        for j in range(W):
            s += w[j] * line[j:j + end]
        y[n, :end] = s / (1 + torch.exp(-s))
        state[at:at + 1] = _like(st["state"][at:at + 1], line[len(line) - W + 1:].unsqueeze(0))
    return {"y": _like(st["y"], y), "state": state}


def _exact_scan(case, st):
    N, C, L, S, G = case["N"], case["C"], case["L"], case["S"], case["G"]
    x, D = _wide(st["x"], C), st["D"][:C].double()
    raw = _wide(st["dt"], C) + st["dt_bias"][:C].double()
    d = torch.logaddexp(raw, torch.zeros_like(raw))
    A = st["A"][:, :C].double()  # [S, C]
    group = torch.arange(C, device="cuda") // (C // G)
    B = _wide(st["B"], G * S).unflatten(2, (G, S)).transpose(2, 3)  # [N, L, S, G]
    Cm = _wide(st["C"], G * S).unflatten(2, (G, S)).transpose(2, 3)
    inside = torch.ones(N, L, 1, device="cuda", dtype=torch.float64)
    for n, end in enumerate(_ends(case, st)):
        inside[n, end:] = 0
    d = d * inside
    gate = None if st["z"] is None else _wide(st["z"], C)
    if case["pass"] != "bwd":
        at = st["slots"].long()
        h = st["state"][at][..., :C].double()
        y = torch.zeros_like(x)
        for l in range(L):
            h = torch.exp(d[:, l].unsqueeze(1) * A) * h + (d[:, l] * x[:, l]).unsqueeze(1) * B[:, l][..., group]
            y[:, l] = (h * Cm[:, l][..., group]).sum(1)
        y = (y + D * x) * inside
        if gate is not None:
            y = y * gate / (1 + torch.exp(-gate))
        state = st["state"].double()
        state[at, :, :C] = h
        return {"y": _like(st["y"], y), "state": state}
    dy = _wide(st["dy"], C) * inside
    keep = torch.zeros(L + 1, N, S, C, dtype=torch.float64, device="cuda")  # h before position l
    for l in range(L):
        keep[l + 1] = torch.exp(d[:, l].unsqueeze(1) * A) * keep[l] + (d[:, l] * x[:, l]).unsqueeze(1) * B[:, l][..., group]
    dz, dyp = None, dy
    if gate is not None:
        sig = 1 / (1 + torch.exp(-gate))
        y = D * x
        for l in range(L):
            y[:, l] += (keep[l + 1] * Cm[:, l][..., group]).sum(1)
        dz, dyp = dy * y * sig * (1 + gate - gate * sig), dy * gate * sig
    dx, dd = D * dyp, torch.zeros_like(x)
    dA = torch.zeros_like(A)
    dB, dC = torch.zeros(N, L, G, S, dtype=torch.float64, device="cuda"), torch.zeros(N, L, G, S, dtype=torch.float64, device="cuda")
    back = torch.zeros(N, S, C, dtype=torch.float64, device="cuda")  # what reaches h at l from later positions
    for l in reversed(range(L)):
        up, dl, xl = dyp[:, l].unsqueeze(1), d[:, l].unsqueeze(1), x[:, l].unsqueeze(1)
        Bl = B[:, l][..., group]
        dC[:, l] = (up * keep[l + 1]).unflatten(2, (G, C // G)).sum(3).transpose(1, 2)
        gl = back + up * Cm[:, l][..., group]
        dB[:, l] = (gl * dl * xl).unflatten(2, (G, C // G)).sum(3).transpose(1, 2)
        back = gl * torch.exp(dl * A)
        through = (gl * Bl).sum(1)
        dx[:, l] += d[:, l] * through
        dd[:, l] = (back * keep[l] * A).sum(1) + x[:, l] * through
        dA += (back * keep[l] * dl).sum(0)
    ddt = dd * inside / (1 + torch.exp(-raw))
    got = {"dx": _like(st["dx"], dx * inside), "ddt": _like(st["ddt"], ddt), "dA": _vector(st["dA"], dA), "dB": _like(st["dB"], dB.flatten(2) * inside),
           "dC": _like(st["dC"], dC.flatten(2)), "dD": _vector(st["dD"], (dyp * x).sum((0, 1))), "ddt_bias": _vector(st["ddt_bias"], ddt.sum((0, 1)))}
    if dz is not None:
        got["dz"] = _like(st["dz"], dz)
    return got


def _exact_norm(case, st):
    C, w = case["C"], st["w"][:case["C"]].double()
    if case["pass"] == "bwd":
        r, up = _wide(st["r"], C), _wide(st["dy"], C)
        ms = r.square().sum(-1, keepdim=True) / C + EPS
        unit = r / ms.sqrt()
        dx = (up * w - unit * (up * w * unit).sum(-1, keepdim=True) / C) / ms.sqrt()
        if st["dr"] is not None:
            dx = dx + _wide(st["dr"], C)
        return {"dx": _like(st["dx"], dx), "dw": _vector(st["dw"], (up * unit).sum((0, 1)))}
    r, got = _wide(st["x"], C), {}
    if st["res"] is not None:
        r = r + _wide(st["res"], C)
        got["r"] = _like(st["r"], r)
        r = r.to(_T[case["dtype"]]).double()  # (by definition the norm of what is stored)
    y = w * r / (r.square().sum(-1, keepdim=True) / C + EPS).sqrt()
    if case["pass"] == "q8":
        scale = y.abs().max(-1).values / 127
        got["scale"] = scale
        got["y"] = _like(st["q"], torch.round(y / scale.unsqueeze(-1)) * scale.unsqueeze(-1))
    else:
        got["y"] = _like(st["y"], y)
    return got


def _exact_mv4(case, st):
    M, C, K, group = case["M"], case["C"], case["K"], case["group"]
    words = st["wq"].reshape(-1, st["wq"].shape[1], 16, 4).long()  # [C/128][Kp][4 j + i][bytes]
    y = torch.zeros(M, K, dtype=torch.float64, device="cuda")
    x = st["x"][:, :C].double()
    for c0 in range(0, C, 8):  # eight channels: one word of each row
        word = words[c0 // 128, :K, (c0 % 32) // 8 * 4 + c0 % 128 // 32]
        for c in range(c0, min(c0 + 8, C)):
            nib = (word[:, (c - c0) // 2] >> (4 * ((c - c0) % 2))) & 15
            wt = torch.where(nib < 8, nib, nib - 16).double() * st["wscale"][c // group, :K].double()
            y += x[:, c:c + 1] * wt
    if st["xscale"] is not None:
        y = y * st["xscale"].double().unsqueeze(1)
    return {"y": _vector(st["y"], y)}
