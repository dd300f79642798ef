"""A state space block of a language model from the library's operators: trained and run over prompts on the blocked tensors of
its 1x1 convolutions, served over single tokens with 4-bit weights.

    r   = x + res                         seq_norm_fwd        (the residual stream, handed on)
    u   = norm(r)
    p   = W_in u         C -> 2 Ci        conv 1x1            its halves: the inner input and the gate z
    c   = silu(conv(p_x))                 seq_conv_fwd
    q   = W_mid c        Ci -> Ci + 2 Sp  conv 1x1            its parts: dt, B and C of the scan
    s   = scan(c, dt, A, B, C, D, z)      seq_scan_fwd
    out = W_out s        Ci -> C          conv 1x1

Sp is S rounded up to the blocks' channels, so that B and C are whole blocks.  Every step reads parts of the tensors of the one before
it in place, by their strides, and backwards writes them there.  All computation is the library's; torch holds memory, and
clears what lies behind the ends of sequences.
"""
from __future__ import annotations

import weakref

import torch

from . import conv, seq

_TORCH = {seq.SEQ_F32: torch.float32, seq.SEQ_BF16: torch.bfloat16}


class _Projection:
    """A 1x1 convolution over sequences: [N, Cb, L, v] -> [N, Kb, L, v]."""

    def __init__(self, N, L, C, K, dtype, device):
        self.h = conv.conv_create(N, C, K, 1, L, 1, 1, 1, 0, dtype)
        self.info = conv.conv_query(self.h)
        self.shape = (K, C, 1, 1)
        v = self.info.vlen
        self.wt = torch.empty(self.info.wt_bytes // (16 // v), dtype=_TORCH[dtype], device=device)
        self.dwt = torch.empty(self.info.dwt_bytes // 4, dtype=torch.float32, device=device)
        self.ws = torch.empty(max(16, self.info.workspace_bytes), dtype=torch.uint8, device=device)

    def __del__(self):
        try:
            conv.conv_destroy(self.h)
        except Exception:
            pass

    def set(self, w):
        """w: [K, C], logical."""
        conv.conv_pack_wt(self.h, w.to(self.wt.dtype).reshape(self.shape).contiguous(), self.wt)

    def fwd(self, x, y, residual=None):
        if residual is None:
            conv.conv_fwd_ws(self.h, x, self.wt, y, self.ws)
        else:
            conv.conv_fwd_fused(self.h, x, self.wt, y, residual=residual, ws=self.ws)

    def bwd(self, dy, dx):
        conv.conv_bwd_data_ws(self.h, dy, self.wt, dx, self.ws)

    def upd(self, x, dy):
        """The weights' gradient, logical [K, C], fp32."""
        conv.conv_upd_ws(self.h, x, dy, self.dwt, self.ws)
        out = torch.empty(self.shape, dtype=torch.float32, device=self.dwt.device)
        conv.conv_unpack_dwt(self.h, self.dwt, out)
        return out[:, :, 0, 0]


def init(C, Ci, S, W, seed=0, device="cuda"):
    """Seeded parameters of a block, logical and fp32: matrices [K, C], the convolution's taps [W, Ci], A [S, Ci]."""
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    step = torch.exp(torch.rand(Ci, generator=g) * 4.6 - 6.9)  # 1e-3 ... 1e-1
    p = {"norm": 1 + 0.1 * n(C), "w_in": n(2 * Ci, C) * C ** -0.5, "taps": n(W, Ci) * W ** -0.5, "bias": 0.1 * n(Ci),
         "w_dt": n(Ci, Ci) * 0.1 * Ci ** -0.5, "w_B": n(S, Ci) * Ci ** -0.5, "w_C": n(S, Ci) * Ci ** -0.5,
         "A": -torch.arange(1, S + 1, dtype=torch.float32).view(S, 1) * (0.8 + 0.4 * torch.rand(S, Ci, generator=g)), "D": torch.ones(Ci),
         "dt_bias": step + torch.log(-torch.expm1(-step)), "w_out": n(C, Ci) * Ci ** -0.5}
    return {k: t.to(device) for k, t in p.items()}


def _rows(*parts):
    """Matrices one below the other, each in as many rows as are given with it, the others zero."""
    w = torch.zeros(sum(n for n, _ in parts), parts[0][1].shape[1], device=parts[0][1].device)
    at = 0
    for n, t in parts:
        w[at:at + t.shape[0]] = t
        at += n
    return w


class SeqBlock:
    """The block over N sequences of L positions: ``forward`` for training and prompts, ``backward`` after it."""

    def __init__(self, N, L, C, Ci, S, W, params, dtype=seq.SEQ_BF16, slots=0, eps=1e-5, device="cuda"):
        self.dims, self.dtype, self.device, self.slots, self.eps = (N, L, C, Ci, S, W), dtype, torch.device(device), slots, eps
        v = self.v = 4 if dtype == seq.SEQ_F32 else 8
        up = lambda n: -(-n // v) * v  # noqa: E731
        self.Cp, self.Cip, self.Sp = up(C), up(Ci), up(S)
        # (an inner width that is no whole number of blocks is padded inside the projections' rows)
        self.w_in = _Projection(N, L, C, 2 * self.Cip, dtype, device)
        self.w_mid = _Projection(N, L, Ci, self.Cip + 2 * self.Sp, dtype, device)
        self.w_mid_t = _Projection(N, L, self.Cip + 2 * self.Sp, Ci, dtype, device)
        self.w_out = _Projection(N, L, Ci, C, dtype, device)
        f = lambda *s: torch.zeros(*s, device=self.device)  # noqa: E731
        self.params = {"norm": f(C), "w_in": f(2 * Ci, C), "taps": f(W, Ci), "bias": f(Ci), "w_dt": f(Ci, Ci), "w_B": f(S, Ci), "w_C": f(S, Ci),
                       "A": f(S, Ci), "D": f(Ci), "dt_bias": f(Ci), "w_out": f(C, Ci)}
        self.nw, self.taps, self.A = f(self.Cp), f(W, self.Cip), f(S, self.Cip)
        self.bias, self.D, self.dt_bias = f(self.Cip), f(self.Cip), f(self.Cip)
        self.steps = weakref.WeakSet()  # (those that are still used)
        self.load(params)

        T = self._tensor
        self.r, self.u, self.out = T(self.Cp), T(self.Cp), T(self.Cp)
        self.p, self.c, self.q, self.s = T(2 * self.Cip), T(self.Cip), T(self.Cip + 2 * self.Sp), T(self.Cip)
        self.px, self.pz = self._split(self.p, self.Cip)
        self.dt, self.B, self.Cm = self._split(self.q, self.Cip, self.Sp)
        self.grads = None
        self.norm = seq.seq_norm_create(N, C, L, dtype, eps)
        self.conv = seq.seq_conv_create(N, Ci, L, W, dtype, slots=slots, views={"x": self.px, "y": self.c, "dy": self.c, "dx": self.px})
        self.scan = seq.seq_scan_create(N, Ci, L, S, dtype, slots=slots, views={
            "x": self.c, "dt": self.dt, "B": self.B, "C": self.Cm, "z": self.pz, "y": self.s,
            "dy": self.s, "dx": self.c, "ddt": self.dt, "dB": self.B, "dC": self.Cm, "dz": self.pz})
        self.positions = torch.arange(L, dtype=torch.int32, device=self.device)
        size = max(h.info.workspace_bytes for h in (self.norm, self.conv, self.scan))
        self.ws = torch.empty(max(16, size), dtype=torch.uint8, device=self.device)

    def _tensor(self, channels):
        N, L = self.dims[:2]
        return torch.zeros(N, channels // self.v, L, self.v, dtype=_TORCH[self.dtype], device=self.device)

    def _split(self, t, *channels):
        """Parts of the blocks of a tensor: those of the given channels, the last as wide as what is left over."""
        at = [0]
        for n in channels:
            at.append(at[-1] + n // self.v)
        return [t[:, a:b] for a, b in zip(at, at[1:] + [t.shape[1]])]

    @torch.no_grad()
    def load(self, params):
        """Parameters (as ``init`` makes them) into the layouts of the operators, and of its steps, each time into the same memory: a graph
        that was recorded before runs with the new ones.  The block keeps numbers of its own: a ``SeqBlockStep`` lays out what was loaded
        last, whatever the tensors given here hold by then."""
        for k, t in self.params.items():
            if params[k].shape != t.shape:
                raise ValueError("%s: a tensor of %s is wanted, not one of %s" % (k, tuple(t.shape), tuple(params[k].shape)))
        for k, t in self.params.items():
            t.copy_(params[k])
        p, Ci, Cip, Sp = self.params, self.dims[3], self.Cip, self.Sp
        self.w_in.set(_rows((Cip, p["w_in"][:Ci]), (Cip, p["w_in"][Ci:])))
        mid = _rows((Cip, p["w_dt"]), (Sp, p["w_B"]), (Sp, p["w_C"]))
        self.w_mid.set(mid)
        self.w_mid_t.set(mid.t())
        self.w_out.set(p["w_out"])
        for t, k in ((self.nw, "norm"), (self.taps, "taps"), (self.bias, "bias"), (self.A, "A"), (self.D, "D"), (self.dt_bias, "dt_bias")):
            t[..., :p[k].shape[-1]] = p[k]
        for step in self.steps:
            step.load()

    def forward(self, x, res, states=None, at=None, lengths=None):
        """x, res: blocked [N, Cb, L, v].  states: the pair that ``states`` makes, moved on from slots `at`; lengths: int32 [N], positions of each
        sequence: what lies beyond may be anything and comes out as zero.  Returns the output and the residual stream."""
        seq.seq_norm_fwd(self.norm, x, res, self.nw, self.r, self.u)
        if lengths is not None:
            # (the norm and the projections take each position on its own, but the gradients of their weights are sums over all of them)
            outside = self._outside(lengths)
            self.r.masked_fill_(outside, 0)
            self.u.masked_fill_(outside, 0)
        self.w_in.fwd(self.u, self.p)
        before, h = states if states is not None else (None, None)
        seq.seq_conv_fwd(self.conv, self.px, self.taps, self.bias, self.c, state_in=before, state_out=before, slots=at, lengths=lengths)
        self.w_mid.fwd(self.c, self.q)
        seq.seq_scan_fwd(self.scan, self.c, self.dt, self.A, self.B, self.Cm, self.s, self.ws, D=self.D, z=self.pz, dt_bias=self.dt_bias,
                         state_in=h, state_out=h, slots=at, lengths=lengths)
        self.w_out.fwd(self.s, self.out)
        return self.out, self.r

    def _outside(self, lengths):
        """[N, 1, L, 1]: the positions that lie behind their sequence's end."""
        N, L = self.dims[:2]
        seq._t(lengths, torch.int32, N, "lengths")
        return (self.positions >= lengths.flatten()[:N].view(N, 1)).view(N, 1, L, 1)

    def _cleared(self, t, outside):
        """A copy of a gradient with zeros outside."""
        return t.as_strided(self.out.shape, self.out.stride()).masked_fill(outside, 0)

    def states(self):
        """Zero states for the block's slots: of the convolution and of the scan."""
        N, L, C, Ci, S, W = self.dims
        return (torch.zeros(self.slots, self.Cip // self.v, W - 1, self.v, dtype=_TORCH[self.dtype], device=self.device),
                torch.zeros(self.slots, S, self.Cip, device=self.device))

    def backward(self, dout, dr, lengths=None):
        """Gradients of the last ``forward`` without states: of x (and of res, which is the same), and a dict of the parameters'.
        lengths: those of ``forward``; dout and dr beyond may be anything, and the gradient of x is zero there.  dr may be None."""
        N, L, C, Ci, S, W = self.dims
        r = self.r
        # (the projections take pointers as they come)
        seq._s(self.norm, "dy", dout)
        seq._so(self.norm, "dr", dr)
        if lengths is not None:
            outside = self._outside(lengths)
            dout, dr = self._cleared(dout, outside), None if dr is None else self._cleared(dr, outside)
            if self.eps == 0:
                r = r.masked_fill(outside, 1)  # (zeros have no norm then; any number does where its gradient is zero)
        if self.grads is None:
            T = self._tensor
            self.grads = {"ds": T(self.Cip), "dq": T(self.Cip + 2 * self.Sp), "dp": T(2 * self.Cip), "dc": T(self.Cip), "du": T(self.Cp), "dx": T(self.Cp)}
        t = self.grads
        f = lambda *s: torch.empty(*s, device=self.device)  # noqa: E731
        g = {"taps": f(W, self.Cip), "bias": f(self.Cip), "A": f(S, self.Cip), "D": f(self.Cip), "dt_bias": f(self.Cip), "norm": f(self.Cp)}
        self.w_out.bwd(dout, t["ds"])
        g["w_out"] = self.w_out.upd(self.s, dout)
        ddt, dB, dC = self._split(t["dq"], self.Cip, self.Sp)
        dpx, dpz = self._split(t["dp"], self.Cip)
        seq.seq_scan_bwd(self.scan, self.c, self.dt, self.A, self.B, self.Cm, t["ds"], t["dc"], ddt, g["A"], dB, dC, self.ws, D=self.D, z=self.pz,
                         dt_bias=self.dt_bias, dD=g["D"], dz=dpz, ddt_bias=g["dt_bias"], lengths=lengths)
        mid = self.w_mid.upd(self.c, t["dq"])
        g["w_dt"], g["w_B"], g["w_C"] = mid[:Ci], mid[self.Cip:self.Cip + S], mid[self.Cip + self.Sp:self.Cip + self.Sp + S]
        # (c goes into the scan and into W_mid: the second gradient is added to the first as the projection stores it)
        self.w_mid_t.fwd(t["dq"], t["dc"], residual=t["dc"])
        seq.seq_conv_bwd(self.conv, self.px, self.taps, self.bias, t["dc"], dpx, g["taps"], g["bias"], self.ws, lengths=lengths)
        w_in = self.w_in.upd(self.u, t["dp"])
        g["w_in"] = torch.cat((w_in[:Ci], w_in[self.Cip:self.Cip + Ci]))
        self.w_in.bwd(t["dp"], t["du"])
        seq.seq_norm_bwd(self.norm, r, self.nw, t["du"], dr, t["dx"], g["norm"], self.ws)
        for k, n in (("taps", Ci), ("bias", Ci), ("A", Ci), ("D", Ci), ("dt_bias", Ci), ("norm", C)):
            g[k] = g[k][..., :n]
        return t["dx"], g


class SeqBlockStep:
    """The block over one new token of each of M sequences, its projections in 4 bits; the norm hands its result on in 8.
    eps: the block's where none is given."""

    def __init__(self, block: SeqBlock, M, group=64, eps=None):
        N, L, C, Ci, S, W = block.dims
        if block.dtype != seq.SEQ_BF16:
            raise ValueError("single tokens are served in bf16")
        self.block, dev, slots = block, block.device, block.slots
        v, Cip, Sp = block.v, block.Cip, block.Sp
        T = lambda n: torch.zeros(M, n // v, 1, v, dtype=torch.bfloat16, device=dev)  # noqa: E731
        self.r, self.out = T(block.Cp), T(block.Cp)
        self.p, self.c, self.q, self.s = T(2 * Cip), T(Cip), T(Cip + 2 * Sp), T(Cip)
        self.px, self.pz = block._split(self.p, Cip)
        self.dt, self.B, self.Cm = block._split(self.q, Cip, Sp)
        self.u = torch.zeros(M, -(-C // 16), 1, 16, dtype=torch.int8, device=dev)
        self.scale = torch.zeros(M, 1, device=dev)
        self.norm = seq.seq_norm_create(M, C, 1, seq.SEQ_BF16, block.eps if eps is None else eps)
        self.conv = seq.seq_conv_create(M, Ci, 1, W, seq.SEQ_BF16, slots=slots, views={"x": self.px})
        self.scan = seq.seq_scan_create(M, Ci, 1, S, seq.SEQ_BF16, slots=slots, views={"x": self.c, "dt": self.dt, "B": self.B, "C": self.Cm, "z": self.pz})

        def quantised(dtype, C, K):
            h = seq.seq_mv4_create(M, C, K, group, dtype)
            return h, torch.empty(h.info.wt_bytes, dtype=torch.uint8, device=dev), torch.empty(h.info.scale_bytes // 4, device=dev)
        self.w_in = quantised(seq.SEQ_I8, C, 2 * Cip)
        self.w_mid = quantised(seq.SEQ_BF16, Ci, Cip + 2 * Sp)
        self.w_out = quantised(seq.SEQ_BF16, Ci, block.Cp)
        self.load()
        block.steps.add(self)

    def load(self):
        """The block's projections into 4 bits, as ``SeqBlock.load`` does with each step of the block."""
        b, p, Ci = self.block, self.block.params, self.block.dims[3]
        for (h, wt, scale), *parts in ((self.w_in, (b.Cip, p["w_in"][:Ci]), (b.Cip, p["w_in"][Ci:])),
                                       (self.w_mid, (b.Cip, p["w_dt"]), (b.Sp, p["w_B"]), (b.Sp, p["w_C"])), (self.w_out, (b.Cp, p["w_out"]))):
            seq.seq_mv4_quant(h, _rows(*parts), wt, scale)

    def __call__(self, x, res, states, at=None):
        """x, res: [M, Cb, 1, v]; states and slots as for ``SeqBlock.forward``."""
        b = self.block
        before, h = states
        seq.seq_norm_fwd_q8(self.norm, x, res, b.nw, self.r, self.u, self.scale)
        seq.seq_mv4(self.w_in[0], self.u, self.w_in[1], self.w_in[2], self.p, xscale=self.scale)
        seq.seq_conv_step(self.conv, self.px, b.taps, b.bias, before, self.c, slots=at)
        seq.seq_mv4(self.w_mid[0], self.c, self.w_mid[1], self.w_mid[2], self.q)
        seq.seq_scan_step(self.scan, self.c, self.dt, b.A, self.B, self.Cm, h, self.s, D=b.D, z=self.pz, dt_bias=b.dt_bias, slots=at)
        seq.seq_mv4(self.w_out[0], self.s, self.w_out[1], self.w_out[2], self.out)
        return self.out, self.r


def main():
    """Times a training step of a block and single tokens of a batch: python -m paper_1808_05567_amd.seq_block"""
    N, L, C, Ci, S, W, M = 2, 2048, 1024, 2048, 16, 4, 16

    def timed(f, n=20):
        f()
        torch.cuda.synchronize()
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(n):
            f()
        b.record()
        torch.cuda.synchronize()
        return a.elapsed_time(b) / n * 1e3
    block = SeqBlock(N, L, C, Ci, S, W, init(C, Ci, S, W), slots=M)
    x, res, dout, dr = (torch.randn(N, C // 8, L, 8, device="cuda").to(torch.bfloat16) for _ in range(4))
    print("block %d -> %d, %d states, bf16: forward of %d x %d positions %.0f us" % (C, Ci, S, N, L, timed(lambda: block.forward(x, res))))
    print("forward and backward %.0f us" % timed(lambda: (block.forward(x, res), block.backward(dout, dr))))
    step, states = SeqBlockStep(block, M), block.states()
    x1, r1 = (torch.randn(M, C // 8, 1, 8, device="cuda").to(torch.bfloat16) for _ in range(2))
    each = timed(lambda: step(x1, r1, states), 200)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(x1, r1, states)
    print("one token of %d sequences, 4-bit weights %.1f us, captured %.1f us" % (M, each, timed(graph.replay, 200)))


if __name__ == "__main__":
    main()
