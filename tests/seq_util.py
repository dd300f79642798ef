"""Helpers of the sequence operators' GPU tests: tensors in the library's layouts inside guarded memory, and bounds."""
import numpy as np
import torch

from paper_1808_05567_amd import seq

TORCH = {seq.SEQ_F32: torch.float32, seq.SEQ_BF16: torch.bfloat16}
DTYPES = (seq.SEQ_F32, seq.SEQ_BF16)
LAYOUTS = ("dense", "rows", "slice")
GUARD = 7.25  # (exact in every type)


def vlen(dtype):
    return 4 if dtype == seq.SEQ_F32 else 8


def rounded(x, dtype):
    """x as numbers of the type, in 64 bits."""
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32))
    return t.to(TORCH[dtype]).double().numpy()


class Seq:
    """A sequence tensor [N, Cb, L, v] in one of the layouts, inside memory that is checked to stay as it was.
    slice: some blocks of a wider tensor whose positions have gaps between them."""

    def __init__(self, N, C, L, dtype, layout="dense", data=None, v=None, torch_type=None, outside=None):
        v = v or vlen(dtype)
        Cb = -(-C // v)
        tt = torch_type or TORCH[dtype]
        self.C = C
        if layout == "dense":
            shape, pick = (N + 2, Cb, L, v), lambda t: t[1:N + 1]
        elif layout == "rows":
            shape, pick = (N + 2, L, Cb, v), lambda t: t[1:N + 1].permute(0, 2, 1, 3)
        else:
            shape, pick = (N, Cb + 3, L + 1, 3, v), lambda t: t[:, 2:Cb + 2, :L, 1]
        self.base = torch.full(shape, 7 if tt == torch.int8 else GUARD, dtype=tt, device="cuda")
        self.t = pick(self.base)
        self.inside = pick(torch.zeros(shape, dtype=torch.bool, device="cuda"))
        if data is None:  # an output: whatever is not written shows
            self.t.fill_(99 if tt == torch.int8 else float("nan"))
        else:
            full = torch.zeros(N, L, Cb * v, dtype=torch.float64)
            full[..., :C] = torch.from_numpy(np.ascontiguousarray(data, dtype=np.float64))
            self.t.copy_(full.view(N, L, Cb, v).permute(0, 2, 1, 3))
        self.before = self.base.clone()
        self.pick = pick

    def get(self):
        """[N, L, C] in 64 bits; what lies around it and, for results, the slots beyond C are checked."""
        N, Cb, L, v = self.t.shape
        mark = torch.zeros(self.base.shape, dtype=torch.bool, device="cuda")
        self.pick(mark).fill_(True)
        assert torch.equal(self.base[~mark], self.before[~mark]), "written outside the tensor"
        full = self.t.permute(0, 2, 1, 3).reshape(N, L, Cb * v).double().cpu().numpy()
        assert not full[..., self.C:].any(), "slots beyond C are not zero"
        return full[..., :self.C]


def vector(x, v, fill=0.0):
    """An fp32 vector (or rows of them), entries beyond C zero."""
    x = np.asarray(x, dtype=np.float32)
    Cp = -(-x.shape[-1] // v) * v
    full = np.full(x.shape[:-1] + (Cp,), fill, dtype=np.float32)
    full[..., :x.shape[-1]] = x
    return torch.from_numpy(full).cuda()


def nans(*shape):
    return torch.full(shape, float("nan"), device="cuda")


def close(got, ref, bound, bf16, what=""):
    """|got - ref| <= bound (of the fp32 arithmetic), plus one rounding to bf16 of what is then stored."""
    got, ref = np.asarray(got, dtype=np.float64), np.asarray(ref, dtype=np.float64)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    limit = bound + (2.0 ** -8 * (np.abs(ref) + bound) + 1e-38 if bf16 else 1e-38)
    bad = ~(np.abs(got - ref) <= limit)
    if bad.any():
        at = np.unravel_index(int(np.argmax(np.where(np.isnan(got), np.inf, np.abs(got - ref) / limit))), got.shape)
        raise AssertionError("%s: %d of %d out of bounds; worst at %s: got %r, wanted %r, allowed %.3g" % (
            what, int(bad.sum()), bad.size, at, got[at], ref[at], limit[at]))


def lengths_of(kind, N, L, rng):
    if kind == "none":
        return None
    if kind == "ragged":
        n = rng.integers(0, L + 1, N)
        n[0] = L
        if N > 1:
            n[1] = 0
        if N > 2:
            n[2] = min(1, L)
        return n.astype(np.int32)
    return np.resize(np.array([-3, L + 5], dtype=np.int32), N)  # (clamped to 0 and L)


def spoil(x, lengths):
    """NaN and infinities where a sequence has ended."""
    if lengths is None:
        return x
    x = x.copy()
    for n, end in enumerate(lengths):
        end = min(max(int(end), 0), x.shape[1])
        x[n, end:] = np.nan
        x[n, end::2] = np.inf
    return x


def ints(x):
    return None if x is None else torch.from_numpy(np.asarray(x, dtype=np.int32)).cuda()
