"""AdamW where a state leaves what its type holds; the recurrence's forward builds for many workgroups whose results go past the caches."""
import re

import numpy as np
import pytest
import torch

import seq_rec_oracle as oracle
from seq_util import DTYPES, TORCH, Seq, close, ints, vector, vlen
from test_gpu_seq_rec import data, scratch, tensors
from paper_1808_05567_amd import seq

pytestmark = pytest.mark.gpu
BLOCK = 256


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("what", [1e20, -1e25, float("inf"), float("-inf"), float("nan")])
def test_a_state_that_is_not_finite(what, dtype):
    """v of a gradient whose square fp32 does not hold is infinite, and m too where the gradient is.  With 8 bits, all 256 numbers that share such a one's scale stand for
    NaN from then on and the parameters are NaN after the next step; in 32 bits it stops or spoils its own number."""
    n, at = 900, 300
    block = slice(at // BLOCK * BLOCK, at // BLOCK * BLOCK + BLOCK)
    finite = abs(what) < float("inf")
    for bits in (32, 8):
        h = seq.seq_adamw_create([n], dtype, bits, decay=0.1)
        gen = torch.Generator("cuda").manual_seed(1)
        p, g = torch.randn(n, device="cuda", generator=gen), torch.randn(n, device="cuda", generator=gen)
        g[at + 1] = 0  # (a code of zero stands for NaN as well)
        runs = []
        for spoilt in (False, True):
            q, d = p.clone(), g.to(TORCH[dtype])
            if spoilt:
                d[at] = what
            m, v, scales = seq.seq_adamw_states(h)
            seq.seq_adamw(h, seq.seq_adamw_tensors(h, [q], [d]), m, v, (1e-2, 1), scales=scales)
            held = (m.clone(), v.clone(), scales)
            if bits == 8:
                s = scales.view(2, -1, 1)
                held = [(x.view(-1, BLOCK) * k).view(-1) for x, k in zip(held, s)]
            first = q.clone()
            seq.seq_adamw(h, seq.seq_adamw_tensors(h, [q], [g.to(TORCH[dtype])]), m, v, (1e-2, 2), scales=scales)
            runs.append((first, q, held))
        (a, b, _), (c, d, (m, v, *_)) = runs
        others = torch.arange(n, device="cuda") != at
        assert torch.equal(a[others], c[others]) and bool(c[at].isfinite()) == finite
        if bits == 32:
            assert torch.equal(b[others], d[others]) and bool(d[at].isfinite()) == finite
            continue
        assert bool(v[block].isnan().all()) and bool(m[block].isfinite().all() if finite else m[block].isnan().all())
        beside = (torch.arange(n, device="cuda") < block.start) | (torch.arange(n, device="cuda") >= block.stop)
        assert torch.equal(b[beside], d[beside]) and bool(d[block].isnan().all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("layout,N,C,L", [("dense", 5, 1044, 1700), ("rows", 33, 1044, 260)])
def test_recurrence_of_more_than_16_megabytes_in_many_workgroups(layout, N, C, L, gate, dtype):
    """At least 512 workgroups, which ask for nothing ahead, each result past the caches; compared at every 61st channel and the last two."""
    rng, p = data(N, C, L, dtype, 6)
    lengths = rng.integers(0, L + 1, N)
    lengths[:3] = L, 0, 1
    t, opt, A, _ = tensors(p, N, C, L, gate, True, lengths, layout, dtype)
    Y, old = Seq(N, C, L, dtype, layout), rng.standard_normal((N, C)).astype(np.float32)
    st = vector(old, vlen(dtype))
    h = seq.seq_rec_create(N, C, L, dtype, slots=N, views={k: q.t for k, q in t.items()} | {"y": Y.t})
    assert int(re.search(r"columns=(\d+)", seq.seq_describe(h)).group(1)) >= 512 and N * h.info.Cb * L * 16 > 16 << 20
    seq.seq_rec_fwd(h, t["x"].t, t["f"].t, t["i"].t, A, Y.t, scratch(h), z=t["z"].t if gate else None, state_in=st, state_out=st, lengths=ints(lengths), **opt)
    some = np.append(np.arange(0, C, 61), [C - 2, C - 1])
    pick = {k: q[..., some] for k, q in p.items()}
    (y, after), (ey, ea) = oracle.rec(*(pick[k] for k in ("x", "f", "i", "A")), z=pick["z"] if gate else None, f_bias=pick["f_bias"], i_bias=pick["i_bias"],
                                      state=old[:, some], lengths=lengths)
    close(Y.get()[..., some], y, ey, dtype == seq.SEQ_BF16, "y")
    close(st.double().cpu().numpy()[:, some], after, ea, False, "state")
