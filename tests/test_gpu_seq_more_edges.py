"""AdamW where a state leaves what its type holds."""
import pytest
import torch

from seq_util import DTYPES, TORCH
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
