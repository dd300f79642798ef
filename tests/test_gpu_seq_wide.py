"""The sequence operators at sizes that reach their other loops: many workgroups' shares of the channels, results past the caches, states of a gigabyte."""
import numpy as np
import pytest
import torch

import seq_oracle as oracle
from seq_util import DTYPES, Seq, close, ints, rounded, vector, vlen
from test_gpu_seq_scan import bound
from paper_1808_05567_amd import seq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,C,S", [(512, 8192, 64), (700, 6000, 33)])
def test_steps_of_a_gigabyte_of_states(N, C, S, dtype):
    """Compared at every 397th channel of some sequences."""
    rng, slots, v = np.random.default_rng(4), N + 1, vlen(dtype)
    f = lambda c: rounded(rng.standard_normal((N, 1, c)).astype(np.float32), dtype)  # noqa: E731
    x, dt, z, B, Cm = f(C), 0.5 * f(C), f(C), f(S), f(S)
    A, bias = np.float64(np.float32(-np.exp(rng.uniform(-3, 2, (S, C))))), np.float64(np.float32(rng.uniform(-6, 0.5, C)))
    X, DT, Z, BT, CT, Y = (Seq(N, n, 1, dtype, "dense", t) for n, t in ((C, x), (C, dt), (C, z), (S, B), (S, Cm), (C, None)))
    h = seq.seq_scan_create(N, C, 1, S, dtype, slots=slots)
    state = torch.randn(slots, S, h.info.Cp, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    state[..., C:] = 0
    where, n, c = rng.permutation(slots)[:N], np.array([0, 1, N // 2, N - 1]), np.arange(0, C, 397)
    pick = lambda: state[torch.from_numpy(where[n]).cuda()][..., torch.from_numpy(c).cuda()].double().cpu().numpy()  # noqa: E731
    spare, old = state[np.setdiff1d(np.arange(slots), where)[0]].clone(), pick()
    seq.seq_scan_step(h, X.t, DT.t, vector(A, v), BT.t, CT.t, state, Y.t, z=Z.t, dt_bias=vector(bias, v), slots=ints(where))
    args = (x[n][..., c], dt[n][..., c], A[:, c], B[n], Cm[n])
    opt = dict(z=z[n][..., c], dt_bias=bias[c], state=old)
    (y, after), (my, ma) = oracle.scan(*args, **opt), oracle.scan(*args, **opt, mag=True)
    close(Y.get()[n][..., c], y, bound(1) * my, dtype == seq.SEQ_BF16, "y")
    close(pick(), after, bound(1) * ma, False, "state")
    assert torch.equal(spare, state[np.setdiff1d(np.arange(slots), where)[0]])
