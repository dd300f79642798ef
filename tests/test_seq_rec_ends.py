"""The recurrence's gradients in the oracle at the ends of what A may be, against differences of its forward pass."""
import numpy as np

import seq_rec_oracle as oracle
from test_seq_abi import difference


def test_numbers_of_A_above_zero_have_no_gradient():
    """They count as zero, so that the forward pass does not change with them: nothing comes in, the state stays the zero that it began with, and a sum of dh h is zero."""
    rng = np.random.default_rng(4)
    N, C, L = 2, 4, 6
    p = {k: rng.standard_normal((N, L, C)) for k in ("x", "f", "i", "z")}
    p["A"] = np.array([0.5, 3.5, -0.7, 30.0])
    dy = rng.standard_normal((N, L, C))
    g, err = oracle.rec_bwd(**p, dy=dy)
    loss = lambda A: float((oracle.rec(**{**p, "A": A})[0][0] * dy).sum())  # noqa: E731
    for c in range(C):
        d = difference(loss, p["A"], c)
        if p["A"][c] > 0:
            assert d == 0 and g["dA"][c] == 0 and err["dA"][c] == 0
            assert not g["df"][..., c].any() and not g["di"][..., c].any() and not g["dx"][..., c].any() and not g["dz"][..., c].any()
        else:
            assert abs(d - g["dA"][c]) < 1e-6 * (1 + abs(d)) and d != 0
