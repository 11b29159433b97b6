"""dA and dB where the split of their float32 factor into 16-bit summands, or its scaling, is what limits them."""

import numpy as np
import pytest
import torch

from tests.test_adapters import Case, close, f64, lib  # noqa: F401  (lib: a fixture of the module)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("rank", [8, 32, 128])
def test_an_infinite_factor_leaves_the_other_ones_their_accuracy(rank, dt):
    """One column of t, and of v, of one adapter is infinite, the others are 2^-16: bounded as in test_adapters.py, 2^-15 S."""
    c = Case((90, 31), 128, 136, 3, rank, dt, mix="tokens", seed=rank)
    c.B[1, :, 5, 2] = float("inf")
    c.dy.mul_(2.0 ** -16)
    v = torch.randn(c.rows + 5, rank, device="cuda") * 2.0 ** -16
    own = np.flatnonzero(c.host_row == 1)
    v[own[::3], 4] = float("inf")
    _, dA, dB = c.backward(v, dx=False)
    x, B, dy, v, dA, dB = (f64(t) for t in (c.x, c.B, c.dy, v, dA, dB))
    B[1, :, 5, 2], v[own[::3], 4] = 0.0, 0.0       # (their products are looked at apart)
    for e, a, at in c.groups():
        if a < 0:
            continue
        t, S = c.s(a) * (dy[at] @ B[a, e]), abs(c.s(a)) * (np.abs(dy[at]) @ np.abs(B[a, e]))
        ranks = [j for j in range(rank) if a != 1 or j != 2]
        close(dA[a, e][ranks], (t.T @ x[at])[ranks], (2.0 ** -15 * (S.T @ np.abs(x[at])))[ranks], "dA")
        ranks = [j for j in range(rank) if a != 1 or j != 4]
        close(dB[a, e][:, ranks], (c.s(a) * (dy[at].T @ v[at]))[:, ranks], (2.0 ** -15 * abs(c.s(a)) * (np.abs(dy[at]).T @ np.abs(v[at])))[:, ranks], "dB")
        if a == 1 and len(at):
            assert not np.isfinite(dA[a, e][2]).any()
