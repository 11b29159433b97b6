"""An infinity or a NaN in an adapter's second matrix (B in the forward, A in dx) changes its own column of the adapter's own rows and nothing
else, whichever kernel the number of rows brings: every other element has the bits that it has when the adapter is sound."""

import numpy as np
import pytest
import torch

from tests.test_adapters import Case, lib  # noqa: F401  (lib: a fixture of the module)

pytestmark = pytest.mark.gpu

# counts, K, N, rank: few rows, a block per tile, the large tiles, tiles cut between CUs
SHAPES = [((20,), 256, 264, 16), ((300, 50), 136, 264, 8), ((700, 90), 512, 520, 40), ((700, 90), 512, 512, 16), ((600,), 4096, 4096, 24),
          ((700, 300), 4104, 1000, 16)]


def same_but(sound, broken, rows, columns, what):
    """Bits the same but for `rows` x `columns`, which are not finite."""
    a, b = sound.view(torch.int16).cpu().numpy().copy(), broken.view(torch.int16).cpu().numpy().copy()
    own = np.ix_(rows, columns)
    assert not np.isfinite(broken.float().cpu().numpy()[own]).any(), what
    a[own] = b[own] = 0
    assert np.array_equal(a, b), (what, np.argwhere(a != b)[:8].tolist(), int((a != b).sum()))


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=[str(i) for i in range(len(SHAPES))])
def test_own_columns_of_own_rows(shape, dt):
    counts, K, N, rank = shape
    c = Case(counts, K, N, 3, rank, dt, mix="tokens", seed=K + N)
    y0, v = c.forward()
    dx0, _, _ = c.backward(v)
    first, last = len(counts) - 1, rank - 1
    own = [np.flatnonzero(c.host_row == 1), np.flatnonzero(c.host_row == 1)]
    bounds = np.cumsum([0, *counts])
    mine = own[0][(own[0] >= bounds[first]) & (own[0] < bounds[first + 1])]      # of the last expert
    kept = c.B.clone(), c.A.clone()
    c.B[1, first, 7, 2], c.B[1, first, 30, 0], c.B[1, first, N - 1, last] = float("-inf"), float("nan"), float("inf")
    y1, v1 = c.forward()
    assert torch.equal(v[:c.rows], v1[:c.rows])
    same_but(y0[:c.rows], y1[:c.rows], mine, [7, 30, N - 1], "y")
    c.B.copy_(kept[0])
    c.A[1, first, 2, 7], c.A[1, first, 0, 61], c.A[1, first, last, K - 1] = float("-inf"), float("nan"), float("inf")
    dx1, _, _ = c.backward(v)
    same_but(dx0[:c.rows], dx1[:c.rows], mine, [7, 61, K - 1], "dx")
