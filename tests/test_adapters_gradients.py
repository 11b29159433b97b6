"""dA and dB where the split of their float32 factor into 16-bit summands, or its scaling, is what limits them."""

import numpy as np
import pytest
import torch

from tests.test_adapters import Case, DT, close, f64, lib  # noqa: F401  (lib: a fixture of the module)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("rank", [8, 32, 128])
def test_an_infinite_factor_leaves_the_other_ones_their_accuracy(rank, dt):
    """One column of t, and of v, of one adapter is infinite, the others are 2^-16: bounded as in test_adapters.py, 2^-15 S."""
    c = Case((90, 31), 128, 136, 3, rank, dt, mix="tokens", seed=rank)
    c.B[1, :, 5, 2] = float("inf")
    c.dy.mul_(2.0 ** -16)
    v = (torch.randn(c.rows + 5, rank, generator=torch.Generator().manual_seed(rank)) * 2.0 ** -16).cuda()
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


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("rank,counts", [(8, (40, 3)), (16, (130, 65)), (24, (70, 9)), (64, (64, 33)), (128, (100, 1))])
def test_factors_keep_float32_accuracy(rank, counts, dt):
    """x and dy have one number per column, a power of two, so that an element of dA or dB is one factor times it, and the split into 16-bit
    summands all that it can lose: (2^-8)^3 of the factor (bf16, three summands) or (2^-11)^2 (fp16, two), and a rounding of 2^-24 per summand.
    v has float32's 24 bits, a quarter of it far smaller than the rest.  t = s (b1 + 2^-8 b2 + 2^-15 b3) for numbers b of B: three products and
    their float32 sum, so two roundings more.
    fp16's smallest numbers are 2^-24 apart, so a second summand is off by 2^-25 at least: of factors that a power of two has brought to a
    largest of 2^13 or more, so by 2^-38 of the pair's largest factor at most."""
    c = Case(counts, 264, 264, 3, rank, dt, mix="tokens", seed=rank + 100)
    c.scale = torch.tensor([0.5, -4.0, 1.0], device="cuda")
    g = torch.Generator().manual_seed(rank)
    x, dy = torch.zeros(c.rows, 264), torch.zeros(c.rows, 264)
    for e, a, at in c.groups():
        for t, cols in ((x, 264), (dy, 200)):       # (columns of dy from 200 on make t)
            t[at[np.arange(cols) % len(at)], np.arange(cols)] = 2.0 ** torch.randint(-3, 4, (cols,), generator=g).float()
        start = 200 + torch.randint(0, 20, (len(at),), generator=g).numpy()
        for k, f in enumerate((1.0, 2.0 ** -8, 2.0 ** -15)):
            dy[at, start + 20 * k] = f
    tight_B, tight_t = dy[:, :200].clone(), dy.clone()
    for with_t in (False, True):
        z = tight_t.clone() if with_t else torch.cat([tight_B, torch.zeros(c.rows, 64)], 1)
        if with_t:
            z[:, :200] = 0
        c.x[:c.rows], c.dy[:c.rows] = x.to(DT[dt]).cuda(), z.to(DT[dt]).cuda()
        v = torch.randn(c.rows + 5, rank, generator=g)
        v[:, 1::4] *= 2.0 ** -18
        v = v.cuda()
        _, dA, dB = c.backward(v, dx=False)
        X, dY, Bm, V, dA, dB = (f64(t) for t in (c.x, c.dy, c.B, v, dA, dB))
        bits = 2.0 ** -24 + 4 * 2.0 ** -24 if dt == "bf16" else 2.0 ** -22 + 3 * 2.0 ** -24
        for e, a, at in c.groups():
            if a < 0:
                continue
            if with_t:
                t, S = c.s(a) * (dY[at] @ Bm[a, e]), abs(c.s(a)) * (np.abs(dY[at]) @ np.abs(Bm[a, e]))
                floor = 2.0 ** -38 * np.abs(t).max(initial=0.0) * np.abs(X[at]).sum(0)[None] if dt == "f16" else 0.0
                close(dA[a, e], t.T @ X[at], (bits + 2 * 2.0 ** -24) * (S.T @ np.abs(X[at])) + floor, "dA")
            else:
                floor = 2.0 ** -38 * abs(c.s(a)) * np.abs(V[at]).max(initial=0.0) * np.abs(dY[at]).sum(0)[:, None] if dt == "f16" else 0.0
                close(dB[a, e], c.s(a) * (dY[at].T @ V[at]), bits * abs(c.s(a)) * (np.abs(dY[at]).T @ np.abs(V[at])) + floor, "dB")
