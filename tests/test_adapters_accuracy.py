"""The low-rank part of moe_adapter_forward and moe_adapter_backward where it outweighs the projection: it has float32's accuracy up
to the one rounding of the result.

Tolerances, in units of the magnitude sums as in test_adapters.py: S of all terms, S_low of the low-rank terms.
  y, dx  one rounding of the result, eps / 2 of it; the float32 sums, 2^-17 S there; a factor of the low-rank terms as two 16-bit summands: a
         summand is off by at most eps / 2 of what it rounds, so the two by (eps / 2)^2 of the factor: 2^-16 S_low (bf16) or 2^-22 (fp16).  fp16's smallest
         numbers are half a step of 2^-25 apart: of the result, and of each of the `rank` factors relative to the row's largest, which is
         at least 2^-4 or brought to 2^13."""

import numpy as np
import pytest
import torch

from paper_2304_11414_amd import binding as B
from tests.test_adapters import Case, DT, close, f64, gelu64, lib  # noqa: F401  (lib: a fixture of the module)

pytestmark = pytest.mark.gpu


def check_product(c, out, x, W, A, Bm, v=None):
    """out = x W + s (x A) B, row by row of the case; W [E, n, k], A [adapters, E, rank, k], B [adapters, E, n, rank]."""
    half = torch.finfo(DT[c.dt]).eps / 2
    tiny = 2.0 ** -25 if c.dt == "f16" else 0.0
    for e, a, at in c.groups():
        u, S, low, top = x[at] @ W[e].T, np.abs(x[at]) @ np.abs(W[e]).T, 0.0, np.zeros((len(at), 1))
        if a >= 0:
            factor, size = c.s(a) * (x[at] @ A[a, e].T), abs(c.s(a)) * (np.abs(x[at]) @ np.abs(A[a, e]).T)
            low = np.abs(factor) @ np.abs(Bm[a, e]).T
            top = np.abs(factor).max(1, keepdims=True) * np.abs(Bm[a, e]).sum(1)[None]
            u, S = u + factor @ Bm[a, e].T, S + size @ np.abs(Bm[a, e]).T
        off = 1.01 * half * half * low + 2.0 ** -17 * S + (2.0 ** -21 * top if c.dt == "f16" else 0.0)
        if c.gelu:
            u, off = gelu64(u), 1.13 * off + 2.0 ** -18 * np.abs(u)
        close(out[at], u, off + half * (np.abs(u) + off) + tiny, "rows of expert %d, adapter %d" % (e, a))


# counts, K, N, adapters, rank: by the kernel that adds the low-rank part
FEW = [((1,), 64, 64, 1, 8, dict(perm=False)), ((3, 0, 17, 12), 256, 520, 5, 16, dict(mix="tokens", top_k=2)),
       ((64, 40), 1000, 72, 3, 64, dict(mix="tokens")), ((33,), 512, 264, 40, 24, dict(mix="tokens", gelu=True))]


def check_both(shape, dt, strong=8.0):
    """Adapters `strong` times the projection's size."""
    counts, K, N, n_a, rank, more = shape
    c = Case(counts, K, N, n_a, rank, dt, seed=K + rank, **more)
    c.scale = (c.scale if c.scale is not None else torch.ones(n_a, device="cuda")) * strong
    y, v = c.forward()
    x, dy, W, A, Bm = (f64(t) for t in (c.x, c.dy, c.W, c.A, c.B))
    check_product(c, f64(y), x, W, A, Bm)
    c.gelu, c.cfg.activation = False, B.MOE_ACT_NONE
    dx, _, _ = c.backward(v)
    check_product(c, f64(dx), dy, W.transpose(0, 2, 1), Bm.transpose(0, 1, 3, 2), A.transpose(0, 1, 3, 2))


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("shape", FEW, ids=[str(i) for i in range(len(FEW))])
def test_few_rows(shape, dt):
    check_both(shape, dt)


TILES = [((130, 7), 72, 136, 3, 8, dict()), ((300, 500), 328, 1000, 4, 40, dict(mix="tokens")), ((700, 0, 260, 1), 512, 512, 6, 16, dict(top_k=2)),
         ((513,), 1024, 768, 2, 128, dict(perm=False, scale=False)), ((600, 90), 1000, 1032, 9, 32, dict(gelu=True)),
         ((1500,), 128, 256, 64, 8, dict(mix="tokens")), ((600,), 4096, 4096, 3, 24, dict(mix="tokens")),
         ((700, 300), 4104, 1000, 3, 32, dict(mix="tokens"))]


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("shape", TILES, ids=[str(i) for i in range(len(TILES))])
def test_tiles(shape, dt):
    check_both(shape, dt)


@pytest.mark.parametrize("projection", [True, False], ids=["projection", "zeros"])
@pytest.mark.parametrize("shape", FEW + TILES, ids=[str(i) for i in range(len(FEW + TILES))])
def test_fp16_factors_of_any_size(shape, projection):
    """scale v and t far beyond fp16's range, and far below it, where y and dx are not: rows of adapters of several sizes side by side."""
    counts, K, N, n_a, rank, more = shape
    sizes = [2.0 ** (18, 0, -20, 10, -12, 30)[i % 6] for i in range(n_a)]
    back = [2.0 ** (-10, 0, 10, -6, 8, -14)[i % 6] for i in range(n_a)]
    for backward in (False, True):
        c = Case(counts, K, N, n_a, rank, "f16", seed=K + rank + 1, **{**more, "gelu": False})
        c.scale = torch.tensor(sizes, device="cuda")
        second = c.A if backward else c.B
        second.mul_(torch.tensor(back, device="cuda", dtype=torch.float16).view(-1, 1, 1, 1))
        if sizes[-1] == 2.0 ** 30 or n_a > 5:      # 2^30 * 2^-14 * 2^-14 in the other factor as well
            (c.B if backward else c.A)[5::6].mul_(2.0 ** -8)
        if not projection:
            c.W.zero_()
        x, dy, W, A, Bm = (f64(t) for t in (c.x, c.dy, c.W, c.A, c.B))
        if not backward:
            check_product(c, f64(c.forward()[0]), x, W, A, Bm)
        else:
            v = torch.zeros(c.rows + 5, rank, device="cuda")
            check_product(c, f64(c.backward(v)[0]), dy, W.transpose(0, 2, 1), Bm.transpose(0, 1, 3, 2), A.transpose(0, 1, 3, 2))
