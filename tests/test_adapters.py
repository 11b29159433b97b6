"""Low-rank adapters beside the experts' projections (moe_adapter_forward, moe_adapter_backward): refusals on the CPU; on the
GPU against the definition in float64.

Tolerances, in units of the magnitude sums S = sum of |factor| |factor| over the terms of an element (every rounding is relative to a term or to a partial sum, each
at most S):
  v      float32 sums of exact products: an element is at most 32 products in an instruction, 8 instructions one after another per
         wavefront and 8 wavefronts (contractions of 2048): 48 roundings, below 2^-18 S.
  y, dx  one rounding of the result, half a step eps / 2 of it; the low-rank summand's factor is rounded once, eps / 2 of its terms (S_low); the float32
         sums 32 + 64 roundings, below 2^-17 S.  GeLU: |GeLU'| <= 1.13 and its own float32 arithmetic, 2^-18 of the argument.
  dA, dB u as at least two 16-bit summands: 2^-17 of each term (8 bits, then 8 of the rest), t as v; over 2000 rows 32 + 2 * 63 roundings and at most
         32 pieces: below 2^-16 S; together 2^-15 S."""

import ctypes
import os

import numpy as np
import pytest
import torch  # before the library is loaded: both then share one HIP runtime

from paper_2304_11414_amd import binding as B
from paper_2304_11414_amd import build as build_mod

gpu = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(B.LIB_PATH):
        build_mod.build_library()
    return B.load_library()


# ---- CPU: refusals -----------------------------------------------------------------------------------

GOOD = dict(rows=100, K=64, N=128, n_exp=2, n_adapters=3, rank=16)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), -2), (dict(K=0), -2), (dict(K=60), -2), (dict(N=4), -2), (dict(N=(1 << 20) + 8), -2), (dict(K=1 << 21), -2),
    (dict(n_exp=0), -2), (dict(n_exp=257), -2), (dict(n_adapters=0), -2), (dict(n_adapters=32769), -2), (dict(rank=0), -2), (dict(rank=12), -2),
    (dict(rank=136), -2), (dict(top_k=0), -2), (dict(top_k=9), -2), (dict(dtype="f32"), -3)])
def test_configurations_refused(kw, status):
    lib, cfg = B.load_library(), B.make_adapter_config(**{**GOOD, **kw})
    p = ctypes.c_void_p(0x1000)
    assert lib.moe_adapter_workspace_bytes(ctypes.byref(cfg)) == 0
    assert lib.moe_adapter_backward_workspace_bytes(ctypes.byref(cfg)) == 0
    assert lib.moe_adapter_forward(ctypes.byref(cfg), *[p] * 11, 1 << 40, None) == status
    assert lib.moe_adapter_backward(ctypes.byref(cfg), *[p] * 14, 1 << 40, None) == status


def test_arguments_refused():
    lib, cfg = B.load_library(), B.make_adapter_config(**GOOD)
    c, p, odd = ctypes.byref(cfg), ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008)
    need, needb = lib.moe_adapter_workspace_bytes(c), lib.moe_adapter_backward_workspace_bytes(c)
    assert 0 < need < needb
    assert lib.moe_adapter_forward(None, *[p] * 11, need, None) == -1
    for i in range(11):
        a = [p] * 11
        a[i] = odd
        assert lib.moe_adapter_forward(c, *a, need, None) == -4
        a[i] = None
        if i not in (5, 7):              # scale and perm may be NULL
            assert lib.moe_adapter_forward(c, *a, need, None) == -1
    assert lib.moe_adapter_forward(c, *[p] * 11, need - 1, None) == -5
    for i in range(14):
        a = [p] * 14
        a[i] = odd
        assert lib.moe_adapter_backward(c, *a, needb, None) == -4
        a[i] = None
        if i not in (5, 7, 10):          # nor dx
            assert lib.moe_adapter_backward(c, *a, needb, None) == -1
    assert lib.moe_adapter_backward(c, *[p] * 14, needb - 1, None) == -5
    gelu = B.make_adapter_config(**GOOD, gelu=True)
    assert lib.moe_adapter_backward_workspace_bytes(ctypes.byref(gelu)) == 0
    assert lib.moe_adapter_backward(ctypes.byref(gelu), *[p] * 14, needb, None) == -2
    gelu.activation = 7
    assert lib.moe_adapter_forward(ctypes.byref(gelu), *[p] * 11, need, None) == -2
    empty = B.make_adapter_config(**{**GOOD, "rows": 0})
    assert lib.moe_adapter_forward(ctypes.byref(empty), *[None] * 11, 0, None) == 0


def test_overlapping_memory_is_refused():
    lib, cfg = B.load_library(), B.make_adapter_config(**GOOD)
    c = ctypes.byref(cfg)
    MB = 1 << 20
    for call, need, n, written in ((lib.moe_adapter_forward, lib.moe_adapter_workspace_bytes(c), 11, (8, 9, 10)),
                                   (lib.moe_adapter_backward, lib.moe_adapter_backward_workspace_bytes(c), 14, (10, 11, 12, 13))):
        at = [(i + 1) * 1024 * MB for i in range(n)]
        for w in written:
            for other in range(n):
                if other != w:
                    a = list(at)
                    a[w] = a[other]
                    assert call(c, *map(ctypes.c_void_p, a), need, None) == -7, (n, w, other)
        a = list(at)
        a[-1] = at[0] - need + 16        # a workspace whose end reaches into x
        assert call(c, *map(ctypes.c_void_p, a), need, None) == -7


def test_backwards_of_more_than_a_grid_holds_are_refused():
    lib = B.load_library()
    most = B.make_adapter_config(rows=64, K=2048, N=2048, n_exp=1, n_adapters=65536, rank=128)
    assert lib.moe_adapter_backward_workspace_bytes(ctypes.byref(most)) > 0
    more = B.make_adapter_config(rows=64, K=2048, N=2056, n_exp=1, n_adapters=65536, rank=8)
    p = [ctypes.c_void_p((i + 1) << 44) for i in range(14)]
    assert lib.moe_adapter_backward_workspace_bytes(ctypes.byref(more)) == 0
    assert lib.moe_adapter_workspace_bytes(ctypes.byref(more)) > 0
    assert lib.moe_adapter_backward(ctypes.byref(more), *p, 1 << 43, None) == -2


# ---- GPU ---------------------------------------------------------------------------------------------

class Case:
    """Inputs of a call, packed by expert, in buffers with rows past the last one."""

    def __init__(self, counts, K, N, n_adapters, rank, dt="bf16", top_k=1, mix="requests", seed=0, extra=5, perm=True, scale=True, gelu=False):
        g = torch.Generator().manual_seed(seed)
        rows, E = sum(counts), len(counts)
        self.counts, self.rows, self.E, self.dt, self.gelu, self.top_k = counts, rows, E, dt, gelu, top_k
        self.K, self.N, self.n_adapters, self.rank = K, N, n_adapters, rank
        tokens = max(1, -(-rows // top_k))     # (an array without elements would be a NULL pointer)
        if mix == "tokens":
            adapter = torch.randint(-1, n_adapters, (tokens,), generator=g)
        elif mix == "none":
            adapter = torch.full((tokens,), -1)
        else:
            adapter = torch.randint(-1, n_adapters, (7,), generator=g).repeat_interleave(-(-tokens // 7))[:tokens]
        adapter[::11] = torch.where(adapter[::11] < 0, torch.tensor(n_adapters + 3), adapter[::11])    # out of range: none as well
        # any assignment order; ascending inside an expert, as the dispatch has it
        order = torch.randperm(tokens * top_k, generator=g)[:rows] if perm else torch.arange(rows)
        parts, at = [], 0
        for n in counts:
            parts.append(order[at:at + n].sort().values)
            at += n
        order = torch.cat(parts) if parts else order
        self.host_row = adapter[order // top_k] if perm else adapter[:rows]
        self.host_row = torch.where((self.host_row < 0) | (self.host_row >= n_adapters), -1, self.host_row).numpy()
        normal = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(DT[dt]).cuda()
        self.x, self.dy = normal(rows + extra, K), normal(rows + extra, N)
        self.x[rows:], self.dy[rows:] = float("nan"), float("nan")                                     # never read
        self.W, self.A, self.B = normal(E, N, K, std=K ** -0.5), normal(n_adapters, E, rank, K, std=K ** -0.5), normal(n_adapters, E, N, rank, std=rank ** -0.5)
        self.scale = (torch.rand(n_adapters, generator=g) * 3 - 1).cuda() if scale else None
        self.adapter = adapter.to(torch.int32).cuda()
        self.perm = torch.cat([order, torch.zeros(extra)]).to(torch.int32).cuda() if perm else None
        self.offsets = torch.tensor([0, *np.cumsum(counts)], dtype=torch.int32, device="cuda")
        self.cfg = B.make_adapter_config(rows + extra, K, N, E, n_adapters, rank, top_k, dt, gelu)

    def forward(self, workspace=None, stream=None):
        y = torch.full((self.rows + 5, self.N), 7.0, dtype=DT[self.dt], device="cuda")
        v = torch.full((self.rows + 5, self.rank), 7.0, device="cuda")
        ws = torch.empty(B.moe_adapter_workspace_bytes(self.cfg), dtype=torch.uint8, device="cuda").fill_(0xA5) if workspace is None else workspace
        B.moe_adapter_forward(self.cfg, self.x, self.offsets, self.W, self.A, self.B, self.scale, self.adapter, self.perm, y, v, ws, stream)
        return y, v

    def backward(self, v, dx=True):
        out = torch.full((self.rows + 5, self.K), 7.0, dtype=DT[self.dt], device="cuda") if dx else None
        dA = torch.full(tuple(self.A.shape), 7.0, device="cuda")
        dB = torch.full(tuple(self.B.shape), 7.0, device="cuda")
        ws = torch.empty(B.moe_adapter_backward_workspace_bytes(self.cfg), dtype=torch.uint8, device="cuda").fill_(0xA5)
        B.moe_adapter_backward(self.cfg, self.x, self.offsets, self.W, self.A, self.B, self.scale, self.adapter, self.perm, self.dy, v, out, dA, dB, ws)
        return out, dA, dB

    def groups(self):
        lo = 0
        for e, n in enumerate(self.counts):
            for a in np.unique(self.host_row[lo:lo + n]):
                yield e, int(a), lo + np.flatnonzero(self.host_row[lo:lo + n] == a)
            lo += n

    def s(self, a):
        return 1.0 if self.scale is None else float(self.scale[a])


def f64(t):
    return t.double().cpu().numpy()


def close(got, want, bound, what):
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:5].tolist(), got[bad][:5], want[bad][:5], bound[bad][:5])


def gelu64(u):
    return u / (1.0 + np.exp(-2.0 * np.sqrt(2.0 / np.pi) * (u + 0.044715 * u ** 3)))


def check_forward(c, y, v):
    x, W, A, Bm, y, v = (f64(t) for t in (c.x, c.W, c.A, c.B, y, v))
    half = torch.finfo(DT[c.dt]).eps / 2
    tiny = 2.0 ** -25 if c.dt == "f16" else 0.0           # half a step of fp16's smallest numbers
    assert np.all(y[c.rows:] == 7.0) and np.all(v[c.rows:] == 7.0)
    for e, a, at in c.groups():
        u, S, low = x[at] @ W[e].T, np.abs(x[at]) @ np.abs(W[e]).T, 0.0
        if a < 0:
            assert np.all(v[at] == 0.0)
        else:
            want = x[at] @ A[a, e].T
            Sv = np.abs(x[at]) @ np.abs(A[a, e]).T
            close(v[at], want, 2.0 ** -18 * Sv, "v")
            low = abs(c.s(a)) * (np.abs(want) @ np.abs(Bm[a, e]).T)
            u = u + c.s(a) * (want @ Bm[a, e].T)
            S = S + abs(c.s(a)) * (Sv @ np.abs(Bm[a, e]).T)
        off = 1.01 * half * low + 2.0 ** -17 * S + tiny * c.rank
        want = u
        if c.gelu:
            want, off = gelu64(u), 1.13 * off + 2.0 ** -18 * np.abs(u)
        close(y[at], want, off + half * (np.abs(want) + off) + tiny, "y")


def check_backward(c, v, dx, dA, dB):
    x, W, A, Bm, dy, v, dA, dB = (f64(t) for t in (c.x, c.W, c.A, c.B, c.dy, v, dA, dB))
    half = torch.finfo(DT[c.dt]).eps / 2
    tiny = 2.0 ** -25 if c.dt == "f16" else 0.0
    wantA, wantB, SA, SB = (np.zeros(t.shape) for t in (dA, dB, dA, dB))
    if dx is not None:
        dx = f64(dx)
        assert np.all(dx[c.rows:] == 7.0)
    for e, a, at in c.groups():
        want, S, low = dy[at] @ W[e], np.abs(dy[at]) @ np.abs(W[e]), 0.0
        if a >= 0:
            t, St = c.s(a) * (dy[at] @ Bm[a, e]), abs(c.s(a)) * (np.abs(dy[at]) @ np.abs(Bm[a, e]))
            want, low, S = want + t @ A[a, e], np.abs(t) @ np.abs(A[a, e]), S + St @ np.abs(A[a, e])
            wantA[a, e], SA[a, e] = t.T @ x[at], St.T @ np.abs(x[at])
            wantB[a, e], SB[a, e] = c.s(a) * (dy[at].T @ v[at]), abs(c.s(a)) * (np.abs(dy[at]).T @ np.abs(v[at]))
        if dx is not None:
            off = 1.01 * half * low + 2.0 ** -17 * S + tiny * c.rank
            close(dx[at], want, off + half * (np.abs(want) + off) + tiny, "dx")
    close(dA, wantA, 2.0 ** -15 * SA, "dA")
    close(dB, wantB, 2.0 ** -15 * SB, "dB")


SHAPES = [
    # counts, K, N, adapters, rank, more: by kernel and by edge
    ((1,), 64, 64, 1, 8, dict(perm=False)),                                    # a single token
    ((1,), 2048, 8192, 8, 16, dict(mix="tokens", gelu=True)),
    ((3, 0, 17, 12), 256, 520, 5, 16, dict(mix="tokens", top_k=2)),            # few rows, an expert without any
    ((33,), 512, 264, 40, 24, dict(mix="tokens", gelu=True)),
    ((64, 40), 1000, 72, 3, 64, dict(mix="tokens")),                           # passes of 64 rows, K no multiple of 32
    ((130, 7), 72, 136, 3, 8, dict()),                                         # a short odd contraction: a block per tile
    ((300, 500), 328, 1000, 4, 40, dict(mix="tokens")),
    ((700, 0, 260, 1), 512, 512, 6, 16, dict(top_k=2)),                        # the large tiles, small ones among them
    ((513,), 1024, 768, 2, 128, dict(perm=False, scale=False)),                # the largest rank
    ((600, 90), 1000, 1032, 9, 32, dict(gelu=True)),                           # k-tiles cut by the row's end
    ((1500,), 128, 256, 64, 8, dict(mix="tokens")),                            # every adapter in every tile
    ((2000, 300), 2048, 512, 3, 16, dict(mix="requests")),                     # tiles cut between CUs
    ((400,), 192, 320, 2, 16, dict(mix="none")),
    ((2000, 300), 4096, 512, 5, 16, dict(mix="tokens")),                       # dx on the large tiles
    ((600,), 4096, 4096, 3, 24, dict(mix="tokens")),                           # dx on large tiles cut between CUs
    ((700, 300), 4104, 1000, 3, 32, dict(mix="tokens")),                       # dx, a block per tile
]


@gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=[str(i) for i in range(len(SHAPES))])
def test_forward(shape, dt):
    counts, K, N, n_a, rank, more = shape
    c = Case(counts, K, N, n_a, rank, dt, seed=K + N, **more)
    y, v = c.forward()
    torch.cuda.synchronize()
    check_forward(c, y, v)


@gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=[str(i) for i in range(len(SHAPES))])
def test_backward(shape, dt):
    counts, K, N, n_a, rank, more = shape
    c = Case(counts, K, N, n_a, rank, dt, seed=K + N + 1, **{**more, "gelu": False})
    v = torch.randn(c.rows + 5, rank, device="cuda")
    out = c.backward(v)
    torch.cuda.synchronize()
    check_backward(c, v, *out)
    again = c.backward(v, dx=False)                     # without dx; the same bits
    assert torch.equal(out[1], again[1]) and torch.equal(out[2], again[2])
    same = c.backward(v)
    assert torch.equal(out[0].view(torch.int16), same[0].view(torch.int16))


@gpu
def test_no_rows_give_zero_gradients():
    c = Case((0, 0), 64, 128, 3, 16, extra=5)
    v = torch.zeros(5, 16, device="cuda")
    dx, dA, dB = c.backward(v)
    assert torch.all(dA == 0) and torch.all(dB == 0) and torch.all(dx == 7.0)
    y, v = c.forward()
    assert torch.all(y == 7.0) and torch.all(v == 7.0)
    c.cfg.rows = 0
    B.moe_adapter_backward(c.cfg, None, c.offsets, None, None, None, None, None, None, None, None, None, dA.fill_(3.0), dB.fill_(3.0),
                           torch.empty(B.moe_adapter_backward_workspace_bytes(c.cfg), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    assert torch.all(dA == 0) and torch.all(dB == 0)


@gpu
@pytest.mark.parametrize("counts,K,N", [((20,), 256, 264), ((300, 50), 136, 264), ((700, 90), 512, 520), ((700, 90), 512, 512),
                                          ((600,), 4096, 4096), ((700, 300), 4104, 1000)])
def test_one_adapters_infinities_stay_with_its_rows(counts, K, N):
    """Rows of other adapters have the bits they have when that adapter is sound; its own rows are NaN where the definition is not
    finite."""
    sound, c = (Case(counts, K, N, 3, 16, mix="tokens", seed=4) for _ in range(2))
    c.A[1, 0, 3, 5] = float("inf")
    c.B[1, 0, 7, 2] = float("-inf")
    c.B[1, -1, 9, 15] = float("nan")
    y0, v0 = sound.forward()
    y1, v1 = c.forward()
    others = torch.from_numpy(np.flatnonzero(c.host_row != 1)).cuda()
    own = torch.from_numpy(np.flatnonzero(c.host_row[:counts[0]] == 1)).cuda()
    assert torch.equal(y0[others].view(torch.int16), y1[others].view(torch.int16))
    assert torch.equal(v0[others], v1[others])
    assert not torch.isfinite(y1[own].float()).any() and not torch.isfinite(v1[own, 3]).any()
    c.A[1, 0, 3, 5] = 0.5                                  # B's alone: their columns, at most their block of 32
    y1, _ = c.forward()
    assert not torch.isfinite(y1[own, 7].float()).any()
    assert torch.isfinite(y1[own][:, 64:].float()).all()
    dx0, dA0, dB0 = sound.backward(v0)
    dx1, dA1, dB1 = c.backward(v0)
    assert torch.equal(dx0[others].view(torch.int16), dx1[others].view(torch.int16))
    for g0, g1 in ((dA0, dA1), (dB0, dB1)):
        assert torch.equal(g0[[0, 2]], g1[[0, 2]])


@gpu
@pytest.mark.parametrize("counts,K,N", [((37, 5), 256, 512), ((900, 300), 512, 512)])
def test_rows_without_an_adapter_have_the_projection_bits(counts, K, N):
    c = Case(counts, K, N, 2, 16, mix="none", perm=False)
    y, _ = c.forward()
    layer = B.make_config(c.rows, N, K, c.E, 1)
    plain = torch.empty(c.rows, N, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(B.moe_ffn_workspace_bytes(layer), dtype=torch.uint8, device="cuda")
    B.moe_expert_ffn_down(layer, c.x, c.offsets, c.W, plain, ws)
    torch.cuda.synchronize()
    assert torch.equal(y[:c.rows].view(torch.int16), plain.view(torch.int16))


@gpu
@pytest.mark.parametrize("counts", [(40, 3), (900, 300)])
def test_captured_calls_replay_with_new_inputs(counts):
    c = Case(counts, 512, 512, 4, 16, mix="tokens", seed=8)
    other = Case(counts, 512, 512, 4, 16, mix="tokens", seed=9)
    B.moe_init()
    ws = torch.empty(B.moe_adapter_workspace_bytes(c.cfg), dtype=torch.uint8, device="cuda")
    wsb = torch.empty(B.moe_adapter_backward_workspace_bytes(c.cfg), dtype=torch.uint8, device="cuda")
    y, v = c.forward(ws)
    dx, dA, dB = c.backward(v)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.moe_adapter_forward(c.cfg, c.x, c.offsets, c.W, c.A, c.B, c.scale, c.adapter, c.perm, y, v, ws)
        B.moe_adapter_backward(c.cfg, c.x, c.offsets, c.W, c.A, c.B, c.scale, c.adapter, c.perm, c.dy, v, dx, dA, dB, wsb)
    for turn in range(4):
        src = other if turn % 2 else Case(counts, 512, 512, 4, 16, mix="tokens", seed=8)
        for name in ("x", "dy", "adapter", "perm", "A", "scale"):
            getattr(c, name).copy_(getattr(src, name))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, v, dx, dA, dB)]
        want_y, want_v = c.forward()
        want = [want_y, want_v, *c.backward(want_v)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a[:c.rows].view(torch.uint8), b[:c.rows].view(torch.uint8)) if a.dim() == 2 else torch.equal(a, b)


@gpu
def test_two_streams_with_workspaces_of_their_own():
    cases = [Case((700, 90), 512, 512, 4, 16, seed=s) for s in (1, 2)]
    want = [c.forward() for c in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cases], []
    for c, s in zip(cases, streams):
        with torch.cuda.stream(s):
            got.append(c.forward())
    torch.cuda.synchronize()
    for (y, v), (y1, v1) in zip(want, got):
        assert torch.equal(y.view(torch.int16), y1.view(torch.int16)) and torch.equal(v, v1)


@gpu
def test_gradients_against_differences():
    """The gradients of sum(dy * y) with respect to an element of A, B and x, from the forward itself: B and x enter linearly, A too, so
    differences of any width are exact but for the rounding of y (fp16, half a step of each of the N * rows terms: bounded by their sum)."""
    c = Case((50, 30), 64, 128, 3, 8, "f16", mix="tokens", seed=2, scale=True)
    y, v = c.forward()
    dx, dA, dB = c.backward(v)
    torch.cuda.synchronize()
    dy = f64(c.dy)[:c.rows]
    a = int(c.host_row[c.host_row >= 0][0])

    def loss():
        y, _ = c.forward()
        y = f64(y)[:c.rows]
        return float((dy * y).sum()), float((np.abs(dy) * np.abs(y)).sum()) * 2.0 ** -11
    for t, grad, at in ((c.A, dA, (a, 0, 2, 5)), (c.B, dB, (a, 0, 9, 3)), (c.x, dx, (4, 7))):
        before = float(t[at])
        t[at] = before + 2.0
        up, e1 = loss()
        t[at] = before - 2.0
        down, e0 = loss()
        width = 4.0
        t[at] = before
        # the rounding errors are independent: their sum stays far below the bound of the sum
        assert abs((up - down) / width - float(grad[at])) <= 0.1 * (e0 + e1) / width + 2.0 ** -9 * abs(float(grad[at])), at
