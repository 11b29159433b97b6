"""moe_adapter_forward and moe_adapter_backward where a full batch runs: more output tiles than compute units, the narrow product's forms for many
rows, and how cut tiles are handed over.  Tolerances as in test_adapters.py."""

import numpy as np
import pytest
import torch

from paper_2304_11414_amd import binding as B
from tests.test_adapters import Case, DT, check_backward, check_forward, close, f64, lib  # noqa: F401  (lib: a fixture of the module)
from tests.test_gpu_edges import HANDOVER_SETTINGS

pytestmark = pytest.mark.gpu

SHAPES = [
    # counts, K, N, adapters, rank, more
    ((4200, 300), 256, 4352, 5, 16, dict()),                    # 17 x 18 tiles of 256; 32 rows a block in the narrow product
    ((4200, 300), 256, 4352, 5, 32, dict(top_k=2)),
    ((2300, 1, 2200), 256, 4360, 40, 24, dict(mix="tokens")),     # a last column tile of 8
    ((200,), 328, 264, 4, 16, dict(gelu=True)),                 # a block per tile, GeLU
    ((600,), 2048, 512, 3, 64, dict(mix="tokens")),               # a cut contraction in the narrow product, ranks up to 64
    ((513, 90), 1024, 1048, 3, 40, dict()),
    ((1000,), 4096, 264, 2, 72, dict()),                        # and above
]


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=[str(i) for i in range(len(SHAPES))])
def test_forward(shape, dt):
    counts, K, N, n_a, rank, more = shape
    c = Case(counts, K, N, n_a, rank, dt, seed=K + N, **more)
    y, v = c.forward()
    check_forward(c, y, v)
    again, _ = c.forward()
    assert torch.equal(y.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=[str(i) for i in range(len(SHAPES))])
def test_backward(shape, dt):
    counts, N, K, n_a, rank, more = shape                       # (dx is the product from N to K)
    c = Case(counts, K, N, n_a, rank, dt, seed=K + N + 1, **{**more, "gelu": False})
    v = torch.randn(c.rows + 5, rank, generator=torch.Generator().manual_seed(rank)).cuda()
    check_backward(c, v, *c.backward(v))


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("K,N", [(2048, 512), (4096, 4096)])
def test_cut_tiles_have_the_same_bits_however_they_are_handed_over(K, N, dt):
    """Partial sums through the shared L2, with device-scope fences, or never waited for and computed by the compute unit that needs them: the
    low-rank part is added once.  fp16: some rows' factors are beyond its range.  Up to 40 k-tiles of 64 (2048 here) tiles that
    are otherwise whole are cut where nobody waits: their sums have another order, so the definition's bounds instead of the bits."""
    counts = (2000, 300) if N < K else (600,)
    c, d = Case(counts, K, N, 5, 24, dt, mix="tokens", seed=K), Case(counts, N, K, 5, 24, dt, mix="tokens", seed=N)
    for case in (c, d):
        case.scale = torch.tensor([1.0, 2.0 ** 17, 0.5, -1.0, 2.0 ** -18], device="cuda")
        case.B[1].mul_(2.0 ** -12)
        case.A[1].mul_(2.0 ** -5)
    v = torch.randn(d.rows + 5, 24, generator=torch.Generator().manual_seed(K)).cuda()
    y, kept = c.forward()
    out = [y[:c.rows], kept[:c.rows], *(t[:d.rows] if t.dim() == 2 else t for t in d.backward(v))]
    check_forward(c, y, kept)
    for option, value, default in HANDOVER_SETTINGS:
        B.moe_set_option(option, value)
        try:
            y, kept = c.forward()
            again = [y[:c.rows], kept[:c.rows], *(t[:d.rows] if t.dim() == 2 else t for t in d.backward(v))]
            torch.cuda.synchronize()
        finally:
            B.moe_set_option(option, default)
        if K <= 40 * 64 and option == B.MOE_OPT_HANDOVER_SPIN_LIMIT:
            check_forward(c, y, kept)
            check_backward(d, v, torch.cat([again[2], torch.full((5, N), 7.0, dtype=DT[dt], device="cuda")]), *again[3:])
            continue
        for name, a, b in zip(("y", "v", "dx", "dA", "dB"), out, again):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), (name, option)


@pytest.mark.parametrize("counts", [(40, 3), (900, 300)])
def test_captured_fp16_calls_replay_with_new_inputs(counts):
    """Scales too: the powers of two of a row's factors follow them."""
    c = Case(counts, 512, 512, 4, 40, "f16", mix="tokens", seed=8)
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
        src = Case(counts, 512, 512, 4, 40, "f16", mix="tokens", seed=8 + turn)
        src.scale[turn % 4] *= 2.0 ** (15 if turn % 2 else -25)
        for name in ("x", "dy", "adapter", "perm", "A", "scale"):
            getattr(c, name).copy_(getattr(src, name))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, v, dx, dA, dB)]
        want_y, want_v = c.forward()
        want = [want_y, want_v, *c.backward(want_v)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a[:c.rows].view(torch.uint8), b[:c.rows].view(torch.uint8)) if a.dim() == 2 else torch.equal(a.view(torch.int32), b.view(torch.int32))


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("counts", [(20,), (400,)])
def test_the_most_adapters(counts, dt):
    """65536 of them: the last one's number is all 16 bits of a row's word, beside rows without any and, in fp16, rows with a power of two."""
    c = Case(counts, 16, 24, 65536, 8, dt, perm=False, seed=counts[0])
    who = torch.tensor([65535, -1, 0, 65534])[torch.arange(counts[0]) % 4]
    c.adapter.copy_(who.to(torch.int32))
    c.host_row = who.numpy()
    c.scale[65534] = 2.0 ** 17
    c.B[65534].mul_(2.0 ** -12)
    c.A[65534].mul_(2.0 ** -12)
    y, v = c.forward()
    check_forward(c, y, v)
    check_backward(c, v, *c.backward(v))
