"""The AdamW step over many tensors (moe_adamw_plan, moe_adamw_step): refusals and the plan on the CPU; on the GPU
against the definition in float64.

Tolerances.  A step of float32 operations, each off by at most 2^-24 of its result: m and v are sums of two products
(three and four roundings, with the gradient's scaling one more), so at most 6 * 2^-24 of the sum of the terms' magnitudes; p is a product minus a
quotient whose numerator and denominator have had at most 16 roundings between them, its own 2 and the factors' 1 each: 24 * 2^-24 of
|p| + |update|."""

import ctypes

import numpy as np
import pytest
import torch  # before the library is loaded: both then share one HIP runtime

from paper_2304_11414_amd import binding as B
from paper_2304_11414_amd import build as build_mod

gpu = pytest.mark.gpu
EPS24 = 2.0 ** -24
LOWEST = -100


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    if not os.path.exists(B.LIB_PATH):
        build_mod.build_library()
    return B.load_library()


# ---- CPU: what is refused, and the plan --------------------------------------------------------------

def table(*sizes, bits=32, **over):
    t = (B.MoeAdamwTensor * max(len(sizes), 1))()
    at = 0x100000
    for e, n in zip(t, sizes):
        for name in ("p", "g", "m", "v", "m_power", "v_power", "half"):
            setattr(e, name, at)
            at += (max(n, 1) * 4 + 15) // 16 * 16
        e.n, e.half_dtype, e.lr_scale = n, B.MOE_BF16, 1.0
        for k, v in over.items():
            setattr(e, k, v)
    return t


def plan(cfg, t, n, size=None):
    lib = B.load_library()
    want = lib.moe_adamw_plan_bytes(ctypes.byref(cfg), t, n)
    buf = ctypes.create_string_buffer(max(want, 16))
    chunks = ctypes.c_int64(-1)
    return lib.moe_adamw_plan(ctypes.byref(cfg), t, n, buf, want if size is None else size, ctypes.byref(chunks)), chunks.value


@pytest.mark.parametrize("kw,status", [(dict(beta1=1.0), -2), (dict(beta1=-0.1), -2), (dict(beta2=1.0), -2), (dict(beta2=float("nan")), -2),
                                       (dict(eps=0.0), -2), (dict(eps=1e-60), -2), (dict(eps=float("inf")), -2), (dict(moment_bits=16), -3)])
def test_configurations_refused(kw, status):
    cfg = B.make_adamw_config(**kw)
    assert plan(cfg, table(10), 1, size=1 << 20)[0] == status
    p = ctypes.c_void_p(0x1000)
    assert B.load_library().moe_adamw_step(ctypes.byref(cfg), p, 1, 1, p, None) == status


@pytest.mark.parametrize("bits", [32, 8])
def test_plan_counts_chunks_and_allows_empty_tensors(bits):
    cfg = B.make_adamw_config(moment_bits=bits)
    sizes = (0, 1, 4096, 4097, 0, 100_000)
    assert plan(cfg, table(*sizes), len(sizes)) == (0, sum(-(-n // 4096) for n in sizes))
    assert plan(cfg, table(), 0) == (0, 0)
    empty = (B.MoeAdamwTensor * 1)()          # n == 0: the pointers are not looked at
    assert plan(cfg, empty, 1) == (0, 0)


def test_tensors_refused():
    c32, c8 = B.make_adamw_config(), B.make_adamw_config(moment_bits=8)
    for name in ("p", "g", "m", "v"):
        assert plan(c32, table(10, **{name: None}), 1)[0] == -1
    assert plan(c8, table(10, v_power=None), 1)[0] == -1
    assert plan(c32, table(10, v_power=None, m_power=None, half=None), 1)[0] == 0
    for name in ("p", "g", "m", "v", "half", "m_power"):
        t = table(10)
        setattr(t[0], name, getattr(t[0], name) + 4)
        assert plan(c8, t, 1)[0] == -4
    assert plan(c32, table(10, half_dtype=B.MOE_F32), 1)[0] == -3
    assert plan(c32, table(10, lr_scale=float("nan")), 1)[0] == -2
    assert plan(c32, table(10, weight_decay=float("inf")), 1)[0] == -2
    assert plan(c32, table(-1), 1, size=1 << 20)[0] == -2
    assert plan(c32, table(1 << 62), 1, size=1 << 20)[0] == -2
    assert plan(c32, table(10), -1, size=1 << 20)[0] == -2
    assert plan(c32, table(10), 1, size=15)[0] == -5
    assert B.load_library().moe_adamw_plan(ctypes.byref(c32), table(10), 1, None, 1 << 20, ctypes.byref(ctypes.c_int64())) == -1


def test_memory_named_twice_is_refused():
    cfg = B.make_adamw_config()
    t = table(1000, 1000)
    t[1].g = t[0].g                            # two tensors may read the same gradient
    assert plan(cfg, t, 2)[0] == 0
    t = table(1000, 1000)
    t[1].p = t[0].p
    assert plan(cfg, t, 2)[0] == -7
    t = table(1000, 1000)
    t[1].v = t[0].m + 4 * 1000 - 16            # the last four elements
    assert plan(cfg, t, 2)[0] == -7
    t = table(1000)
    t[0].m = t[0].v
    assert plan(cfg, t, 1)[0] == -7
    t = table(1000, 1000)
    t[1].g = t[0].half                         # read by one, written by another
    assert plan(cfg, t, 2)[0] == -7
    assert B.load_library().moe_status_string(-7) != B.load_library().moe_status_string(-99)


def test_step_arguments_refused():
    lib, cfg, p = B.load_library(), B.make_adamw_config(), ctypes.c_void_p(0x1000)
    c = ctypes.byref(cfg)
    assert lib.moe_adamw_step(None, p, 1, 1, p, None) == -1
    assert lib.moe_adamw_step(c, None, 1, 1, p, None) == -1
    assert lib.moe_adamw_step(c, p, 1, 1, None, None) == -1
    assert lib.moe_adamw_step(c, ctypes.c_void_p(0x1008), 1, 1, p, None) == -4
    assert lib.moe_adamw_step(c, p, 1, 1, ctypes.c_void_p(0x1004), None) == -4
    assert lib.moe_adamw_step(c, p, -1, 1, p, None) == -2
    assert lib.moe_adamw_step(c, p, 0, 1, p, None) == -2
    assert lib.moe_adamw_step(c, p, 1, 1 << 31, p, None) == -2
    assert lib.moe_adamw_step(c, p, 0, 0, p, None) == 0      # nothing to do


# ---- GPU --------------------------------------------------------------------------------------------

def e4m3():
    """The values of the codes 0 .. 126."""
    c = np.arange(127)
    return np.where(c < 8, c * 2.0 ** -9, (8 + c % 8) * 2.0 ** (c // 8 - 10.0))


def widen(codes, power):
    v = np.concatenate([e4m3(), [np.nan]])[codes & 127] * np.where(codes & 128, -1.0, 1.0)
    return v * np.repeat(np.where(power == 255, np.nan, 2.0 ** (power.astype(np.float64) - 127)), 32)[:len(codes)]


def phase(n, step, half):
    i = np.arange(n, dtype=np.uint64) % 512
    w = (i * 0x85EBCA6B + np.uint64(step * 0x9E3779B9 % 2 ** 32)) % 2 ** 32
    return ((w >> np.uint64(12)).astype(np.int64) ^ (half << 19)) / 2.0 ** 20


def check_codes(got, power, value, ph, positive):
    """Codes and powers against the definition; where a value is within float32's rounding of a border either side is right."""
    a, grid = np.abs(value), np.append(e4m3(), np.inf)
    for b in range(len(power)):
        s = slice(32 * b, 32 * b + 32)
        top = a[s].max()
        e = LOWEST
        if top > 0:
            e = max(LOWEST, int(np.floor(np.log2(top))) - 8)
            while top > 448.0 * 2.0 ** e * (1 + 1e-6):
                e += 1
        near = top > 0 and abs(top / (448.0 * 2.0 ** (int(power[b]) - 127)) - 1) < 1e-6
        assert int(power[b]) == e + 127 or near, (b, int(power[b]), e + 127)
        y = a[s] / 2.0 ** (int(power[b]) - 127.0)
        low = np.searchsorted(grid, y, side="right") - 1
        step = np.where(low < 8, 2.0 ** -9, 2.0 ** (low // 8 - 10.0))
        t = (y - grid[low]) / step + ph[s]
        code = np.minimum(low + (t >= 1), 126)
        if positive:
            code = np.where((value[s] > 0) & (code == 0), 1, code)
        mine = got[s].astype(int) & 127
        border = (np.abs(t - 1) < 3e-5) | (np.abs(t - np.round(t)) < 3e-5) & (np.abs(mine - code) <= 1)
        assert np.all((mine == code) | border), b
        assert np.all(((got[s] & 128) != 0) == ((value[s] < 0) & (not positive)))


def reference(p, g, m, v, step, lr, wd, gs, b1=0.9, b2=0.999, eps=1e-8):
    b1, b2, eps = float(b1), float(b2), float(np.float32(eps))
    g = g * gs
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    u = lr / (1 - b1 ** step) * m / (np.sqrt(v) / np.sqrt(1 - b2 ** step) + eps)
    return p * (1 - lr * wd) - u, m, v, np.abs(u)


def make(sizes, bits, half, seed, guard=64):
    """Tensors inside larger buffers (16-byte aligned, whose other elements have to stay)."""
    gen = torch.Generator().manual_seed(seed)
    made = []
    for n in sizes:
        def buf(fill, dtype=torch.float32, count=n):
            whole = torch.full((count + 2 * guard,), 7, dtype=dtype)
            whole[guard:guard + count] = fill
            whole = whole.cuda()
            return whole[guard:guard + count], whole
        t = {}
        t["p"] = buf(torch.randn(n, generator=gen) * 0.02)
        t["g"] = buf(torch.randn(n, generator=gen) * torch.exp(2.0 * torch.randn(n, generator=gen)))
        if bits == 32:
            t["m"], t["v"] = buf(torch.randn(n, generator=gen) * 0.1), buf(torch.rand(n, generator=gen))
        else:
            t["m"], t["v"] = buf(0, torch.uint8), buf(0, torch.uint8)
            k = (n + 31) // 32
            t["m_power"], t["v_power"] = buf(0, torch.uint8, k), buf(0, torch.uint8, k)
        if half is not None:
            t["half"] = buf(0, getattr(torch, half))
        made.append(t)
    return made


def views(made, **more):
    return [dict({k: v[0] for k, v in t.items()}, **{k: f(i) for k, f in more.items()}) for i, t in enumerate(made)]


def host(made, name):
    return [t[name][0].cpu().numpy().astype(np.float64 if name not in ("m", "v", "m_power", "v_power") or t[name][0].dtype.is_floating_point
                                            else np.uint8) for t in made]


@gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("half", [None, "bfloat16", "float16"])
@pytest.mark.parametrize("sizes", [(1,), (3, 0, 31, 32, 33), (4095, 4096, 4097), (7, 50_001, 8, 12_289)])
def test_three_steps_against_float64(bits, half, sizes):
    made = make(sizes, bits, half, seed=len(sizes))
    cfg = B.make_adamw_config(0.9, 0.999, 1e-8, bits)
    scale, decay = lambda i: 1.0 + i, lambda i: 0.1 * i
    pl = B.moe_adamw_plan(cfg, views(made, lr_scale=scale, weight_decay=decay))
    lr, gs = float(np.float32(1e-3)), 0.25
    for step in (1, 2, 3):
        before = {k: host(made, k) for k in made[0] if k not in ("half",)}
        B.moe_adamw_step(cfg, pl, B.moe_adamw_scalars(step, lr, gs))
        torch.cuda.synchronize()
        after = {k: host(made, k) for k in made[0] if k not in ("half",)}
        for i, n in enumerate(sizes):
            if n == 0:
                continue
            m, v = before["m"][i], before["v"][i]
            if bits == 8:
                m, v = widen(m, before["m_power"][i]), widen(v, before["v_power"][i]) ** 2
            wd = float(np.float32(decay(i)))
            p, m1, v1, u = reference(before["p"][i], before["g"][i], m, v, step, lr * scale(i), wd, gs)
            g = before["g"][i] * gs
            assert np.all(np.abs(after["p"][i] - p) <= 24 * EPS24 * (np.abs(before["p"][i]) + u)), (i, step)
            if bits == 32:
                assert np.all(np.abs(after["m"][i] - m1) <= 6 * EPS24 * (0.9 * np.abs(m) + 0.1 * np.abs(g)))
                assert np.all(np.abs(after["v"][i] - v1) <= 6 * EPS24 * v1)
            else:
                check_codes(after["m"][i], after["m_power"][i], m1, phase(n, step, 0), False)
                check_codes(after["v"][i], after["v_power"][i], np.sqrt(v1), phase(n, step, 1), True)
            if half is not None:   # the rounding of what is stored
                assert torch.equal(made[i]["half"][0], made[i]["p"][0].to(made[i]["half"][0].dtype))
    for t in made:                 # what lies beside the tensors
        for name, (inner, whole) in t.items():
            assert torch.all(whole[:64] == 7) and torch.all(whole[64 + inner.numel():] == 7), name


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_skip_writes_nothing_and_steps_below_one_are_one(bits):
    cfg = B.make_adamw_config(moment_bits=bits)
    a, b = make((5000,), bits, "bfloat16", 3), make((5000,), bits, "bfloat16", 3)
    pa, pb = B.moe_adamw_plan(cfg, views(a)), B.moe_adamw_plan(cfg, views(b))
    B.moe_adamw_step(cfg, pa, B.moe_adamw_scalars(1, 1e-3, skip=True))
    for name, (_, whole) in a[0].items():
        assert torch.equal(whole, b[0][name][1]), name
    B.moe_adamw_step(cfg, pa, B.moe_adamw_scalars(-3, 1e-3))
    B.moe_adamw_step(cfg, pb, B.moe_adamw_scalars(1, 1e-3))
    for name, (_, whole) in a[0].items():
        assert torch.equal(whole, b[0][name][1]), name


@gpu
def test_8bit_roots_follow_a_slow_change_in_the_mean():
    """A moment that nearest rounding would never move: v decays from r = 1 by 0.05 % a step, the codes next to 1 are 6 % apart.  The mean of the
    4096 elements (512 phases) follows b2^(t / 2) within half a code step, and no element is further off than one step per
    turn of its phase: checked as 10 %."""
    n = 4096
    t = dict(p=torch.zeros(n, device="cuda"), g=torch.zeros(n, device="cuda"), m=torch.zeros(n, dtype=torch.uint8, device="cuda"),
             v=torch.full((n,), 0x78, dtype=torch.uint8, device="cuda"),        # 256
             m_power=torch.zeros(n // 32, dtype=torch.uint8, device="cuda"), v_power=torch.full((n // 32,), 119, dtype=torch.uint8, device="cuda"))
    cfg = B.make_adamw_config(moment_bits=8)
    pl = B.moe_adamw_plan(cfg, [t])
    values = B.moe_adamw_scalars(1, 1e-3)
    for step in range(1, 1201):
        B.moe_adamw_step(cfg, pl, B.moe_adamw_scalars(step, 1e-3, out=values))
    r = widen(t["v"].cpu().numpy(), t["v_power"].cpu().numpy())
    want = 0.999 ** 600
    assert abs(r.mean() / want - 1) < 0.0625, (r.mean(), want)
    assert r.max() < want * 1.25 and r.min() > want * 0.8


@gpu
def test_infinite_gradients_reach_their_block_alone():
    for bits in (32, 8):
        made = make((100, 200), bits, "float16", 9)
        made[0]["g"][0][40] = float("inf")
        made[1]["g"][0][199] = float("nan")
        cfg = B.make_adamw_config(moment_bits=bits)
        B.moe_adamw_step(cfg, B.moe_adamw_plan(cfg, views(made)), B.moe_adamw_scalars(1, 1e-3))
        for t, at in zip(made, (40, 199)):
            p = t["p"][0].cpu().numpy()
            assert list(np.flatnonzero(~np.isfinite(p))) == [at]
            if bits == 8:
                for k in ("m", "v"):
                    power = t[k + "_power"][0].cpu().numpy()
                    assert list(np.flatnonzero(power == 255)) == [at // 32]
                    bad = np.flatnonzero(t[k][0].cpu().numpy() == 127)
                    assert set(range(at // 32 * 32, min(at // 32 * 32 + 32, len(p)))) <= set(bad)


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_captured_step_reads_its_values_at_replay_and_other_streams_agree(bits):
    cfg = B.make_adamw_config(moment_bits=bits)
    a, b = make((3000, 17), bits, "bfloat16", 5), make((3000, 17), bits, "bfloat16", 5)
    pa, pb = B.moe_adamw_plan(cfg, views(a)), B.moe_adamw_plan(cfg, views(b))
    values = B.moe_adamw_scalars(1, 1e-3)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.moe_adamw_step(cfg, pa, values)
    side = torch.cuda.Stream()
    for step in range(1, 6):
        B.moe_adamw_scalars(step, 1e-3 / step, out=values)
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            B.moe_adamw_step(cfg, pb, B.moe_adamw_scalars(step, 1e-3 / step))
        torch.cuda.synchronize()
        for s, t in zip(a, b):
            for name in s:
                assert torch.equal(s[name][1], t[name][1]), (step, name)


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_a_plan_of_other_moments_writes_nothing(bits):
    a, b = make((5000, 33), bits, "bfloat16", 3), make((5000, 33), bits, "bfloat16", 3)
    plan = B.moe_adamw_plan(B.make_adamw_config(moment_bits=bits), views(a))
    B.moe_adamw_step(B.make_adamw_config(moment_bits=40 - bits), plan, B.moe_adamw_scalars(1, 1e-3))
    torch.cuda.synchronize()
    for s, t in zip(a, b):
        for name, (_, whole) in s.items():
            assert torch.equal(whole, t[name][1]), name
