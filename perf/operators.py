"""Performance cases of what stands beside the MoE layer in fine-tuning and in serving fine-tuned models: low-rank
adapters of many requests beside the experts' projections, with their gradients, and the AdamW step over many tensors.

A case names an `op` and its sizes:
  forward    moe_adapter_forward: serving, and the forward of a fine-tuning step
  backward   moe_adapter_backward: the adapters' gradients and the data gradient, expert weights frozen
  adamw      moe_adamw_step over the tensors of a plan, moments in 32 or in 8 bits

Adapter cases.  `T` tokens, `k` picks each, are packed by expert as the dispatch leaves them (T * k rows).  `mix`: "requests":
the tokens are the prompts of `requests` requests one after another, each with one of `adapters` adapters or, one in ten,
none; "tokens": every token is another request's.
AdamW cases.  `tensors` tensors of `least` to `most` elements (spread over the logarithm, fixed by the case) lie in one
buffer per kind (weights, gradients, moments), each from a multiple of 512 elements on.
"""

import math
import random

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
_GAP = 512     # elements: where a tensor may begin in a buffer
_BLOCK = 32    # elements that share the power of two of an 8-bit moment
_LOWEST = -100  # the lowest such power


def _adapted(name, op, T, K, N, E, adapters, rank, k=1, mix="requests", requests=8, dt="bf16", gelu=False):
    c = dict(op=op, T=T, K=K, N=N, E=E, k=k, adapters=adapters, rank=rank, mix=mix, requests=requests, dt=dt, gelu=gelu)
    if name:
        c["name"] = name
    return c


def _adamw(name, bits, tensors, least, most, step, half="bf16", shuffle=1):
    c = dict(op="adamw", bits=bits, tensors=tensors, least=least, most=most, step=step, half=half, shuffle=shuffle)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # Token generation for a single request through the dense projection (one expert), GeLU behind it: latency.
        _adapted("forward_1_token", "forward", 1, 2048, 8192, 1, 8, 16, mix="tokens", gelu=True),
        # Token generation for 48 requests, each with an adapter of its own draw, top-2 of 8 experts: every expert's
        # weights and most adapters are read for a handful of rows.
        _adapted("forward_48_requests", "forward", 48, 2048, 8192, 8, 32, 16, k=2, mix="tokens", gelu=True),
        # A few prompts of odd length through sizes that are multiples of 8 only, fp16, a rank that is no power of two.
        _adapted("forward_odd_f16", "forward", 1177, 1000, 4000, 4, 5, 24, requests=6, dt="f16"),
        # A full batch of prompts of 24 requests through the up projection of the GPT-style layer.
        _adapted("forward_prompts", "forward", 8192, 2048, 8192, 8, 16, 32, requests=24, gelu=True),
        # A small fine-tuning batch, fp16 (the precision the paper trains in), the smallest rank.
        _adapted("backward_small_f16", "backward", 301, 1024, 4096, 1, 3, 8, requests=4, dt="f16"),
        # The down projection of the GPT-style layer, 16 adapters trained at once.
        _adapted("backward_down", "backward", 8192, 8192, 2048, 8, 16, 16, requests=24),
        # One dense projection with few adapters of a large rank.
        _adapted("backward_dense", "backward", 4096, 2048, 8192, 1, 4, 64, requests=8),
        # The adapters of one layer: many small tensors of odd sizes.
        _adamw("adamw_adapters", 32, 96, 1000, 300_000, 10),
        # The expert weights of a layer: two tensors that only the memory bounds.
        _adamw("adamw_experts", 32, 2, 60_000_000, 67_108_864, 1000),
        # The same with the moments in 8 bits.
        _adamw("adamw8_adapters", 8, 96, 1000, 300_000, 10, half="f16"),
        _adamw("adamw8_experts", 8, 2, 60_000_000, 67_108_864, 1000),
    ]


_MOST_FLOPS = 2.0 * 8192 * 2048 * 8192      # of a drawn projection
_MOST_WEIGHTS = 8 * 2048 * 8192             # its expert matrices
_MOST_ADAPTERS = 16 * 8 * 32 * (2048 + 8192)


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.35:
        least = _log_int(rng, 1, 10_000)
        return _adamw(None, rng.choice([32, 8]), _log_int(rng, 1, 200), least, _log_int(rng, least, 400_000), _log_int(rng, 1, 20_000),
                      half=rng.choice(["bf16", "f16"]), shuffle=rng.randrange(1 << 20))
    while True:
        unit = rng.choice([8, 8, 64, 64, 64])
        K, N = (unit * max(1, _log_int(rng, 64, 8192) // unit) for _ in range(2))
        T, k, E = _log_int(rng, 1, 8192), rng.choice([1, 1, 2]), rng.choice([1, 1, 2, 4, 7, 8])
        k = min(k, E)
        adapters, rank = _log_int(rng, 1, 64), rng.choice([8, 16, 16, 24, 32, 64])
        if 2.0 * T * k * K * N <= _MOST_FLOPS and E * K * N <= _MOST_WEIGHTS and E * adapters * rank * (K + N) <= _MOST_ADAPTERS:
            op = rng.choice(["forward", "forward", "backward"])
            return _adapted(None, op, T, K, N, E, adapters, rank, k=k, mix="tokens" if T <= 128 and rng.random() < 0.7 else "requests",
                            requests=_log_int(rng, 1, 48), dt=rng.choice(["bf16", "bf16", "f16"]), gelu=op == "forward" and rng.random() < 0.4)


# ---- inputs ---------------------------------------------------------------------------------------

def _sizes(case):
    rng = random.Random(case["shuffle"])
    return [_log_int(rng, case["least"], case["most"]) for _ in range(case["tensors"])]


def _prepare_adamw(case, gen):
    sizes, starts, end = _sizes(case), [], 0
    for n in sizes:
        starts.append(end)
        end += -(-n // _GAP) * _GAP

    def filled(make):   # a buffer with `make`'s values where the tensors are and zeros between them
        a = make(torch.empty(end, device="cuda"))
        for s, n in zip(starts, sizes):
            a[s + n:s + -(-n // _GAP) * _GAP] = 0
        return a

    st = dict(case=case, sizes=sizes, starts=starts, lr=1e-4, weight_decay=0.01, beta1=0.9, beta2=0.999, eps=1e-8, step=case["step"],
              grad_scale=1.0 / 128)
    st["p"] = filled(lambda a: a.normal_(0.0, 0.02, generator=gen))
    st["g"] = filled(lambda a: a.normal_(0.0, 0.1, generator=gen))       # of a loss scaled by 128
    st["half"] = st["p"].to(_DTYPES[case["half"]])
    if case["bits"] == 32:
        st["m"] = filled(lambda a: a.normal_(0.0, 1e-4, generator=gen))
        st["v"] = filled(lambda a: a.normal_(0.0, 1e-3, generator=gen).square_())
    else:
        for name, low in (("m", 108), ("r", 110)):
            codes = filled(lambda a: a.normal_(0.0, 70.0, generator=gen).clamp_(-440.0, 440.0))
            codes = (codes.abs_() if name == "r" else codes).to(torch.float8_e4m3fn).view(torch.uint8)
            used = codes.view(-1, _BLOCK).ne(0).any(1)
            power = torch.randint(low - 3, low, (end // _BLOCK,), device="cuda", generator=gen, dtype=torch.uint8)
            st[name], st[name + "_power"] = codes, torch.where(used, power, torch.full_like(power, 127 + _LOWEST))
    if own:
        from paper_2304_11414_amd import binding as B
        st["config"] = B.make_adamw_config(st["beta1"], st["beta2"], st["eps"], case["bits"])
        views = [dict(p=st["p"][s:s + n], g=st["g"][s:s + n], half=st["half"][s:s + n], weight_decay=st["weight_decay"],
                      **(dict(m=st["m"][s:s + n], v=st["v"][s:s + n]) if case["bits"] == 32 else
                         dict(m=st["m"][s:s + n], v=st["r"][s:s + n], m_power=st["m_power"][s // _BLOCK:(s + n + _BLOCK - 1) // _BLOCK],
                              v_power=st["r_power"][s // _BLOCK:(s + n + _BLOCK - 1) // _BLOCK]))) for s, n in zip(starts, sizes)]
        st["plan"] = B.moe_adamw_plan(st["config"], views)
        st["scalars"] = B.moe_adamw_scalars(st["step"], st["lr"], st["grad_scale"])
    return st


def _prepare_adapted(case, gen):
    T, K, N, E, k, rank, n_a = (case[x] for x in ("T", "K", "N", "E", "k", "rank", "adapters"))
    dt, rows = _DTYPES[case["dt"]], T * k

    def normal(*shape, std=1.0):
        a = torch.empty(shape, device="cuda", dtype=dt)
        for part in a.view(shape[0], -1):
            part.normal_(0.0, std, generator=gen)
        return a

    # k different experts for every token; packed by expert, in token order inside it
    picks = torch.rand(T, E, device="cuda", generator=gen).argsort(1)[:, :k].reshape(-1)
    perm = picks.argsort(stable=True).to(torch.int32)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = torch.bincount(picks, minlength=E).cumsum(0)
    if case["mix"] == "tokens":
        adapter = torch.randint(0, n_a, (T,), device="cuda", generator=gen)
    else:
        cuts = torch.randint(0, T + 1, (case["requests"],), device="cuda", generator=gen).sort().values
        request = torch.bucketize(torch.arange(T, device="cuda"), cuts, right=True)
        mine = torch.randint(0, n_a, (case["requests"] + 1,), device="cuda", generator=gen)
        none = torch.rand(case["requests"] + 1, device="cuda", generator=gen) < 0.1
        adapter = torch.where(none, -1, mine)[request]
    st = dict(case=case, perm=perm, offsets=offsets, bounds=offsets.tolist(), adapter=adapter.to(torch.int32),
              x=normal(rows, K), W=normal(E, N, K, std=K ** -0.5), A=normal(n_a, E, rank, K, std=K ** -0.5), B=normal(n_a, E, N, rank, std=rank ** -0.5),
              scale=torch.empty(n_a, device="cuda").uniform_(0.5, 2.0, generator=gen),
              v=torch.empty(rows, rank, device="cuda"))
    if case["op"] == "backward":
        st["dy"] = normal(rows, N)
        # what the forward kept
        row = adapter[perm.long() // k]
        for e in range(E):
            lo, hi = st["bounds"][e], st["bounds"][e + 1]
            wide = st["x"][lo:hi].float() @ st["A"][:, e].reshape(n_a * rank, K).float().t()
            st["v"][lo:hi] = _narrow(wide, row[lo:hi], n_a)
        st.update(dx=torch.empty(rows, K, device="cuda", dtype=dt), dA=torch.empty(n_a, E, rank, K, device="cuda"),
                  dB=torch.empty(n_a, E, N, rank, device="cuda"))
    else:
        st["y"] = torch.empty(rows, N, device="cuda", dtype=dt)
    if own:
        from paper_2304_11414_amd import binding as B
        cfg = B.make_adapter_config(rows, K, N, E, n_a, rank, top_k=k, dtype=case["dt"], gelu=case["gelu"])
        size = (B.moe_adapter_backward_workspace_bytes if case["op"] == "backward" else B.moe_adapter_workspace_bytes)(cfg)
        st.update(config=cfg, workspace=torch.empty(size, dtype=torch.uint8, device="cuda"))
    return st


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return _prepare_adamw(case, gen) if case["op"] == "adamw" else _prepare_adapted(case, gen)


# ---- one pass ---------------------------------------------------------------------------------------

def _gelu(u):
    return 0.5 * u * (1.0 + torch.tanh(0.7978845608028654 * (u + 0.044715 * u * u * u)))


def _spread(values, row, n_a):
    """[rows, rank] -> [rows, n_a * rank]: each row's values in its adapter's columns, zeros elsewhere."""
    wide = values.new_zeros(values.shape[0], n_a, values.shape[1])
    at = torch.arange(values.shape[0], device=values.device)
    wide[at, row.clamp(min=0)] = torch.where(row[:, None] >= 0, values, 0.0)
    return wide.flatten(1)


def _narrow(wide, row, n_a):
    """The inverse: each row's own columns; zeros for a row without an adapter."""
    at = torch.arange(wide.shape[0], device=wide.device)
    return torch.where(row[:, None] >= 0, wide.unflatten(1, (n_a, wide.shape[1] // n_a))[at, row.clamp(min=0)], 0.0)


def _plain_forward(st):
    c = st["case"]
    n_a, row = c["adapters"], st["adapter"][st["perm"].long() // c["k"]].long()
    scale = st["scale"][row.clamp(min=0)][:, None]
    for e in range(c["E"]):
        rows = slice(st["bounds"][e], st["bounds"][e + 1])
        x, r = st["x"][rows].float(), row[rows]
        v = _narrow(x @ st["A"][:, e].flatten(0, 1).float().t(), r, n_a)
        b = st["B"][:, e].float().transpose(1, 2).reshape(-1, c["N"])
        u = x @ st["W"][e].float().t() + _spread(v * scale[rows], r, n_a) @ b
        st["y"][rows] = (_gelu(u) if c["gelu"] else u).to(st["y"].dtype)
        st["v"][rows] = v
    return {"y": st["y"], "v": st["v"]}


def _plain_backward(st):
    c = st["case"]
    n_a, rank, row = c["adapters"], c["rank"], st["adapter"][st["perm"].long() // c["k"]].long()
    scale = st["scale"][row.clamp(min=0)][:, None]
    for e in range(c["E"]):
        rows = slice(st["bounds"][e], st["bounds"][e + 1])
        x, dy, r = st["x"][rows].float(), st["dy"][rows].float(), row[rows]
        b = st["B"][:, e].float().transpose(1, 2).reshape(-1, c["N"])
        t = _spread(_narrow(dy @ b.t(), r, n_a) * scale[rows], r, n_a)
        st["dx"][rows] = (dy @ st["W"][e].float() + t @ st["A"][:, e].flatten(0, 1).float()).to(st["dx"].dtype)
        st["dA"][:, e] = (t.t() @ x).view(n_a, rank, c["K"])
        sv = _spread(st["v"][rows] * scale[rows], r, n_a)
        st["dB"][:, e] = (sv.t() @ dy).view(n_a, rank, c["N"]).transpose(1, 2)
    return {"dx": st["dx"], "dA": st["dA"], "dB": st["dB"]}


def _widen(codes, power):
    """The 32-bit values of an 8-bit moment."""
    return (codes.view(torch.float8_e4m3fn).float().view(-1, _BLOCK) * torch.exp2(power.float() - 127.0)[:, None]).flatten()


def _pack(value, phase, positive):
    """A 32-bit moment in 8 bits: the codes, and the power of two of each block.  Rounded down or up by whether the
    part cut off and the element's phase (20 bits) add up to a whole step."""
    a = value.abs().view(-1, _BLOCK)
    f, e = torch.frexp(a.amax(1))                           # the block's largest: f * 2^e, 0.5 <= f < 1
    e = torch.where(f > 0, e - 9 + (f > 0.875).int(), _LOWEST).clamp(min=_LOWEST)  # at most 448 after division by 2^e
    y = (a * torch.exp2(-e.float())[:, None]).flatten()
    normal = ((y.view(torch.int32) + phase) >> 20) - 960    # the sign, exponent and 3 bits of a normal code
    small = ((y * 536870912.0).to(torch.int32) + phase) >> 20  # steps of 2^-9
    code = torch.where(y >= 0.015625, normal, small).clamp(max=126)
    code = torch.where((value > 0) & (code == 0), 1, code) if positive else code + 128 * (value < 0)
    return code.to(torch.uint8), (e + 127).to(torch.uint8)


def _plain_adamw(st):
    g = st["g"] * st["grad_scale"]
    b1, b2, t = st["beta1"], st["beta2"], st["step"]
    if st["case"]["bits"] == 32:
        m = st["m"].mul_(b1).add_(g * (1.0 - b1))
        v = st["v"].mul_(b2).add_(g * g * (1.0 - b2))
        root = v.sqrt()
    else:
        m = b1 * _widen(st["m"], st["m_power"]) + (1.0 - b1) * g
        old = _widen(st["r"], st["r_power"])
        root = (b2 * (old * old) + (1.0 - b2) * (g * g)).sqrt()
    denominator = root * (1.0 - b2 ** t) ** -0.5 + st["eps"]
    st["p"].mul_(1.0 - st["lr"] * st["weight_decay"]).sub_(st["lr"] / (1.0 - b1 ** t) * m / denominator)
    st["half"].copy_(st["p"])
    if st["case"]["bits"] == 32:
        return {"p": st["p"], "half": st["half"], "m": m, "v": v}
    at = torch.arange(_GAP, device=g.device)
    phase = ((at * 0x85EBCA6B + t * 0x9E3779B9) % 2 ** 32 >> 12).to(torch.int32)
    phase = phase.repeat(g.numel() // _GAP)
    st["m"], st["m_power"] = _pack(m, phase, False)
    st["r"], st["r_power"] = _pack(root, phase ^ 0x80000, True)
    return _adamw8_values(st)


def _adamw8_values(st):
    eight, power = torch.float8_e4m3fn, torch.float8_e8m0fnu
    return {"p": st["p"], "half": st["half"], "m": st["m"].view(eight), "m_power": st["m_power"].view(power), "r": st["r"].view(eight),
            "r_power": st["r_power"].view(power)}


def run(st):
    op = st["case"]["op"]
    if not own:
        return {"forward": _plain_forward, "backward": _plain_backward, "adamw": _plain_adamw}[op](st)
    from paper_2304_11414_amd import binding as B
    if op == "forward":
        B.moe_adapter_forward(st["config"], st["x"], st["offsets"], st["W"], st["A"], st["B"], st["scale"], st["adapter"], st["perm"],
                              st["y"], st["v"], st["workspace"])
        return {"y": st["y"], "v": st["v"]}
    if op == "backward":
        B.moe_adapter_backward(st["config"], st["x"], st["offsets"], st["W"], st["A"], st["B"], st["scale"], st["adapter"], st["perm"],
                               st["dy"], st["v"], st["dx"], st["dA"], st["dB"], st["workspace"])
        return {"dx": st["dx"], "dA": st["dA"], "dB": st["dB"]}
    B.moe_adamw_step(st["config"], st["plan"], st["scalars"])
    return {"p": st["p"], "half": st["half"], "m": st["m"], "v": st["v"]} if st["case"]["bits"] == 32 else _adamw8_values(st)


def work(case):
    if case["op"] == "adamw":
        n = sum(_sizes(case))
        return {"bytes": n * (30 if case["bits"] == 32 else 18 + 4 / _BLOCK), "flops": 16 * n}
    rows, K, N, rank = case["T"] * case["k"], case["K"], case["N"], case["rank"]
    pairs = case["E"] * case["adapters"]
    experts, used = min(case["E"], rows), min(pairs, rows)
    read = rows * (K + N) * 2 + rows * rank * 4 + experts * K * N * 2 + used * rank * (K + N) * 2
    if case["op"] == "forward":
        return {"bytes": read, "flops": 2.0 * rows * (K * N + rank * (K + N))}
    return {"bytes": read + rows * K * 2 + pairs * rank * (K + N) * 4, "flops": 2.0 * rows * (K * N + 2 * rank * (K + N))}


# ---- the definition in 64 bits ------------------------------------------------------------------------

def _exact_adapted(case, st):
    d = torch.float64
    token = torch.div(st["perm"].long(), case["k"], rounding_mode="floor")
    whose = st["adapter"].long()[token]
    x, rows = st["x"].to(d), case["T"] * case["k"]
    v = torch.zeros(rows, case["rank"], dtype=d, device="cuda")
    forward = case["op"] == "forward"
    out = torch.zeros(rows, case["N"] if forward else case["K"], dtype=d, device="cuda")
    if not forward:
        dy, dA, dB = st["dy"].to(d), torch.zeros_like(st["dA"], dtype=d), torch.zeros_like(st["dB"], dtype=d)
    for e in range(case["E"]):
        lo, hi = st["bounds"][e], st["bounds"][e + 1]
        W = st["W"][e].to(d)
        out[lo:hi] = x[lo:hi] @ W.T if forward else dy[lo:hi] @ W
        for a in range(case["adapters"]):
            at = lo + (whose[lo:hi] == a).nonzero()[:, 0]
            if not at.numel():
                continue
            A, B, s = st["A"][a, e].to(d), st["B"][a, e].to(d), float(st["scale"][a])
            if forward:
                v[at] = x[at] @ A.T
                out[at] += s * (v[at] @ B.T)
            else:
                t = s * (dy[at] @ B)
                out[at] += t @ A
                dA[a, e] = t.T @ x[at]
                dB[a, e] = s * (dy[at].T @ st["v"][at].to(d))
    if not forward:
        return {"dx": out, "dA": dA, "dB": dB}
    if case["gelu"]:
        out = out / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (out + 0.044715 * out ** 3)))
    return {"y": out, "v": v}


def _exact_codes(value, phase, positive):
    top = value.abs().reshape(-1, _BLOCK).max(1).values
    # the least e of at least -100 with top <= 448 * 2^e
    e = torch.full_like(top, float(_LOWEST))
    e = torch.where(top > 0, torch.maximum(e, torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0))), e)
    e = torch.where(448.0 * 2.0 ** (e - 1) >= top, torch.maximum(e - 1, torch.full_like(e, float(_LOWEST))), e)
    e = torch.where(448.0 * 2.0 ** e < top, e + 1, e)
    y = value.abs() / (2.0 ** e).repeat_interleave(_BLOCK)
    step = 2.0 ** (torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3.0)   # between neighbouring codes
    step = torch.where(y < step * 8.0, step / 2.0, step).clamp(min=2.0 ** -9)
    code = (torch.floor(y / step + phase / 2.0 ** 20) * step).clamp(max=448.0)
    if positive:
        code = torch.where((value > 0) & (code == 0), torch.full_like(code, 2.0 ** -9), code)
    return code * torch.sign(value), 2.0 ** e


def _exact_adamw(case, st):
    d = torch.float64
    g = st["g"].to(d) * st["grad_scale"]
    p, b1, b2, t = st["p"].to(d), st["beta1"], st["beta2"], st["step"]
    if case["bits"] == 32:
        m, v = st["m"].to(d), st["v"].to(d)
    else:
        value = [st[x].view(torch.float8_e4m3fn).to(d) * (2.0 ** (st[x + "_power"].to(d) - 127.0)).repeat_interleave(_BLOCK) for x in ("m", "r")]
        m, v = value[0], value[1] ** 2
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g ** 2
    p = p - st["lr"] * (st["weight_decay"] * p + (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + st["eps"]))
    if case["bits"] == 32:
        return {"p": p, "half": p, "m": m, "v": v}
    del g
    i = torch.arange(p.numel(), device="cuda") % _GAP
    phase = torch.remainder(i * 2246822507 + t * 2654435769, 4294967296) // 4096
    mc, mp = _exact_codes(m, phase, False)
    rc, rp = _exact_codes(torch.sqrt(v), torch.remainder(phase + 2 ** 19, 2 ** 20), True)
    return {"p": p, "half": p, "m": mc, "m_power": mp, "r": rc, "r_power": rp}


def exact(case, seed):
    st = prepare(case, seed)
    return _exact_adamw(case, st) if case["op"] == "adamw" else _exact_adapted(case, st)
