"""The new calls as a program uses them together: an MoE layer with frozen experts and adapters of several requests on both
projections: route, slice, two adapted projections, combine; the adapters' gradients; the AdamW step that writes the 16-bit
adapters the next forward reads.  Checked against automatic differentiation in float64 on the CPU with the routing that the layer chose.

Tolerance of a gradient, in the 2-norm: between the loss and a gradient at most six tensors have been rounded to bf16 (x W, GeLU of it, the second
projection or its gradient, dU, and the low-rank factors), each off by at most 2^-8 of its own norm, and |GeLU'| <= 1.13: 6 * 1.13 * 2^-8
= 2.7 %."""

import numpy as np
import pytest
import torch

from paper_2304_11414_amd import binding as B

pytestmark = pytest.mark.gpu
OFF = 6 * 1.13 * 2.0 ** -8


def gelu(u):
    return 0.5 * u * (1.0 + torch.tanh(0.7978845608028654 * (u + 0.044715 * u ** 3)))


class Layer:
    def __init__(self, T=200, d=128, F=256, E=4, k=2, adapters=3, rank=8, seed=0):
        g = torch.Generator().manual_seed(seed)
        n = lambda *s, std: (torch.randn(*s, generator=g) * std).to(torch.bfloat16).cuda()
        self.T, self.d, self.F, self.E, self.k, self.rows = T, d, F, E, k, T * k
        self.x, self.Wg = n(T, d, std=1.0), n(E, d, std=d ** -0.5)
        self.W1, self.W2 = n(E, F, d, std=d ** -0.5), n(E, d, F, std=F ** -0.5)
        self.request = (torch.arange(T) * 5 // T - 1).to(torch.int32).cuda()      # -1 (none), 0, 1, 2, 3 (no such adapter: none)
        self.scale = torch.tensor([0.5, 1.0, 2.0], device="cuda")
        self.adapters = {name: n(*shape, std=0.3 * shape[-1] ** -0.5) for name, shape in
                         dict(A1=(adapters, E, rank, d), B1=(adapters, E, F, rank), A2=(adapters, E, rank, F), B2=(adapters, E, d, rank)).items()}
        self.cfg = B.make_config(T, d, F, E, k, renorm_topk=True)
        self.up = B.make_adapter_config(self.rows, d, F, E, adapters, rank, top_k=k)
        self.down = B.make_adapter_config(self.rows, F, d, E, adapters, rank, top_k=k)
        e = lambda *s, dt=torch.bfloat16: torch.empty(*s, dtype=dt, device="cuda")
        i32, f32 = torch.int32, torch.float32
        self.idx, self.gate = e(T, k, dt=i32), e(T, k, dt=f32)
        self.counts, self.offsets, self.perm, self.inv = e(E, dt=i32), e(E + 1, dt=i32), e(self.rows, dt=i32), e(T, k, dt=i32)
        self.xs, self.U, self.ys, self.out = e(self.rows, d), e(self.rows, F), e(self.rows, d), e(T, d)
        self.v1, self.v2 = e(self.rows, rank, dt=f32), e(self.rows, rank, dt=f32)
        size = max(B.moe_dispatch_workspace_bytes(self.cfg), *(f(c) for f in (B.moe_adapter_workspace_bytes, B.moe_adapter_backward_workspace_bytes)
                                                               for c in (self.up, self.down)))
        self.ws = e(size, dt=torch.uint8)

    def route(self):
        B.moe_gate(self.cfg, self.x, self.Wg, None, None, None, self.idx, self.gate)
        B.moe_slice_dispatch(self.cfg, self.x, self.idx, self.counts, self.offsets, self.perm, self.inv, self.xs, self.ws)

    def forward(self):
        a = self.adapters
        B.moe_adapter_forward(self.up, self.xs, self.offsets, self.W1, a["A1"], a["B1"], self.scale, self.request, self.perm, self.U, self.v1, self.ws)
        self.H = gelu(self.U.float()).to(torch.bfloat16)
        B.moe_adapter_forward(self.down, self.H, self.offsets, self.W2, a["A2"], a["B2"], self.scale, self.request, self.perm, self.ys, self.v2, self.ws)
        B.moe_combine(self.cfg, self.ys, self.inv, self.gate, self.out)

    def serve(self):
        """The same with the GeLU in the first call, which rounds the pre-activations nowhere."""
        a, out = self.adapters, torch.empty_like(self.out)
        up = B.make_adapter_config(self.rows, self.d, self.F, self.E, self.up.n_adapters, self.up.rank, top_k=self.k, gelu=True)
        H, ys = torch.empty_like(self.U), torch.empty_like(self.ys)
        B.moe_adapter_forward(up, self.xs, self.offsets, self.W1, a["A1"], a["B1"], self.scale, self.request, self.perm, H, self.v1, self.ws)
        B.moe_adapter_forward(self.down, H, self.offsets, self.W2, a["A2"], a["B2"], self.scale, self.request, self.perm, ys, self.v2, self.ws)
        B.moe_combine(self.cfg, ys, self.inv, self.gate, out)
        return out

    def backward(self, d_out):
        a = self.adapters
        grads = {name: torch.empty(t.shape, device="cuda") for name, t in a.items()}
        dY = (d_out[self.perm.long() // self.k].float() * self.gate.view(-1)[self.perm.long()][:, None]).to(torch.bfloat16)
        dH = torch.empty_like(self.U)
        B.moe_adapter_backward(self.down, self.H, self.offsets, self.W2, a["A2"], a["B2"], self.scale, self.request, self.perm, dY, self.v2, dH,
                               grads["A2"], grads["B2"], self.ws)
        u = self.U.float()
        th = torch.tanh(0.7978845608028654 * (u + 0.044715 * u ** 3))
        slope = 0.5 * (1 + th) + 0.5 * u * (1 - th * th) * 0.7978845608028654 * (1 + 3 * 0.044715 * u * u)
        dU = (dH.float() * slope).to(torch.bfloat16)
        dx = torch.empty_like(self.xs)
        B.moe_adapter_backward(self.up, self.xs, self.offsets, self.W1, a["A1"], a["B1"], self.scale, self.request, self.perm, dU, self.v1, dx,
                               grads["A1"], grads["B1"], self.ws)
        return grads, dx

    def reference(self, d_out, adapters=None):
        """out, the gradients of sum(d_out * out) and that of the sliced tokens, in float64."""
        D = lambda t: t.detach().double().cpu()
        a = {n: D(t).requires_grad_() for n, t in (adapters or self.adapters).items()}
        token = self.perm.long().cpu() // self.k
        who = self.request.long().cpu()[token]
        who = torch.where((who < 0) | (who >= self.scale.numel()), -1, who)
        xs = D(self.x)[token].requires_grad_()
        lo, hi = self.offsets.tolist()[:-1], self.offsets.tolist()[1:]

        def adapted(z, W, A, Bm):
            parts = []
            for e in range(self.E):
                for r in range(lo[e], hi[e]):
                    y = W[e] @ z[r]
                    if who[r] >= 0:
                        y = y + float(self.scale[who[r]]) * (Bm[who[r], e] @ (A[who[r], e] @ z[r]))
                    parts.append(y)
            return torch.stack(parts)
        H = gelu(adapted(xs, D(self.W1), a["A1"], a["B1"]))
        ys = adapted(H, D(self.W2), a["A2"], a["B2"])
        w = D(self.gate).view(-1)[self.perm.long().cpu()]
        out = torch.zeros(self.T, self.d, dtype=torch.float64).index_add(0, token, ys * w[:, None])
        (out * D(d_out)).sum().backward()
        return out.detach(), {n: t.grad for n, t in a.items()}, xs.grad


def near(got, want, off, what):
    got = got.double().cpu()
    assert float((got - want).norm()) <= off * float(want.norm()), (what, float((got - want).norm() / want.norm()))


@pytest.mark.parametrize("bits", [32, 8])
def test_fine_tuning_steps_of_a_layer(bits):
    L = Layer(seed=bits)
    g = torch.Generator().manual_seed(1)
    d_out = torch.randn(L.T, L.d, generator=g).to(torch.bfloat16).cuda()
    L.route()
    master = {n: t.float() for n, t in L.adapters.items()}
    grads = {n: torch.empty_like(t) for n, t in master.items()}
    moments = {}
    for n, t in master.items():
        z = lambda size: torch.zeros(size, dtype=torch.uint8 if bits == 8 else torch.float32, device="cuda")
        moments[n] = dict(m=z(t.numel()), v=z(t.numel()))
        if bits == 8:
            moments[n].update(m_power=z(-(-t.numel() // 32)), v_power=z(-(-t.numel() // 32)))
    opt = B.make_adamw_config(0.9, 0.99, 1e-6, bits)
    plan = B.moe_adamw_plan(opt, [dict(p=master[n], g=grads[n], half=L.adapters[n], weight_decay=0.1, **moments[n]) for n in master])
    lr = 1e-3
    for step in (1, 2):
        L.forward()
        out, want, want_dx = L.reference(d_out)
        near(L.out, out, OFF, "out")
        near(L.serve(), out, OFF, "served")
        got, dx = L.backward(d_out)
        for n in grads:
            grads[n].copy_(got[n])
            near(got[n], want[n], OFF, n)
        near(dx, want_dx, OFF, "dx")
        before = {n: t.double().cpu() for n, t in master.items()}
        B.moe_adamw_step(opt, plan, B.moe_adamw_scalars(step, lr))
        torch.cuda.synchronize()
        for n in master:
            assert torch.equal(L.adapters[n], master[n].to(torch.bfloat16))
            if step == 1:      # both moments from zero: the update is lr * g / (|g| + eps') whatever the moments are stored in
                gr = grads[n].double().cpu()
                after = before[n] * (1 - lr * 0.1) - lr * gr / (gr.abs() + opt.eps)
                assert float((master[n].double().cpu() - after).abs().max()) <= 24 * 2.0 ** -24 * (float(before[n].abs().max()) + lr)
            else:
                assert not torch.equal(before[n], master[n].double().cpu())
