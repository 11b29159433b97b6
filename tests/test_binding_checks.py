"""What the Python calls of the adapters and the optimizer step refuse before a kernel would misread it: host memory, other types, too few
elements, gaps, another device than the current one.  On the CPU: a tensor that only says that it is on a device takes the place of those that are."""

import types

import pytest
import torch

from paper_2304_11414_amd import binding as B

CFG = dict(rows=100, K=64, N=128, n_exp=2, n_adapters=3, rank=16)
HALF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


class Fake:
    """Shape, type and device of a tensor; nothing reads it (the call is refused, or the library's is replaced)."""

    def __init__(self, dtype, *shape, device=0, contiguous=True):
        self.t, self.dtype, self.device_index, self.contiguous = torch.empty(shape, dtype=dtype, device="meta"), dtype, device, contiguous

    def get_device(self):
        return self.device_index

    def numel(self):
        return self.t.numel()

    def element_size(self):
        return self.t.element_size()

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return 0x1000


def good(**over):
    a = dict(x=Fake(HALF, 100, 64), offsets=Fake(I32, 3), W=Fake(HALF, 2, 128, 64), A=Fake(HALF, 3, 2, 16, 64), B=Fake(HALF, 3, 2, 128, 16),
             scale=Fake(F32, 3), adapter=Fake(I32, 100), perm=Fake(I32, 100), dy=Fake(HALF, 100, 128), y=Fake(HALF, 100, 128), v=Fake(F32, 100, 16),
             dx=Fake(HALF, 100, 64), dA=Fake(F32, 3, 2, 16, 64), dB=Fake(F32, 3, 2, 128, 16), workspace=Fake(torch.uint8, 1 << 20))
    return {**a, **over}


NAMES = {"moe_adapter_forward": ("x", "offsets", "W", "A", "B", "scale", "adapter", "perm", "y", "v", "workspace"),
         "moe_adapter_backward": ("x", "offsets", "W", "A", "B", "scale", "adapter", "perm", "dy", "v", "dx", "dA", "dB", "workspace")}


@pytest.fixture(autouse=True)
def library(monkeypatch):
    """Every call of the library is counted and succeeds."""
    made = []
    call = lambda *a: made.append(a) or 0
    monkeypatch.setattr(B, "load_library", lambda: types.SimpleNamespace(moe_adapter_forward=call, moe_adapter_backward=call, moe_adamw_step=call))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(cuda_stream=0, device_index=0))
    return made


def run(call, **over):
    a, stream = good(**over), over.pop("stream", None)
    return getattr(B, call)(B.make_adapter_config(**CFG), *(a[n] for n in NAMES[call]), stream=stream)


@pytest.mark.parametrize("call", NAMES)
def test_adapter_arrays(call, library):
    run(call)
    run(call, scale=None, perm=None, dx=None)
    assert len(library) == 2
    for name in NAMES[call]:
        t = good()[name]
        wrong = [Fake(t.dtype, *t.t.shape, device=-1), Fake(t.dtype, *t.t.shape, device=1), Fake(t.dtype, *t.t.shape, contiguous=False)]
        if name != "workspace":       # (its size is the library's to check)
            wrong += [Fake(torch.float64, *t.t.shape)]
            wrong += [Fake(t.dtype, t.numel() - 1)] if name != "adapter" else [Fake(t.dtype, 0)]
        for bad in wrong:
            with pytest.raises(B.MoeError):
                run(call, **{name: bad})
    with pytest.raises(B.MoeError):
        run(call, stream=types.SimpleNamespace(cuda_stream=0, device_index=1))
    assert len(library) == 2


@pytest.mark.parametrize("call", NAMES)
def test_all_tensors_on_another_device_than_the_current_one(call, library):
    elsewhere = {n: Fake(t.dtype, *t.t.shape, device=1) for n, t in good().items()}
    with pytest.raises(B.MoeError):
        run(call, **elsewhere)
    assert not library


def test_adamw_step(library):
    cfg, memory, values = B.make_adamw_config(), Fake(torch.uint8, 256), Fake(I32, 4)
    B.moe_adamw_step(cfg, B.AdamwPlan(memory, 1, 1, []), values)
    assert len(library) == 1
    for bad in (Fake(I32, 4, device=-1), Fake(I32, 4, device=1), Fake(F32, 4), Fake(I32, 3), Fake(I32, 4, contiguous=False), torch.zeros(4, dtype=I32)):
        with pytest.raises(B.MoeError):
            B.moe_adamw_step(cfg, B.AdamwPlan(memory, 1, 1, []), bad)
    with pytest.raises(B.MoeError):
        B.moe_adamw_step(cfg, B.AdamwPlan(Fake(torch.uint8, 256, device=1), 1, 1, []), Fake(I32, 4, device=1))
    assert len(library) == 1


def test_adamw_scalars_on_a_named_device():
    s = B.moe_adamw_scalars(7, 0.5, 0.25, True, device="cpu")
    assert s.tolist()[:2] == [7, 1] and s[2:].view(torch.float32).tolist() == [0.5, 0.25]
