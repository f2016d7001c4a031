"""The binding's append and block calls refuse tensors that lie on another device than their context, before anything reaches the
library (no GPU: tensors that only say where they are, and a library that only counts its calls)."""
import types

import pytest
import torch

from paper_2511_06029_b200 import binding

F32, BF16, I8, I32 = torch.float32, torch.bfloat16, torch.int8, torch.int32


class Tensor:
    """What the binding asks of a tensor."""

    def __init__(self, shape, dtype, device=1):
        self.shape, self.dtype, self.index = torch.Size(shape), dtype, device
        self.is_cuda, self.device = device >= 0, torch.device("cuda", device) if device >= 0 else torch.device("cpu")

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return True

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def data_ptr(self):
        return 256


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append(name) or binding.OK


L, B, HQ, HKV, D, T, CAP, N = 2, 3, 4, 2, 64, 16, 5, 7


def context(monkeypatch):
    monkeypatch.setattr(binding, "_raw_stream", lambda device: 0)
    c = binding.Context.__new__(binding.Context)
    c.lib, c.device, c.h = Library(), 1, None
    return c


def block_cache(device):
    lead = (L, B, HKV, CAP)
    t = lambda shape, dtype: Tensor(shape, dtype, device)  # noqa: E731
    return binding.BlockCache(HQ, t(lead + (T, D), I8), t(lead + (T, D), I8), t(lead, F32), t(lead, F32), t(lead + (2, D), I8), t((L, B, HKV, T, D), BF16),
                              t((L, B, HKV, T, D), BF16), t((L, B, HKV), I32))


def plain_cache(device):
    lead = (L, B, HKV, 32)
    return types.SimpleNamespace(len=Tensor((L, B, HKV), I32, device), batch=B, n_kv_heads=HKV, n_q_heads=HQ, head_dim=D, act_dtype=BF16, c=binding.lethe_cache())


def rotary(device):
    return binding.Rotary([0] * 32, [0.0] * 32, Tensor((1, N), I32, device))


# call -> the tensors it takes: name -> how it is made on a device
ROWS = {"cache": block_cache, "start": lambda d: Tensor((B + 1,), I32, d), "k": lambda d: Tensor((L, N, HKV, D), BF16, d), "v": lambda d: Tensor((L, N, HKV, D), BF16, d),
        "rotary": rotary, "q": lambda d: Tensor((L, N, HQ, D), BF16, d), "q_out": lambda d: Tensor((L, N, HQ, D), BF16, d)}
QUERY = {"cache": block_cache, "q": lambda d: Tensor((L, B, HQ, D), BF16, d), "selected": lambda d: Tensor((L, B, HKV, 2), I32, d)}
CALLS = {
    "append": (dict(ROWS, cache=plain_cache, pos=lambda d: Tensor((N,), I32, d)),
               lambda c, a: c.append(a["cache"], 0, L, a["start"], N, a["k"], a["v"], a["pos"], rotary=a["rotary"], q=a["q"], q_out=a["q_out"])),
    "block_append": (ROWS, lambda c, a: c.block_append(a["cache"], 0, L, a["start"], N, a["k"], a["v"], rotary=a["rotary"], q=a["q"], q_out=a["q_out"])),
    "block_read": ({"cache": block_cache, "begin": lambda d: Tensor((B,), I32, d), "k": lambda d: Tensor((L, B, HKV, N, D), BF16, d),
                    "v": lambda d: Tensor((L, B, HKV, N, D), BF16, d)}, lambda c, a: c.block_read(a["cache"], 0, L, a["begin"], a["k"], a["v"])),
    "block_select": (QUERY, lambda c, a: c.block_select(a["cache"], 0, L, a["q"], 0, 1, a["selected"])),
    "block_attend": (dict(QUERY, out=lambda d: Tensor((L, B, HQ, D), BF16, d), lse=lambda d: Tensor((L, B, HQ), F32, d)),
                     lambda c, a: c.block_attend(a["cache"], 0, L, a["q"], [0.1] * L, a["out"], lse=a["lse"], selected=a["selected"])),
}


@pytest.mark.parametrize("name", CALLS)
def test_the_call_goes_through(monkeypatch, name):
    c = context(monkeypatch)
    takes, call = CALLS[name]
    call(c, {k: make(1) for k, make in takes.items()})
    assert c.lib.calls == ["lethe_" + name]


@pytest.mark.parametrize("name,which", [(name, which) for name, (takes, _) in CALLS.items() for which in takes])
@pytest.mark.parametrize("device", [0, 2, -1])
def test_another_device_is_refused(monkeypatch, name, which, device):
    c = context(monkeypatch)
    takes, call = CALLS[name]
    with pytest.raises(AssertionError):
        call(c, {k: make(device if k == which else 1) for k, make in takes.items()})
    assert c.lib.calls == []
