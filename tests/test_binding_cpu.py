"""What the binding checks before it calls the library, without a GPU: the library is a stand-in that notes its calls."""
import contextlib
import ctypes
import types

import pytest
import torch

import paper_2408_00167_amd as F


class Library:
    """Every call succeeds and is noted."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            if name == "finch_create":
                args[1]._obj.value = 4096 + 64 * len(self.calls)
            return F.FINCH_OK
        return call


@pytest.fixture
def lib(monkeypatch):
    lib = Library()
    monkeypatch.setattr(F, "_lib", lib)
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "device", lambda index: contextlib.nullcontext())
    return lib


def batch(fin, min_block):
    """As QuantizeBatch and AttentionBatch look to a call."""
    return types.SimpleNamespace(host=None, dev_ptr=0, n=1, key=fin.key, suits=None, index=0, min_block=min_block, planned=(fin, 0))


def test_scales_are_counted_by_the_context_s_block_however_it_was_set(lib):
    fin = F.Finch(F.FINCH_BF16, 128, 4)
    fin.ws = torch.zeros(256, dtype=torch.uint8)
    few = batch(fin, 64)  # scales for blocks of 64 rows
    fin.quantize(few, stream=0)
    fin.attend(few, stream=0)
    for set_block in (fin.set_scale_block, lambda rows: F.finch_set_option(fin.ctx, F.FINCH_OPT_SCALE_BLOCK, rows),
                      lambda rows: F.finch_set_option(ctypes.c_void_p(fin.ctx.value), F.FINCH_OPT_SCALE_BLOCK, rows)):
        set_block(32)
        assert fin.scale_block == 32
        lib.calls.clear()
        for call in (fin.quantize, fin.attend):
            with pytest.raises(ValueError):
                call(few, stream=0)
        assert lib.calls == []
        set_block(128)
        fin.quantize(few, stream=0)
        fin.attend(few, stream=0)
    other = F.Finch(F.FINCH_BF16, 128, 4)
    assert other.scale_block == 64 and fin.scale_block == 128
    fin.close()
    assert fin.scale_block == 64
    other.close()


def test_the_workspace_lies_on_the_context_s_gpu_whatever_device_is_current(lib, monkeypatch):
    """A context is bound to the GPU that is current when it is made; a workspace of another GPU must not reach its kernels."""
    fin = F.Finch(F.FINCH_BF16, 128, 4)          # GPU 0 is current
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    asked = []

    def empty(*size, device=None, dtype=None):
        asked.append(torch.device(device))
        return torch.zeros(*size, dtype=dtype)
    monkeypatch.setattr(torch, "empty", empty)
    fin._grow(1000)
    assert fin.device == torch.device("cuda", 0) and asked == [torch.device("cuda", 0)]
    second = F.Finch(F.FINCH_BF16, 128, 4)
    assert second.device == torch.device("cuda", 1) and F.Finch(F.FINCH_BF16, 128, 4, device="cuda:0").index == 0
