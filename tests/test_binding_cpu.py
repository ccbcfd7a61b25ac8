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
    return types.SimpleNamespace(host=None, dev_ptr=0, n=1, key=fin.key, suits=None, index=0, min_block=min_block, block=None, planned=(fin, 0))


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
    with pytest.raises(ValueError):  # a batch that one context has taken is looked over by the other
        other.quantize(batch(fin, 128), stream=0)
    fin.close()
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


@pytest.fixture
def on_host(monkeypatch):
    """Batches of tensors in host memory, which are described and not uploaded."""
    monkeypatch.setattr(F, "_on_one_gpu", lambda batch, tensors: setattr(batch, "index", 0))
    monkeypatch.setattr(F, "_upload", lambda batch, struct, device: setattr(batch, "dev_ptr", 0))


def eight_bits(c, scales, rows=1, group=4, d=128):
    byte = lambda *s: torch.zeros(*s, dtype=torch.uint8)  # noqa: E731
    half = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    return dict(q=half(rows, group, d), out=half(rows, group, d), k_cache=byte(c, d), v_cache=byte(c, d), k_scale=byte(scales), v_scale=byte(scales),
                k_chunk=half(rows, d), v_chunk=half(rows, d))


def test_an_empty_8_bit_cache_has_no_scales(on_host):
    """As QuantizeBatch takes it: no rows, no blocks, no scales."""
    batch = F.AttentionBatch([eight_bits(0, 0), eight_bits(100, 2)])
    assert [batch.host[i].c for i in range(2)] == [0, 100] and batch.min_block == 50
    assert not batch.host[0].k_scale and not batch.host[0].v_scale
    only_one = eight_bits(0, 0)
    only_one["k_scale"] = torch.zeros(1, dtype=torch.uint8)
    assert F.AttentionBatch([only_one]).min_block == 1
    assert not F.AttentionBatch([only_one]).host[0].k_scale
    with pytest.raises(ValueError):
        F.AttentionBatch([eight_bits(1, 0)])
    with pytest.raises(ValueError):
        F.AttentionBatch([{**eight_bits(0, 0), "v_scale": None}])


def test_a_batch_that_names_its_block_is_not_read_with_another(lib, on_host):
    """Scales for blocks of 16 rows are more than enough for blocks of 64, and mean other rows."""
    fin = F.Finch(F.FINCH_BF16, 128, 4)
    fin.ws = torch.zeros(256, dtype=torch.uint8)
    cache = eight_bits(100, 7)
    rows = dict(k=torch.zeros(100, 128, dtype=torch.bfloat16), v=torch.zeros(100, 128, dtype=torch.bfloat16), k_out=cache["k_cache"], v_out=cache["v_cache"],
                k_scale=cache["k_scale"], v_scale=cache["v_scale"])
    made, read = F.QuantizeBatch([rows], block=16), F.AttentionBatch([cache], block=16)
    for context_s in (64, 32, 128):
        fin.set_scale_block(context_s)
        lib.calls.clear()
        with pytest.raises(ValueError):
            fin.quantize(made)
        with pytest.raises(ValueError):
            fin.attend(read)
        assert lib.calls == []
    fin.set_scale_block(16)
    fin.quantize(made, stream=0)
    fin.attend(read, stream=0)
    for bad in (0, 8, 48, 256):
        with pytest.raises(ValueError):
            F.AttentionBatch([cache], block=bad)
        with pytest.raises(ValueError):
            F.QuantizeBatch([rows], block=bad)
    with pytest.raises(ValueError):  # 100 rows are seven blocks of 16
        F.AttentionBatch([eight_bits(100, 6)], block=16)
    with pytest.raises(ValueError):
        F.QuantizeBatch([{**rows, "v_scale": torch.zeros(6, dtype=torch.uint8)}], block=16)
