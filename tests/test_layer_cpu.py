"""The calls around the compression in a model's layer, as far as they need no GPU: layouts of the descriptors, frequencies,
refusals (the checks run on the host before anything is launched)."""
import ctypes
import math

import pytest

import paper_2408_00167_amd as F
from tests import layer_reference as R

BASE = 1 << 32


def check(call, desc, dtype=F.FINCH_BF16, d=128, G=4, how=None, block=64):
    lib = F.load_library()
    cfg = F.finch_config(dtype, d, G, 0)
    arr = (type(desc) * 1)(desc)
    return lib.finch_debug_layer_check(ctypes.byref(cfg), block, call, ctypes.byref(how) if how is not None else None, arr, 1)


def rows(**kw):
    r = F.finch_rows(q=BASE, k=BASE + (1 << 20), v=BASE + (2 << 20), q_out=BASE + (3 << 20), k_out=BASE + (4 << 20), v_out=BASE + (5 << 20),
                     q_row=4096, q_head=128, k_row=1024, k_head=128, v_row=1024, v_head=128, q_out_row=128, q_out_head=128 * 16,
                     k_out_row=128, k_out_head=128 * 16, v_out_row=128, v_out_head=128 * 16, n=16, kv_heads=8, pos0=0, slots=0)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def rotary(**kw):
    h = F.finch_rotary(F.FINCH_ROPE_HALF, 128, BASE + (9 << 20), None, None, 1e-6, 1.0)
    for k, v in kw.items():
        setattr(h, k, v)
    return h


def attention(**kw):
    a = F.finch_attention(q=BASE, k_cache=BASE + (1 << 24), v_cache=BASE + (2 << 24), k_chunk=BASE + (3 << 24), v_chunk=BASE + (4 << 24),
                          out=BASE + (5 << 24), lse=BASE + (6 << 24), q_row=4096, q_head=128, out_row=512, out_head=128, cache_row=128, chunk_row=1024,
                          n_que=8, c=100, m=8, causal=1)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def quantization(**kw):
    q = F.finch_quantization(k=BASE, v=BASE + (1 << 24), k_out=BASE + (2 << 24), v_out=BASE + (3 << 24), k_scale=BASE + (4 << 24),
                             v_scale=BASE + (4 << 24) + 64, in_row=128, out_row=128, n=100, reserved=0)
    for k, v in kw.items():
        setattr(q, k, v)
    return q


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(F.finch_rows) == 176 and F.finch_rows.q_row.offset == 64 and F.finch_rows.n.offset == 160
    assert ctypes.sizeof(F.finch_rotary) == 40 and F.finch_rotary.eps.offset == 32
    assert ctypes.sizeof(F.finch_rope_scaling) == 40
    assert ctypes.sizeof(F.finch_quantization) == 72 and F.finch_quantization.n.offset == 64
    assert ctypes.sizeof(F.finch_attention) == 144 and F.finch_attention.q_row.offset == 80 and F.finch_attention.n_que.offset == 128


def test_frequencies():
    f, gain = F.finch_rope_frequencies(64, 10000.0)
    assert gain == 1.0 and f == pytest.approx([10000.0 ** (-2 * u / 64) for u in range(32)], rel=1e-14)
    lin, gain = F.finch_rope_frequencies(64, 10000.0, F.FINCH_SCALING_LINEAR, 4.0)
    assert gain == 1.0 and lin == pytest.approx([x / 4 for x in f], rel=1e-14)
    ban, gain = F.finch_rope_frequencies(128, 500000.0, F.FINCH_SCALING_BANDED, 8.0, 1.0, 4.0, 8192)
    for u, x in enumerate(ban):
        y = 500000.0 ** (-2 * u / 128)
        length = 2 * math.pi / y  # tokens of a turn
        if length < 8192 / 4:
            want = y
        elif length > 8192:
            want = y / 8
        else:
            mix = (8192 / length - 1) / 3
            want = (1 - mix) * y / 8 + mix * y
        assert x == pytest.approx(want, rel=1e-13)
    assert gain == 1.0 and ban[0] == 1.0 and ban[-1] < f[-1]
    ramp, gain = F.finch_rope_frequencies(128, 10000.0, F.FINCH_SCALING_RAMP, 16.0, 1.0, 32.0, 4096)
    assert gain == pytest.approx(0.1 * math.log(16) + 1, rel=1e-6)

    def pair(turns):
        return 128 * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(10000))
    lo, hi = math.floor(pair(32)), math.ceil(pair(1))
    for u, x in enumerate(ramp):
        y, r = 10000.0 ** (-2 * u / 128), min(1.0, max(0.0, (u - lo) / (hi - lo)))
        assert x == pytest.approx(y / 16 * r + y * (1 - r), rel=1e-13)


@pytest.mark.parametrize("args", [(63,), (0,), (-2,), (64, 1.0), (64, 1e4, 4), (64, 1e4, -1), (64, 1e4, 1, 0.5), (64, 1e4, 2, 8.0, 0.0, 4.0, 8192.0),
                                  (64, 1e4, 2, 8.0, 4.0, 4.0, 8192.0), (64, 1e4, 3, 8.0, 1.0, 32.0, 0.0), (64, float("nan"))])
def test_frequencies_refuse(args):
    with pytest.raises(F.FinchError) as e:
        F.finch_rope_frequencies(*args)
    assert e.value.status == F.FINCH_ERR_INVALID_ARG


def test_frequencies_need_room():
    buf = (ctypes.c_double * 4)()
    assert F.load_library().finch_rope_frequencies(16, 1e4, None, buf, 4, None) == F.FINCH_ERR_CAPACITY
    assert F.load_library().finch_rope_frequencies(8, 1e4, None, buf, 4, None) == F.FINCH_OK


def test_rotate_accepts():
    assert check(0, rows(), how=rotary()) == F.FINCH_OK
    assert check(0, rows(k=None, v=None, k_out=None, v_out=None), how=rotary()) == F.FINCH_OK
    assert check(0, rows(n=0, q=None, k_out=None), how=rotary()) == F.FINCH_OK
    assert check(0, rows(slot=BASE + 4, slots=500, k_out_head=128 * 500, v_out_head=128 * 500), how=rotary()) == F.FINCH_OK
    assert check(0, rows(), how=rotary(pairing=F.FINCH_ROPE_OFF, dims=0, freq=None, gain=float("nan"))) == F.FINCH_OK
    # an output on its own input
    assert check(0, rows(q_out=BASE, q_out_row=4096, q_out_head=128), how=rotary()) == F.FINCH_OK


@pytest.mark.parametrize("kw", [dict(n=-1), dict(kv_heads=0), dict(q_out=None), dict(q=BASE + 2), dict(k_out=BASE + 8), dict(pos=BASE + 2),
                                dict(slot=BASE + 1, slots=20), dict(q_row=4097), dict(k_head=-128), dict(q_out_row=64), dict(q_out_head=128),
                                dict(slot=BASE, slots=17), dict(slot=BASE, slots=-1), dict(v_row=1 << 40)])
def test_rotate_refuses(kw):
    assert check(0, rows(**kw), how=rotary()) == F.FINCH_ERR_INVALID_ARG


def test_rotate_refuses_settings():
    for kw in (dict(pairing=3), dict(freq=None), dict(gain=float("inf")), dict(q_norm=BASE + 8), dict(k_norm=BASE, eps=-1.0), dict(freq=BASE + 4)):
        assert check(0, rows(), how=rotary(**kw)) == F.FINCH_ERR_INVALID_ARG, kw
    for kw in (dict(dims=0), dict(dims=24), dict(dims=144)):
        assert check(0, rows(), how=rotary(**kw)) == F.FINCH_ERR_UNSUPPORTED, kw
    assert check(0, rows(), how=None) == F.FINCH_ERR_INVALID_ARG
    assert check(0, rows(n=(1 << 24) + 1, q_out_head=1 << 33), how=rotary()) == F.FINCH_ERR_CAPACITY


def test_attend_accepts():
    assert check(2, attention()) == F.FINCH_OK
    assert check(2, attention(n_que=0, q=None)) == F.FINCH_OK
    assert check(2, attention(c=0, k_cache=None, v_cache=None, lse=None)) == F.FINCH_OK
    assert check(2, attention(m=0, k_chunk=None, v_chunk=None, causal=0)) == F.FINCH_OK
    assert check(2, attention(c=0, m=0, k_cache=None, v_cache=None, k_chunk=None, v_chunk=None)) == F.FINCH_OK
    assert check(2, attention(k_scale=BASE + 3, v_scale=BASE + 5, cache_row=144)) == F.FINCH_OK
    assert check(2, attention(out_row=128, out_head=128 * 8)) == F.FINCH_OK   # [head][row][channel]
    assert check(2, attention(q_row=0, q_head=0)) == F.FINCH_OK              # one row for all
    assert check(2, attention(cache_row=0)) == F.FINCH_OK
    assert check(2, attention(out=BASE + (3 << 24) + 256 * 100)) == F.FINCH_OK  # behind the chunk's 7 * 2048 + 256 bytes


@pytest.mark.parametrize("kw", [dict(n_que=-1), dict(c=-1), dict(m=-1), dict(causal=2), dict(q=None), dict(out=None), dict(out=BASE + (5 << 24) + 8),
                                dict(lse=BASE + 2), dict(m_live=BASE + 1), dict(q_row=4), dict(out_row=64), dict(out_head=64), dict(out_row=128),
                                dict(out_row=256, out_head=256), dict(k_cache=None), dict(v_chunk=None), dict(k_chunk=BASE + 1), dict(cache_row=-128),
                                dict(chunk_row=129), dict(k_scale=BASE), dict(out=BASE), dict(out=BASE + (3 << 24) + 2048 * 7 + 240),
                                dict(out=BASE + (1 << 24) + 99 * 256)])
def test_attend_refuses(kw):
    assert check(2, attention(**kw)) == F.FINCH_ERR_INVALID_ARG


def test_attend_refuses_what_it_has_not():
    assert check(2, attention(k_scale=BASE, v_scale=BASE), dtype=F.FINCH_F32) == F.FINCH_ERR_UNSUPPORTED
    assert check(2, attention(c=1 << 24, m=1)) == F.FINCH_ERR_CAPACITY
    assert check(2, attention(n_que=(1 << 22) + 1)) == F.FINCH_ERR_CAPACITY


def test_quantize_checks():
    assert check(1, quantization()) == F.FINCH_OK
    assert check(1, quantization(n=0, k=None)) == F.FINCH_OK
    # keys and values in turn, row by row
    assert check(1, quantization(out_row=256, v_out=BASE + (2 << 24) + 128)) == F.FINCH_OK
    assert check(1, quantization(out_row=240, v_out=BASE + (2 << 24) + 128)) == F.FINCH_ERR_INVALID_ARG
    assert check(1, quantization(out_row=256, v_out=BASE + (2 << 24) + 112)) == F.FINCH_ERR_INVALID_ARG
    for kw in (dict(n=-1), dict(reserved=1), dict(k=None), dict(v_scale=None), dict(k=BASE + 8), dict(v_out=BASE + (3 << 24) + 4), dict(out_row=64),
               dict(in_row=4), dict(out_row=130), dict(k_out=BASE), dict(v_scale=BASE + (4 << 24) + 1), dict(v_out=BASE + (2 << 24))):
        assert check(1, quantization(**kw)) == F.FINCH_ERR_INVALID_ARG, kw
    assert check(1, quantization(n=(1 << 24) + 1)) == F.FINCH_ERR_CAPACITY


def test_reference_knows_its_formats():
    import torch
    t = R.e4m3_table()
    assert t[126] == 448 and t[1] == 2.0 ** -9 and t[8] == 2.0 ** -6 and bool((t[1:] > t[:-1]).all())
    x = torch.tensor([[448.0, 1.0625, -1.1875, 2.0 ** -10, 0.0, 3 * 2.0 ** -10, 17.0, 19.0] * 16])
    v, e = R.quantized(x, 16)
    assert e == [0] and v[0, :8].tolist() == [448.0, 1.0, -1.25, 0.0, 0.0, 2.0 ** -8, 16.0, 20.0]
    assert R.quantized(x * 1.01, 16)[1] == [1] and R.quantized(x * 0, 16)[1] == [0] and R.quantized(x * 2.0 ** -120, 16)[1] == [-100]
    want = torch.arange(128, dtype=torch.uint8)[:127]
    assert torch.equal(R.e4m3_values(want), want.view(torch.float8_e4m3fn).double())


def test_attention_kernels_keep_their_rows_in_registers():
    """At most four 4-byte values a lane are spilled; a tile of keys, or a row's results, are 16 to 64."""
    import re

    from tests.test_kernel_registers import kernels
    seen = 0
    for name, meta in kernels().items():
        m = re.search(r"(attend_rows16|attend_rows|attend_tiles|attend_rows_f32|attend_join)ILi(\d+)E", name)
        if m:
            seen += 1
            assert meta[".vgpr_spill_count"] <= 4, f"{name}: {meta['.vgpr_spill_count']} spilled"
    assert seen == 18  # three bf16 kernels of 2 head sizes, 8-bit caches or not, fp32 of 2, joins of 2 for either type


def test_rotate_refuses_positions_past_32_bits():
    """pos0 + t has to fit, as the header says: t goes to n - 1."""
    top = (1 << 31) - 1
    assert check(0, rows(pos0=top - 15), how=rotary()) == F.FINCH_OK
    assert check(0, rows(pos0=top - 14), how=rotary()) == F.FINCH_ERR_INVALID_ARG
    assert check(0, rows(pos0=-top - 1), how=rotary()) == F.FINCH_OK
    # given positions are read instead, and without a rotation none are
    assert check(0, rows(pos0=top, pos=BASE + 4), how=rotary()) == F.FINCH_OK
    assert check(0, rows(pos0=top), how=rotary(pairing=F.FINCH_ROPE_OFF, dims=0, freq=None)) == F.FINCH_OK


def test_rotate_strides_times_slots_past_63_bits():
    """Offsets of 2^30 slots have to stay below 2^60 elements as those of 2^24 tokens do."""
    far = dict(slot=BASE + 4, slots=1 << 30, v=None, v_out=None)
    ok = dict(k_out_row=128, k_out_head=1 << 36)
    assert check(0, rows(**far, **ok), how=rotary()) == F.FINCH_ERR_INVALID_ARG          # 2^30 rows of 128 pass the next head
    assert check(0, rows(**far, k_out_row=8 * 128, k_out_head=128), how=rotary()) == F.FINCH_OK
    for row in ((1 << 33), (1 << 35), (1 << 36) - 8):
        assert check(0, rows(**far, k_out_row=row, k_out_head=128), how=rotary()) == F.FINCH_ERR_CAPACITY, row
    assert check(0, rows(slot=BASE + 4, slots=1 << 26, v=None, v_out=None, k_out_row=(1 << 36) - 8, k_out_head=128), how=rotary()) == F.FINCH_ERR_CAPACITY
