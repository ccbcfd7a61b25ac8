"""Python binding of libfinch.so (the C ABI declared in include/finch.h).

Argument marshalling only: every step of the path (scoring, top-r, compaction), and of what
stands around it in a layer (rotation, attention, 8-bit caches), runs in the HIP kernels behind
the C ABI.  There is no CPU or PyTorch fallback: if
the shared library is missing or no GPU is usable, the calls raise.

PyTorch is used for device memory and streams: tensors supply device pointers,
`torch.cuda.current_stream()` supplies the stream.
"""
from __future__ import annotations

import ctypes
import os
import weakref
from typing import Dict, List, Optional, Sequence

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
# FINCH_LIBRARY names another build of the same sources to load instead (the measurement build
# with phase timers, libfinch_phases.so); it must exist - there is no fallback.
LIB_PATH = os.environ.get("FINCH_LIBRARY") or os.path.join(_PKG_DIR, "libfinch.so")

FINCH_OK = 0
FINCH_ERR_INVALID_ARG = -1
FINCH_ERR_UNSUPPORTED = -2
FINCH_ERR_CAPACITY = -3
FINCH_ERR_WORKSPACE = -4
FINCH_ERR_HIP = -5
FINCH_ERR_TIMEOUT = -6

FINCH_F32 = 0
FINCH_BF16 = 1

EXPORTED_SYMBOLS = (
    "finch_create", "finch_destroy", "finch_workspace_size", "finch_score", "finch_topk",
    "finch_compact", "finch_step", "finch_schedule", "finch_schedule_mode", "finch_last_hip_error",
    "finch_status_string", "finch_version", "finch_profile", "finch_profile_read",
    "finch_set_option", "finch_set_reposition", "finch_prompt_lse", "finch_loop", "finch_loop_workspace_size",
    "finch_step_static", "finch_static_scratch_bytes", "finch_loop_check",
    "finch_workspace_status", "finch_rotate", "finch_rope_frequencies", "finch_quantize", "finch_attend",
    "finch_attend_workspace_size",
)

KERNEL_NAMES = ("rowstats", "lse", "colsum", "select", "gather", "owner", "prompt_lse")

FINCH_OPT_STEP_PATH = 1
FINCH_OPT_SLICE_KEYS = 3
FINCH_OPT_LAYER_GROUP = 4
FINCH_OPT_LAYER_WAIT_TICKS = 5
FINCH_OPT_SCALE_BLOCK = 6
FINCH_SCHEDULE_PROPORTIONAL, FINCH_SCHEDULE_CONSTANT = 0, 1
FINCH_PATH_AUTO = 0
FINCH_PATH_SEPARATE = 1
FINCH_PATH_OWNER = 3
FINCH_ROPE_OFF, FINCH_ROPE_HALF, FINCH_ROPE_INTERLEAVED = 0, 1, 2
FINCH_ORDER_ASCENDING, FINCH_ORDER_RANK = 0, 1
FINCH_SCALING_NONE, FINCH_SCALING_LINEAR, FINCH_SCALING_BANDED, FINCH_SCALING_RAMP = 0, 1, 2, 3


class FinchError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str = ""):
        self.status = status
        super().__init__(f"{where}: status {status} ({detail})")


class finch_reposition(ctypes.Structure):
    _fields_ = [("pairing", ctypes.c_int32), ("order", ctypes.c_int32), ("base", ctypes.c_double)]


class finch_config(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("group_size", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class finch_problem(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k_cache", ctypes.c_void_p), ("v_cache", ctypes.c_void_p),
                ("k_chunk", ctypes.c_void_p), ("v_chunk", ctypes.c_void_p),
                ("k_out", ctypes.c_void_p), ("v_out", ctypes.c_void_p),
                ("scores", ctypes.c_void_p), ("idx", ctypes.c_void_p),
                ("n_que", ctypes.c_int32), ("c", ctypes.c_int32), ("m", ctypes.c_int32),
                ("r", ctypes.c_int32), ("k_que", ctypes.c_void_p), ("lse_extra", ctypes.c_void_p),
                ("q_doc", ctypes.c_void_p)]


_ROWS_STRIDES = ("q_row", "q_head", "k_row", "k_head", "v_row", "v_head",
                 "q_out_row", "q_out_head", "k_out_row", "k_out_head", "v_out_row", "v_out_head")


class finch_rows(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("q", "k", "v", "q_out", "k_out", "v_out", "pos", "slot")] +
                [(n, ctypes.c_int64) for n in _ROWS_STRIDES] +
                [(n, ctypes.c_int32) for n in ("n", "kv_heads", "pos0", "slots")])


class finch_rotary(ctypes.Structure):
    _fields_ = [("pairing", ctypes.c_int32), ("dims", ctypes.c_int32), ("freq", ctypes.c_void_p),
                ("q_norm", ctypes.c_void_p), ("k_norm", ctypes.c_void_p), ("eps", ctypes.c_float), ("gain", ctypes.c_float)]


class finch_rope_scaling(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("reserved", ctypes.c_int32), ("factor", ctypes.c_double),
                ("low", ctypes.c_double), ("high", ctypes.c_double), ("context", ctypes.c_double)]


class finch_quantization(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("k", "v", "k_out", "v_out", "k_scale", "v_scale")] +
                [("in_row", ctypes.c_int64), ("out_row", ctypes.c_int64), ("n", ctypes.c_int32), ("reserved", ctypes.c_int32)])


class finch_attention(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("q", "k_cache", "v_cache", "k_chunk", "v_chunk", "out", "lse", "k_scale", "v_scale",
                                                "m_live")] +
                [(n, ctypes.c_int64) for n in ("q_row", "q_head", "out_row", "out_head", "cache_row", "chunk_row")] +
                [(n, ctypes.c_int32) for n in ("n_que", "c", "m", "causal")])


_lib = None


def load_library() -> ctypes.CDLL:
    """Load libfinch.so (built in-tree by `python -m paper_2408_00167_amd.build`)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        how = ("python -m paper_2408_00167_amd.build --phase-timers" if LIB_PATH.endswith("libfinch_phases.so")
               else "python -m paper_2408_00167_amd.build")
        raise FileNotFoundError(f"{LIB_PATH} is missing: build it with `{how}` (there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    P = ctypes.POINTER
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    lib.finch_create.argtypes = [P(finch_config), P(vp)]
    lib.finch_create.restype = ctypes.c_int
    lib.finch_destroy.argtypes = [vp]
    lib.finch_destroy.restype = ctypes.c_int
    lib.finch_workspace_size.argtypes = [vp, P(finch_problem), i32, P(sz)]
    lib.finch_workspace_size.restype = ctypes.c_int
    for name in ("finch_score", "finch_topk", "finch_compact", "finch_step"):
        fn = getattr(lib, name)
        fn.argtypes = [vp, P(finch_problem), vp, i32, vp, sz, vp]
        fn.restype = ctypes.c_int
    lib.finch_schedule.argtypes = [i64, i32, i64, P(i32), i32]
    lib.finch_schedule.restype = ctypes.c_int
    lib.finch_schedule_mode.argtypes = [i64, i32, i64, i32, P(i32), i32]
    lib.finch_schedule_mode.restype = ctypes.c_int
    lib.finch_last_hip_error.argtypes = [vp]
    lib.finch_last_hip_error.restype = i32
    lib.finch_status_string.argtypes = [ctypes.c_int]
    lib.finch_status_string.restype = ctypes.c_char_p
    lib.finch_profile.argtypes = [vp, i32]
    lib.finch_profile.restype = ctypes.c_int
    lib.finch_profile_read.argtypes = [vp, P(ctypes.c_float), P(i32)]
    lib.finch_profile_read.restype = ctypes.c_int
    lib.finch_loop_workspace_size.argtypes = [vp, P(finch_problem), P(i32), i32, P(sz)]
    lib.finch_loop_workspace_size.restype = ctypes.c_int
    lib.finch_loop.argtypes = [vp, P(finch_problem), vp, P(i32), vp, i32, vp, sz, vp]
    lib.finch_loop.restype = ctypes.c_int
    lib.finch_prompt_lse.argtypes = [vp, P(finch_problem), vp, i32, vp]
    lib.finch_prompt_lse.restype = ctypes.c_int
    lib.finch_set_reposition.argtypes = [vp, P(finch_reposition)]
    lib.finch_set_reposition.restype = ctypes.c_int
    lib.finch_step_static.argtypes = [vp, P(finch_problem), vp, i32, vp]
    lib.finch_step_static.restype = ctypes.c_int
    lib.finch_static_scratch_bytes.argtypes = []
    lib.finch_static_scratch_bytes.restype = sz
    lib.finch_workspace_status.argtypes = [vp, vp, vp, P(i32)]
    lib.finch_workspace_status.restype = ctypes.c_int
    lib.finch_loop_check.argtypes = [P(finch_config), P(finch_problem), P(i32), i32]
    lib.finch_loop_check.restype = ctypes.c_int
    lib.finch_set_option.argtypes = [vp, i32, i64]
    lib.finch_set_option.restype = ctypes.c_int
    lib.finch_rotate.argtypes = [vp, P(finch_rotary), P(finch_rows), vp, i32, vp]
    lib.finch_rotate.restype = ctypes.c_int
    lib.finch_rope_frequencies.argtypes = [i32, ctypes.c_double, P(finch_rope_scaling), P(ctypes.c_double), i32, P(ctypes.c_float)]
    lib.finch_rope_frequencies.restype = ctypes.c_int
    lib.finch_quantize.argtypes = [vp, P(finch_quantization), vp, i32, vp]
    lib.finch_quantize.restype = ctypes.c_int
    lib.finch_attend_workspace_size.argtypes = [vp, P(finch_attention), i32, P(sz)]
    lib.finch_attend_workspace_size.restype = ctypes.c_int
    lib.finch_attend.argtypes = [vp, P(finch_attention), vp, i32, vp, sz, vp]
    lib.finch_attend.restype = ctypes.c_int
    lib.finch_version.argtypes = []
    lib.finch_version.restype = i32
    _lib = lib
    return lib


def _check(status: int, where: str, ctx=None):
    if status != FINCH_OK:
        lib = load_library()
        detail = lib.finch_status_string(status).decode()
        if status == FINCH_ERR_HIP and ctx is not None:
            detail += f", hipError {lib.finch_last_hip_error(ctx)}"
        raise FinchError(status, where, detail)


# ------------------------------------------------------------------ C ABI mirrors

# The Finch of each context handle: it has to know FINCH_OPT_SCALE_BLOCK however that is set, as its checks of scales go by it.
_finches = weakref.WeakValueDictionary()


def finch_create(dtype: int, head_dim: int, group_size: int) -> ctypes.c_void_p:
    lib = load_library()
    cfg = finch_config(dtype, head_dim, group_size, 0)
    ctx = ctypes.c_void_p()
    _check(lib.finch_create(ctypes.byref(cfg), ctypes.byref(ctx)), "finch_create")
    return ctx


def finch_destroy(ctx) -> None:
    _finches.pop(getattr(ctx, "value", ctx), None)
    _check(load_library().finch_destroy(ctx), "finch_destroy")


def finch_workspace_size(ctx, host_desc, n: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load_library().finch_workspace_size(ctx, host_desc, n, ctypes.byref(out)),
           "finch_workspace_size", ctx)
    return out.value


def _call(name: str, ctx, host_desc, dev_desc_ptr: int, n: int, ws_ptr: int, ws_bytes: int,
          stream: int) -> None:
    fn = getattr(load_library(), name)
    _check(fn(ctx, host_desc, ctypes.c_void_p(dev_desc_ptr), n, ctypes.c_void_p(ws_ptr),
              ws_bytes, ctypes.c_void_p(stream)), name, ctx)


def finch_prompt_lse(ctx, host_desc, dev_desc_ptr: int, n: int, stream: int = 0) -> None:
    _check(load_library().finch_prompt_lse(ctx, host_desc, ctypes.c_void_p(dev_desc_ptr), n,
                                           ctypes.c_void_p(stream)), "finch_prompt_lse", ctx)


def finch_score(ctx, host_desc, dev_desc_ptr, n, ws_ptr, ws_bytes, stream=0):
    _call("finch_score", ctx, host_desc, dev_desc_ptr, n, ws_ptr, ws_bytes, stream)


def finch_topk(ctx, host_desc, dev_desc_ptr, n, ws_ptr, ws_bytes, stream=0):
    _call("finch_topk", ctx, host_desc, dev_desc_ptr, n, ws_ptr, ws_bytes, stream)


def finch_compact(ctx, host_desc, dev_desc_ptr, n, ws_ptr, ws_bytes, stream=0):
    _call("finch_compact", ctx, host_desc, dev_desc_ptr, n, ws_ptr, ws_bytes, stream)


def finch_step(ctx, host_desc, dev_desc_ptr, n, ws_ptr, ws_bytes, stream=0):
    _call("finch_step", ctx, host_desc, dev_desc_ptr, n, ws_ptr, ws_bytes, stream)


def finch_step_static(ctx, host_desc, dev_desc_ptr, n, stream=0):
    _check(load_library().finch_step_static(ctx, host_desc, ctypes.c_void_p(dev_desc_ptr), n,
                                            ctypes.c_void_p(stream)), "finch_step_static", ctx)


def finch_static_scratch_bytes() -> int:
    return int(load_library().finch_static_scratch_bytes())


def finch_schedule(n_cont: int, m: int, k: int, constant_budget: bool = False) -> List[int]:
    steps = max(0, -(-n_cont // m)) if m > 0 else 0
    buf = (ctypes.c_int32 * max(1, steps))()
    if constant_budget:
        _check(load_library().finch_schedule_mode(n_cont, m, k, FINCH_SCHEDULE_CONSTANT, buf, steps),
               "finch_schedule_mode")
    else:
        _check(load_library().finch_schedule(n_cont, m, k, buf, steps), "finch_schedule")
    return list(buf[:steps])


def finch_profile(ctx, enable: bool) -> None:
    _check(load_library().finch_profile(ctx, 1 if enable else 0), "finch_profile", ctx)


def finch_profile_read(ctx) -> Dict[str, Dict[str, float]]:
    n = len(KERNEL_NAMES)
    ms = (ctypes.c_float * n)()
    cnt = (ctypes.c_int32 * n)()
    _check(load_library().finch_profile_read(ctx, ms, cnt), "finch_profile_read", ctx)
    return {KERNEL_NAMES[i]: {"ms": float(ms[i]), "launches": int(cnt[i])} for i in range(n)}


def finch_set_option(ctx, option: int, value: int) -> None:
    _check(load_library().finch_set_option(ctx, option, value), "finch_set_option", ctx)
    if option == FINCH_OPT_SCALE_BLOCK:
        fin = _finches.get(getattr(ctx, "value", ctx))
        if fin is not None:
            fin.scale_block, fin.key = value, tuple(list(fin.key))  # (another key: batches are looked over again)


def finch_set_reposition(ctx, pairing: int = FINCH_ROPE_OFF, order: int = FINCH_ORDER_ASCENDING,
                         base: float = 10000.0) -> None:
    how = finch_reposition(pairing, order, base)
    _check(load_library().finch_set_reposition(ctx, ctypes.byref(how)), "finch_set_reposition", ctx)


def finch_loop_workspace_size(ctx, host_desc, host_step_first, n_steps: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load_library().finch_loop_workspace_size(ctx, host_desc, host_step_first, n_steps,
                                                    ctypes.byref(out)),
           "finch_loop_workspace_size", ctx)
    return out.value


def finch_loop(ctx, host_desc, dev_desc: int, host_step_first, dev_step_first: int, n_steps: int,
               workspace: int, workspace_bytes: int, stream: int = 0) -> None:
    _check(load_library().finch_loop(ctx, host_desc, ctypes.c_void_p(dev_desc), host_step_first,
                                     ctypes.c_void_p(dev_step_first), n_steps,
                                     ctypes.c_void_p(workspace), workspace_bytes,
                                     ctypes.c_void_p(stream)),
           "finch_loop", ctx)


def finch_loop_check(dtype: int, head_dim: int, group_size: int, host_desc, host_step_first,
                     n_steps: int) -> int:
    """Host-only argument checks of finch_loop; returns the status (no exception)."""
    cfg = finch_config(dtype, head_dim, group_size, 0)
    return int(load_library().finch_loop_check(ctypes.byref(cfg), host_desc, host_step_first, n_steps))


def finch_rotate(ctx, how: finch_rotary, host_desc, dev_desc_ptr: int, n: int, stream: int = 0) -> None:
    _check(load_library().finch_rotate(ctx, ctypes.byref(how), host_desc, ctypes.c_void_p(dev_desc_ptr), n,
                                       ctypes.c_void_p(stream)), "finch_rotate", ctx)


def finch_rope_frequencies(dims: int, base: float = 10000.0, kind: int = FINCH_SCALING_NONE, factor: float = 1.0,
                           low: float = 0.0, high: float = 0.0, context: float = 0.0):
    """(radians per position of the dims / 2 channel pairs, the gain that goes with them)."""
    scaling = finch_rope_scaling(kind, 0, factor, low, high, context)
    freq, gain = (ctypes.c_double * max(1, dims // 2))(), ctypes.c_float(1.0)
    _check(load_library().finch_rope_frequencies(dims, base, ctypes.byref(scaling), freq, max(0, dims // 2), ctypes.byref(gain)),
           "finch_rope_frequencies")
    return list(freq[:dims // 2]), float(gain.value)


def finch_quantize(ctx, host_desc, dev_desc_ptr: int, n: int, stream: int = 0) -> None:
    _check(load_library().finch_quantize(ctx, host_desc, ctypes.c_void_p(dev_desc_ptr), n, ctypes.c_void_p(stream)),
           "finch_quantize", ctx)


def finch_attend_workspace_size(ctx, host_desc, n: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load_library().finch_attend_workspace_size(ctx, host_desc, n, ctypes.byref(out)), "finch_attend_workspace_size", ctx)
    return out.value


def finch_attend(ctx, host_desc, dev_desc_ptr: int, n: int, ws_ptr: int, ws_bytes: int, stream: int = 0) -> None:
    _call("finch_attend", ctx, host_desc, dev_desc_ptr, n, ws_ptr, ws_bytes, stream)


def finch_version() -> int:
    return load_library().finch_version()


# ----------------------------------------------------------------- marshalling help

def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors handed to the library must be contiguous")
    return t.data_ptr() if t.numel() > 0 else None


class Batch:
    """A descriptor array on the host and its copy on the device.

    `problems` is a sequence of dicts with tensors q, k_cache, v_cache, k_chunk,
    v_chunk, k_out, v_out, scores, idx, and optionally k_que, lse_extra, q_doc (any may be
    None where the C ABI allows NULL) and ints n_que, c, m, r.  The tensors are only read for their device
    pointers; the caller keeps them alive.
    """

    def __init__(self, problems: Sequence[Dict], device="cuda"):
        import torch
        n = len(problems)
        self.n = n
        self.host = (finch_problem * max(1, n))()
        for i, pb in enumerate(problems):
            d = self.host[i]
            for name in ("q", "k_cache", "v_cache", "k_chunk", "v_chunk", "k_out", "v_out",
                         "scores", "idx", "k_que", "lse_extra", "q_doc"):
                setattr(d, name, _ptr(pb.get(name)))
            d.n_que, d.c, d.m, d.r = int(pb["n_que"]), int(pb["c"]), int(pb["m"]), int(pb["r"])
        raw = bytes(self.host)[: n * ctypes.sizeof(finch_problem)]
        self.dev = torch.frombuffer(bytearray(raw if raw else b"\0" * 8), dtype=torch.uint8).to(device)
        self.dev_ptr = self.dev.data_ptr()


class LoopBatch:
    """The descriptor arrays of all steps of a chunk loop, step after step, with the
    table of where each step starts, on the host and on the device (finch_loop).

    `steps` is a sequence of per-step problem lists as `Batch` takes them; slot j of
    every step must describe the same problem and later steps may only drop slots
    from the end."""

    def __init__(self, steps: Sequence[Sequence[Dict]], device="cuda"):
        import torch
        flat = [pb for st in steps for pb in st]
        self.batch = Batch(flat, device=device)
        self.n_steps = len(steps)
        first = [0]
        for st in steps:
            first.append(first[-1] + len(st))
        self.host_first = (ctypes.c_int32 * len(first))(*first)
        self.dev_first = torch.tensor(first, dtype=torch.int32, device=device)


def _upload(batch, struct, device):
    """The descriptors' copy on the device of the batch's tensors (or `device` where there are none)."""
    import torch
    raw = bytes(batch.host)[: batch.n * ctypes.sizeof(struct)]
    batch.dev = torch.frombuffer(bytearray(raw if raw else b"\0" * 8), dtype=torch.uint8).to(device if batch.index is None else batch.index)
    batch.dev_ptr = batch.dev.data_ptr()


def _on_one_gpu(batch, tensors) -> None:
    """The kernels follow pointers: a tensor in host memory, or on another GPU, must not get that far."""
    for t in tensors:
        if t is not None:
            i = t.get_device()
            if i < 0 or (batch.index is not None and i != batch.index):
                raise ValueError("the tensors of a batch must lie on one GPU")
            batch.index = i


def _rows_of(t, dims: int, what: str):
    """A tensor whose last dimension lies element after element, or a ValueError."""
    if t.dim() != dims:
        raise ValueError(f"{what}: {t.dim()} dimensions, want {dims}")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{what}: the channels of a head must lie one after the other")
    return t


def _flat(t, n: int, dtype, what: str):
    """Device pointer of a contiguous tensor of at least n elements of one type (None: none)."""
    if t is None:
        return None
    if t.dtype != dtype or not t.is_contiguous() or t.numel() < n:
        raise ValueError(f"{what}: want {n} contiguous elements of {dtype}")
    return t.data_ptr() if t.numel() else None


def _same(ts, what: str):
    a = ts[0]
    for t in ts[1:]:
        if t.dtype != a.dtype or t.shape[-1] != a.shape[-1]:
            raise ValueError(f"{what}: types and channels must agree")


def _of_block(batch, block) -> None:
    """The block that a batch's scales are for (None: whichever the context has), and whether they are enough for it."""
    if block is not None and (block not in (16, 32, 64, 128) or batch.min_block > block):
        raise ValueError(f"scales for blocks of {block} rows: want 16, 32, 64 or 128, and one for each block")
    batch.block = block


class Rotary:
    """What `Finch.rotate` does to queries and keys: pairing, rotated channels, frequencies ([dims / 2] float64 on the
    device: see finch_rope_frequencies), gain, and the weights of a norm per head ([head_dim])."""

    def __init__(self, pairing: int = FINCH_ROPE_HALF, dims: int = 0, freq=None, gain: float = 1.0, q_norm=None, k_norm=None,
                 eps: float = 1e-6):
        import torch
        self.tensors, self.index = (freq, q_norm, k_norm), None  # kept alive; their GPU
        _on_one_gpu(self, self.tensors)
        self.norm = next((w for w in (q_norm, k_norm) if w is not None), None)
        for w in (q_norm, k_norm):
            if w is not None and (w.dtype != self.norm.dtype or w.dim() != 1 or w.shape != self.norm.shape or not w.is_contiguous()):
                raise ValueError("norm weights: want one contiguous [head_dim] tensor each, of one type")
        self.struct = finch_rotary(pairing, dims, _flat(freq, dims // 2, torch.float64, "freq"), _ptr(q_norm), _ptr(k_norm), eps, gain)


class RowsBatch:
    """Descriptors of `Finch.rotate`.  `requests` is a sequence of dicts with tensors q [n][G * kv_heads][d], k and v
    [n][kv_heads][d] (each may be None; views of a packed projection will do), q_out, k_out, v_out of the same layout, and
    optionally int32 `pos` [n] and `slot` [n] (rows of k_out and v_out), or an int `pos0`."""

    def __init__(self, requests: Sequence[Dict], device="cuda"):
        import torch
        self.n = len(requests)
        self.host = (finch_rows * max(1, self.n))()
        self.key = self.suits = self.index = None  # (dtype, channels, query heads per KV head or None); the context's it suits; its GPU
        self.min_block, self.block = 1, None  # (no scales)
        for i, r in enumerate(requests):
            d = self.host[i]
            _on_one_gpu(self, [r.get(name) for name in ("q", "k", "v", "q_out", "k_out", "v_out", "pos", "slot")])
            parts = {name: r.get(name) for name in ("q", "k", "v")}
            given = {name: t for name, t in parts.items() if t is not None}
            if not given:
                raise ValueError("a request needs q, k or v")
            _same(list(given.values()) + [r[name + "_out"] for name in given], "rows")
            d.n = next(iter(given.values())).shape[0]
            slot = r.get("slot")
            for name, t in given.items():
                out = _rows_of(r[name + "_out"], 3, name + "_out")
                _rows_of(t, 3, name)
                room = out.shape[0]
                if t.shape[0] != d.n or t.shape[1] != out.shape[1] or (room != d.n and (slot is None or name == "q")):
                    raise ValueError(f"{name}: {tuple(t.shape)} and {tuple(out.shape)} do not go together")
                for at, x in ((name, t), (name + "_out", out)):
                    setattr(d, at, x.data_ptr() if x.numel() else None)
                    setattr(d, at + "_row", x.stride(0) if x.shape[0] > 1 else 0)
                    setattr(d, at + "_head", x.stride(1) if x.shape[1] > 1 else 0)
            heads = [given[name].shape[1] for name in ("k", "v") if name in given]
            group = None
            if heads:
                d.kv_heads = heads[0]
                if heads[0] < 1 or heads[-1] != heads[0] or ("q" in given and given["q"].shape[1] % heads[0]):
                    raise ValueError("k and v need as many heads, q a multiple of that")
                group = given["q"].shape[1] // heads[0] if "q" in given else None
            else:
                d.kv_heads = int(r.get("kv_heads", 0))
                if d.kv_heads < 1 or given["q"].shape[1] % d.kv_heads:
                    raise ValueError("q needs a multiple of kv_heads heads")
                group = given["q"].shape[1] // d.kv_heads
            d.pos, d.pos0 = _flat(r.get("pos"), d.n, torch.int32, "pos"), int(r.get("pos0", 0))
            if slot is not None:
                rooms = {r[name + "_out"].shape[0] for name in ("k", "v") if name in given}
                if len(rooms) > 1:
                    raise ValueError("k_out and v_out need as many rows")
                d.slot, d.slots = _flat(slot, d.n, torch.int32, "slot"), rooms.pop() if rooms else 0
            first = next(iter(given.values()))
            key = (first.dtype, first.shape[-1], group if group is not None else (self.key[2] if self.key else None))
            if self.key and (key[:2] != self.key[:2] or (self.key[2] is not None and key[2] != self.key[2])):
                raise ValueError("requests of one batch: types, channels and heads per group must agree")
            self.key = key
        _upload(self, finch_rows, device)


class QuantizeBatch:
    """Descriptors of `Finch.quantize`: dicts with k, v [n][d], k_out, v_out [n][d] (float8_e4m3fn or uint8), k_scale, v_scale
    (uint8, one per block of rows).  `block`: see AttentionBatch."""

    def __init__(self, problems: Sequence[Dict], device="cuda", block: Optional[int] = None):
        import torch
        self.n = len(problems)
        self.host = (finch_quantization * max(1, self.n))()
        self.key, self.suits, self.index, self.min_block = None, None, None, 1
        eight = (torch.uint8, torch.float8_e4m3fn)
        for i, pb in enumerate(problems):
            d = self.host[i]
            k, v, ko, vo, ks, vs = (pb[name] for name in ("k", "v", "k_out", "v_out", "k_scale", "v_scale"))
            _on_one_gpu(self, (k, v, ko, vo, ks, vs))
            shape, dtype = k.shape, k.dtype
            if len(shape) != 2 or v.shape != shape or ko.shape != shape or vo.shape != shape or v.dtype != dtype:
                raise ValueError("k, v, k_out and v_out need one shape [n][d], k and v one type")
            if ko.dtype not in eight or vo.dtype not in eight:
                raise ValueError("k_out, v_out: want uint8 or float8_e4m3fn")
            n, width = shape
            (kr, kc), (vr, vc), (kor, koc), (vor, voc) = k.stride(), v.stride(), ko.stride(), vo.stride()
            if not kc == vc == koc == voc == 1:
                raise ValueError("the channels of a head must lie one after the other")
            if n > 1 and (kr != vr or kor != vor):
                raise ValueError("k and v, and k_out and v_out, need the same distance between rows")
            d.n, d.in_row, d.out_row = n, kr if n > 1 else width, kor if n > 1 else width
            d.k_scale, d.v_scale = _flat(ks, 1 if n else 0, torch.uint8, "k_scale"), _flat(vs, 1 if n else 0, torch.uint8, "v_scale")
            if n:
                d.k, d.v, d.k_out, d.v_out = k.data_ptr(), v.data_ptr(), ko.data_ptr(), vo.data_ptr()
                self.min_block = max(self.min_block, -(-n // min(ks.numel(), vs.numel())))
            key = (dtype, width, None)
            if self.key not in (None, key):
                raise ValueError("problems of one batch: types and channels must agree")
            self.key = key
        _of_block(self, block)
        _upload(self, finch_quantization, device)


_ATTENTION_TENSORS = ("q", "out", "k_cache", "v_cache", "k_chunk", "v_chunk", "lse", "k_scale", "v_scale", "m_live")


class AttentionBatch:
    """Descriptors of `Finch.attend`: dicts with q and out [n_que][G][d], k_cache, v_cache [c][d], k_chunk, v_chunk [m][d] (pairs
    may be None), and optionally lse ([G * n_que] float32), k_scale and v_scale (uint8; the cache rows are then e4m3 bytes, float8_e4m3fn
    or uint8), m_live (one int32), causal (default True).  The tensors are only read for their device pointers and strides.
    `block`: the rows per power of two that the 8-bit caches were made with; a context that is set to another number refuses the batch.
    Without it they are read with the context's number, which nothing in the bytes can confirm."""

    def __init__(self, problems: Sequence[Dict], device="cuda", block: Optional[int] = None):
        import torch
        self.n = len(problems)
        self.host = (finch_attention * max(1, self.n))()
        self.key, self.suits, self.index, self.min_block, self.planned = None, None, None, 1, None
        for i, pb in enumerate(problems):
            d = self.host[i]
            _on_one_gpu(self, [pb.get(name) for name in _ATTENTION_TENSORS])
            q, out = pb["q"], pb["out"]
            shape, dtype = q.shape, q.dtype
            if len(shape) != 3 or out.shape != shape or out.dtype != dtype:
                raise ValueError("q and out need one shape [n_que][G][d] and type")
            n_que, group, width = shape
            (qr, qh, qc), (outr, outh, outc) = q.stride(), out.stride()
            if qc != 1 or outc != 1:
                raise ValueError("the channels of a head must lie one after the other")
            d.n_que = n_que
            d.q_row, d.out_row = (qr, outr) if n_que > 1 else (width, width)
            d.q_head, d.out_head = (qh, outh) if group > 1 else (width, width)
            if n_que:
                d.q, d.out = q.data_ptr(), out.data_ptr()
            eight = pb.get("k_scale") is not None or pb.get("v_scale") is not None
            for part, count in (("cache", "c"), ("chunk", "m")):
                k, v = pb.get("k_" + part), pb.get("v_" + part)
                if k is None and v is None:
                    continue
                if k is None or v is None:
                    raise ValueError(f"k_{part} and v_{part}: both or neither")
                rows, ks, vs = k.shape, k.stride(), v.stride()
                if len(rows) != 2 or v.shape != rows or k.dtype != v.dtype or rows[1] != width or ks[1] != 1 or vs[1] != 1 or (rows[0] > 1 and ks != vs):
                    raise ValueError(f"k_{part} and v_{part}: shapes [rows][d], types and distances of rows must agree, channels lie one after the other")
                if k.dtype not in ((torch.uint8, torch.float8_e4m3fn) if eight and part == "cache" else (dtype,)):
                    raise ValueError(f"k_{part}: rows of {k.dtype}")
                if rows[0]:
                    setattr(d, count, rows[0])
                    setattr(d, part + "_row", ks[0] if rows[0] > 1 else width)
                    setattr(d, "k_" + part, k.data_ptr())
                    setattr(d, "v_" + part, v.data_ptr())
            if eight:
                for name in ("k_scale", "v_scale"):
                    if pb.get(name) is None:
                        raise ValueError("k_scale and v_scale: both or neither")
                    at = _flat(pb[name], 1 if d.c else 0, torch.uint8, name)
                    if d.c:
                        setattr(d, name, at)
                        self.min_block = max(self.min_block, -(-d.c // pb[name].numel()))
            d.lse = _flat(pb.get("lse"), group * n_que, torch.float32, "lse")
            d.m_live = _flat(pb.get("m_live"), 1, torch.int32, "m_live")
            d.causal = 1 if pb.get("causal", True) else 0
            key = (dtype, width, group)
            if self.key not in (None, key):
                raise ValueError("problems of one batch: types, channels and heads per group must agree")
            self.key = key
        _of_block(self, block)
        _upload(self, finch_attention, device)


class Finch:
    """A context plus a workspace tensor that grows on demand (outside any timed
    or captured region the caller should pre-size it with `reserve`, `reserve_loop` or
    `reserve_attend`).  A captured call goes on using the workspace of its time: keep a
    reference to `ws` beside the graph, as a later call that needs more replaces it.  Batches and the
    tensors in them are the caller's to keep until the work on them is done."""

    def __init__(self, dtype: int, head_dim: int, group_size: int, device="cuda"):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("paper_2408_00167_amd needs a GPU: there is no CPU fallback")
        self.device = torch.device(device)
        self.lib = load_library()
        self.index = torch.cuda.current_device() if self.device.index is None else self.device.index
        self.device = torch.device(self.device.type, self.index)  # (the workspace's as well, whatever device is current later)
        with torch.cuda.device(self.index):  # (a context is bound to the device that is current when it is made)
            self.ctx = finch_create(dtype, head_dim, group_size)
        _finches[self.ctx.value] = self
        self.ws = None
        self.key = (torch.bfloat16 if dtype == FINCH_BF16 else torch.float32, head_dim, group_size)
        self.scale_block = 64  # rows that share a power of two in 8-bit caches (set_scale_block)

    def close(self):
        if self.ctx is not None:
            finch_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_step_path(self, path: int) -> None:
        finch_set_option(self.ctx, FINCH_OPT_STEP_PATH, path)

    def set_reposition(self, pairing: int = FINCH_ROPE_OFF, order: int = FINCH_ORDER_ASCENDING,
                       base: float = 10000.0) -> None:
        finch_set_reposition(self.ctx, pairing, order, base)

    def reserve(self, batch: Batch) -> int:
        import torch
        need = finch_workspace_size(self.ctx, batch.host, batch.n)
        self._grow(need)
        return need

    def _grow(self, need: int) -> None:
        """A larger workspace replaces the present one only once nothing enqueued on any
        stream can still be using it (growth is rare; pre-size with reserve outside hot
        loops)."""
        import torch
        if self.ws is None or self.ws.numel() < need:
            if self.ws is not None:
                torch.cuda.synchronize(self.device)
            self.ws = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)

    def _run(self, name: str, batch: Batch, stream=None):
        import torch
        self.reserve(batch)
        s = torch.cuda.current_stream(self.device).cuda_stream if stream is None else stream
        _call(name, self.ctx, batch.host, batch.dev_ptr, batch.n, self.ws.data_ptr(),
              self.ws.numel(), s)

    def score(self, batch: Batch, stream=None):
        self._run("finch_score", batch, stream)

    def topk(self, batch: Batch, stream=None):
        self._run("finch_topk", batch, stream)

    def compact(self, batch: Batch, stream=None):
        self._run("finch_compact", batch, stream)

    def step(self, batch: Batch, stream=None):
        self._run("finch_step", batch, stream)

    def step_static(self, batch: Batch, stream=None):
        """finch_step on the library's own scratch: no workspace, nothing allocated."""
        import torch
        s = torch.cuda.current_stream(self.device).cuda_stream if stream is None else stream
        finch_step_static(self.ctx, batch.host, batch.dev_ptr, batch.n, s)

    def workspace_status(self, stream=None) -> int:
        """Waits for the stream; 0, or the status word of the last launches (FINCH_ERR_TIMEOUT raised)."""
        import torch
        s = torch.cuda.current_stream(self.device).cuda_stream if stream is None else stream
        flags = ctypes.c_int32(0)
        if self.ws is None:
            return 0
        _check(load_library().finch_workspace_status(self.ctx, ctypes.c_void_p(self.ws.data_ptr()),
                                                     ctypes.c_void_p(s), ctypes.byref(flags)),
               "finch_workspace_status", self.ctx)
        return int(flags.value)

    def prompt_lse(self, batch: Batch, stream=None):
        import torch
        s = torch.cuda.current_stream(self.device).cuda_stream if stream is None else stream
        finch_prompt_lse(self.ctx, batch.host, batch.dev_ptr, batch.n, s)

    def reserve_loop(self, lb: LoopBatch) -> int:
        import torch
        need = finch_loop_workspace_size(self.ctx, lb.batch.host, lb.host_first, lb.n_steps)
        self._grow(need)
        return need

    def loop(self, lb: LoopBatch, stream=None):
        import torch
        self.reserve_loop(lb)
        s = torch.cuda.current_stream(self.device).cuda_stream if stream is None else stream
        finch_loop(self.ctx, lb.batch.host, lb.batch.dev_ptr, lb.host_first, lb.dev_first.data_ptr(),
                   lb.n_steps, self.ws.data_ptr(), self.ws.numel(), s)

    def set_scale_block(self, rows: int) -> None:
        """Rows that share a power of two in 8-bit caches (16, 32, 64 or 128)."""
        finch_set_option(self.ctx, FINCH_OPT_SCALE_BLOCK, rows)

    def _suits(self, batch, what: str) -> None:
        """A batch built of tensors of another type or shape than the context's would be misread."""
        key = batch.key
        if key is not None and (key[:2] != self.key[:2] or key[2] not in (None, self.key[2])):
            raise ValueError(f"{what}: batch of {key}, context of {self.key}")
        if batch.index not in (None, self.index):
            raise ValueError(f"{what}: batch on GPU {batch.index}, context on {self.index}")
        # scales are read and written by the context's block of rows: there have to be enough, and for that block
        if batch.min_block > self.scale_block:
            raise ValueError(f"{what}: too few scales for blocks of this size")
        if batch.block not in (None, self.scale_block):
            raise ValueError(f"{what}: scales for blocks of {batch.block} rows, context set to {self.scale_block}")
        batch.suits = self.key

    def _stream(self, stream):
        """The stream's handle; the current one's without the 3 us that an object for it takes."""
        import torch
        return torch._C._cuda_getCurrentRawStream(self.index) if stream is None else stream

    def rotate(self, batch: RowsBatch, how: Rotary, stream=None):
        """Norm, rotary embedding and placing of projected rows."""
        if batch.suits is not self.key:
            self._suits(batch, "rotate")
        if how.index not in (None, self.index):
            raise ValueError("rotate: frequencies or weights on another GPU than the context's")
        if how.norm is not None and (how.norm.dtype, how.norm.shape[0]) != self.key[:2]:
            raise ValueError("rotate: norm weights of another type or size than the context's heads")
        st = self.lib.finch_rotate(self.ctx, how.struct, batch.host, batch.dev_ptr, batch.n, self._stream(stream))
        if st:
            _check(st, "finch_rotate", self.ctx)

    def quantize(self, batch: QuantizeBatch, stream=None):
        """Rows of K and V as e4m3 with one power of two per block of rows."""
        if batch.suits is not self.key:
            self._suits(batch, "quantize")
        st = self.lib.finch_quantize(self.ctx, batch.host, batch.dev_ptr, batch.n, self._stream(stream))
        if st:
            _check(st, "finch_quantize", self.ctx)

    def reserve_attend(self, batch: AttentionBatch) -> int:
        need = finch_attend_workspace_size(self.ctx, batch.host, batch.n)
        self._grow(need)
        batch.planned = (self, need)
        return need

    def attend(self, batch: AttentionBatch, stream=None):
        """Attention over [cache ; chunk]."""
        if batch.suits is not self.key:
            self._suits(batch, "attend")
        if batch.planned is None or batch.planned[0] is not self or self.ws is None or self.ws.numel() < batch.planned[1]:
            self.reserve_attend(batch)
        st = self.lib.finch_attend(self.ctx, batch.host, batch.dev_ptr, batch.n, self.ws.data_ptr(), self.ws.numel(), self._stream(stream))
        if st:
            _check(st, "finch_attend", self.ctx)
