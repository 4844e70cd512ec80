"""Thin Python binding of the C ABI in include/kivi.h (argument marshalling only).

Every step of the path runs in the HIP library; PyTorch only provides device memory and the
stream.  There is no CPU fallback: if libkivi_hip.so is missing, loading fails loudly.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG_DIR, "libkivi_hip.so")

KIVI_OK = 0
KIVI_ERR_INVALID_ARG = -1
KIVI_ERR_UNSUPPORTED = -2
KIVI_ERR_WORKSPACE = -3
KIVI_ERR_HIP = -4
KIVI_FLUSH_WINDOW = 0
KIVI_FLUSH_ALG1 = 1
KIVI_DECODE_AUTO = 0
KIVI_DECODE_VALU = 1
KIVI_DECODE_MFMA = 2
KIVI_DECODE_MFMA_ONE = 3
KIVI_DECODE_MFMA_TWO = 4
KIVI_TYPE_FP16 = 0
KIVI_TYPE_BF16 = 1

EXPORTS = [
    "kivi_status_string", "kivi_cache_sizes", "kivi_decode_workspace_bytes", "kivi_decode_plan",
    "kivi_quantize_key_groups", "kivi_quantize_value_tokens", "kivi_prefill", "kivi_append_residual",
    "kivi_flush_residual", "kivi_decode_attention", "kivi_decode_step", "kivi_stream_read_probe",
    "kivi_batch_slice", "kivi_decode_step_ragged", "kivi_decode_attention_ragged",
    "kivi_decode_attention_static", "kivi_decode_launches_ragged",
    "kivi_norm_rotate", "kivi_prompt_workspace_bytes", "kivi_prompt_attention", "kivi_paged_sizes",
    "kivi_paged_append", "kivi_paged_attention",
]
KIVI_STATIC_WORKSPACE_BYTES = 8 << 20


class KiviError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


class kivi_layout_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "batch", "n_q_heads", "n_kv_heads", "head_dim", "bits", "group", "residual",
        "cap_q_tokens", "cap_r_tokens", "decode_path")]


class kivi_cache_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in (
        "k_codes", "k_scale", "k_zero", "v_codes", "v_scale", "v_zero", "k_resid", "v_resid")] + \
        [(n, ctypes.c_int32) for n in ("n_kq", "n_vq", "k_r_start", "n_kr", "v_r_start", "n_vr")]


class kivi_seq_state_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_kq", "n_vq", "k_r_start", "n_kr", "v_r_start", "n_vr")]


class kivi_decode_plan_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("family", "launches", "splits_quantised", "splits_fp16",
                                              "tiles_per_split_quantised", "tiles_per_split_fp16",
                                              "units_per_kv_head")]


class kivi_cache_sizes_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_size_t) for n in (
        "k_codes", "k_scale", "k_zero", "v_codes", "v_scale", "v_zero", "k_resid", "v_resid")]


class kivi_tensor_t(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p)] + [(n, ctypes.c_int64) for n in ("stride_b", "stride_h", "stride_t")]


class kivi_rotation_t(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("positions", ctypes.c_void_p)] + \
        [(n, ctypes.c_int32) for n in ("n_positions", "rotary_dim", "interleaved")]


class kivi_norm_rotate_job_t(ctypes.Structure):
    _fields_ = [("src", kivi_tensor_t), ("dst", kivi_tensor_t), ("weight", ctypes.c_void_p), ("weight_offset", ctypes.c_float)] + \
        [(n, ctypes.c_int32) for n in ("n_heads", "src_type", "dst_type")]


class kivi_prompt_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "n_q_heads", "n_kv_heads", "head_dim", "type", "max_q", "max_k")] + \
        [("q_starts", ctypes.c_void_p), ("k_starts", ctypes.c_void_p)] + \
        [(n, ctypes.c_int32) for n in ("q_rows", "k_rows", "window", "sinks")] + [("softmax_scale", ctypes.c_float)]


class kivi_paged_layout_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "max_sequences", "n_q_heads", "n_kv_heads", "head_dim", "bits", "group", "residual",
        "page_tokens", "n_pages", "cap_r_tokens")]


class kivi_paged_cache_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("pages", "k_resid", "v_resid")]


class kivi_paged_sizes_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_size_t) for n in ("pages", "k_resid", "v_resid", "workspace")]


class kivi_paged_batch_t(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("page_table_stride", ctypes.c_int64)] + \
        [(n, ctypes.c_void_p) for n in ("page_table", "lengths", "slots")]


class kivi_paged_rows_t(ctypes.Structure):
    _fields_ = [(n, kivi_tensor_t) for n in ("k", "v", "q", "q_out")] + \
        [(n, ctypes.c_int32) for n in ("type", "n_rows", "max_new")] + \
        [("starts", ctypes.c_void_p), ("rotation", ctypes.POINTER(kivi_rotation_t))]


class kivi_paged_query_t(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("out", ctypes.c_void_p)] + \
        [(n, ctypes.c_int32) for n in ("out_type", "window", "sinks")] + [("softmax_scale", ctypes.c_float)]


_lib: Optional[ctypes.CDLL] = None


def load_library() -> ctypes.CDLL:
    """dlopen libkivi_hip.so (built in-tree by paper_2402_02750_amd/build.py)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it first (python -m paper_2402_02750_amd.build). "
            "There is no fallback path.")
    lib = ctypes.CDLL(LIB_PATH)
    P, I32, I64, VP = ctypes.POINTER, ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
    lib.kivi_status_string.restype = ctypes.c_char_p
    lib.kivi_status_string.argtypes = [ctypes.c_int]
    lib.kivi_cache_sizes.argtypes = [P(kivi_layout_t), P(kivi_cache_sizes_t)]
    lib.kivi_decode_workspace_bytes.argtypes = [P(kivi_layout_t), P(ctypes.c_size_t)]
    lib.kivi_decode_plan.argtypes = [P(kivi_layout_t), P(kivi_cache_t), P(kivi_decode_plan_t)]
    for name in ("kivi_quantize_key_groups", "kivi_quantize_value_tokens"):
        getattr(lib, name).argtypes = [P(kivi_layout_t), VP, I64, I64, I64, I32, P(kivi_cache_t), VP]
    lib.kivi_prefill.argtypes = [P(kivi_layout_t), VP, I64, I64, I64, VP, I64, I64, I64, I32, I32,
                                 P(kivi_cache_t), VP]
    lib.kivi_append_residual.argtypes = [P(kivi_layout_t), P(kivi_cache_t), VP, VP, VP]
    lib.kivi_flush_residual.argtypes = [P(kivi_layout_t), P(kivi_cache_t), I32, P(I32), P(I32), VP]
    lib.kivi_decode_attention.argtypes = [P(kivi_layout_t), P(kivi_cache_t), VP, ctypes.c_float,
                                          VP, VP, ctypes.c_size_t, VP]
    lib.kivi_decode_launches_ragged.argtypes = [P(kivi_layout_t), P(kivi_seq_state_t), P(I32)]
    lib.kivi_decode_attention_static.argtypes = [P(kivi_layout_t), P(kivi_cache_t), VP, ctypes.c_float, VP, VP]
    lib.kivi_decode_step.argtypes = [P(kivi_layout_t), P(kivi_cache_t), VP, VP, VP, ctypes.c_float, I32,
                                     VP, VP, ctypes.c_size_t, VP]
    lib.kivi_stream_read_probe.argtypes = [VP, ctypes.c_size_t, VP, VP]
    lib.kivi_batch_slice.argtypes = [P(kivi_layout_t), P(kivi_cache_t), I32, I32, P(kivi_seq_state_t),
                                     P(kivi_layout_t), P(kivi_cache_t)]
    lib.kivi_decode_step_ragged.argtypes = [P(kivi_layout_t), P(kivi_cache_t), P(kivi_seq_state_t), VP, VP, VP,
                                            ctypes.c_float, I32, VP, VP, ctypes.c_size_t, VP]
    lib.kivi_decode_attention_ragged.argtypes = [P(kivi_layout_t), P(kivi_cache_t), P(kivi_seq_state_t), VP,
                                                 ctypes.c_float, VP, VP, ctypes.c_size_t, VP]
    # (structs by address: byref() of one above, or the same fields packed into bytes, which takes a third of the time)
    lib.kivi_norm_rotate.argtypes = [VP, I32, I32, ctypes.c_float, VP, VP]
    lib.kivi_prompt_workspace_bytes.argtypes = [VP, VP]
    lib.kivi_prompt_attention.argtypes = [VP] * 6 + [ctypes.c_size_t, VP]
    lib.kivi_paged_sizes.argtypes = [VP, VP]
    lib.kivi_paged_append.argtypes = [VP] * 5
    lib.kivi_paged_attention.argtypes = [VP] * 5 + [ctypes.c_size_t, VP]
    for name in EXPORTS[1:]:
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().kivi_status_string(status).decode()


def _check(status: int, where: str):
    if status != KIVI_OK:
        raise KiviError(status, where)


def make_layout(batch, n_q_heads, n_kv_heads, bits, residual, cap_q_tokens, cap_r_tokens,
                head_dim=128, group=32, decode_path=KIVI_DECODE_AUTO) -> kivi_layout_t:
    return kivi_layout_t(batch, n_q_heads, n_kv_heads, head_dim, bits, group, residual,
                         cap_q_tokens, cap_r_tokens, decode_path)


def kivi_cache_sizes(layout: kivi_layout_t) -> kivi_cache_sizes_t:
    sizes = kivi_cache_sizes_t()
    _check(load_library().kivi_cache_sizes(ctypes.byref(layout), ctypes.byref(sizes)), "kivi_cache_sizes")
    return sizes


def kivi_decode_plan(layout: kivi_layout_t, cache) -> kivi_decode_plan_t:
    """How kivi_decode_attention would serve the cache's current state (`cache`: a Cache or kivi_cache_t)."""
    plan = kivi_decode_plan_t()
    c = cache.c if hasattr(cache, "c") else cache
    _check(load_library().kivi_decode_plan(ctypes.byref(layout), ctypes.byref(c), ctypes.byref(plan)), "kivi_decode_plan")
    return plan


def kivi_decode_workspace_bytes(layout: kivi_layout_t) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().kivi_decode_workspace_bytes(ctypes.byref(layout), ctypes.byref(n)),
           "kivi_decode_workspace_bytes")
    return n.value


def _stream_handle(stream, device=None) -> Optional[int]:
    if stream is None:
        import torch
        # (current_stream() takes 2.8 us)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if device is None else device)
    if device is not None and stream.device_index != device:
        raise KiviError(KIVI_ERR_INVALID_ARG, f"stream of cuda:{stream.device_index}, the current device is cuda:{device}")
    return stream.cuda_stream


def _strides_bht(x):
    assert x.dim() == 4 and x.stride(3) == 1, "expected [b, h, t, 128] with contiguous channels"
    return x.stride(0), x.stride(1), x.stride(2)


class Cache:
    """Device buffers (torch tensors) + the kivi_cache_t that points at them."""

    _NAMES = ("k_codes", "k_scale", "k_zero", "v_codes", "v_scale", "v_zero", "k_resid", "v_resid")

    # Optional byte offset between the starts of consecutive arrays inside their allocations (an
    # experiment knob: the decode kernel visits the chunks of different units in different order, so
    # its speed no longer depends on how the arrays are placed relative to each other).
    DEFAULT_SKEW = 0

    def __init__(self, layout: kivi_layout_t, device="cuda", skew=None):
        """`skew` (a multiple of 16 bytes, default DEFAULT_SKEW): the i-th array starts i * skew bytes
        into its allocation."""
        skew = self.DEFAULT_SKEW if skew is None else skew
        import torch
        assert skew % 16 == 0
        self.layout = layout
        sizes = kivi_cache_sizes(layout)
        self.buffers = {}
        self.c = kivi_cache_t()
        for i, name in enumerate(self._NAMES):
            nbytes = max(int(getattr(sizes, name)), 16)
            raw = torch.empty(nbytes + i * skew, dtype=torch.uint8, device=device)
            buf = raw[i * skew:]
            self.buffers[name] = buf
            setattr(self.c, name, buf.data_ptr())
        ws = kivi_decode_workspace_bytes(layout)
        # zero-filled once: the decode kernel keeps its split counters at zero between calls
        self.workspace = torch.zeros(max(ws, 16), dtype=torch.uint8, device=device)

    # convenience typed views (tests compare these against the oracle)
    def view(self, name):
        import torch
        l = self.layout
        units = (l.batch, l.n_kv_heads)
        tiles = l.cap_q_tokens // 32
        buf = self.buffers[name]
        if name in ("k_codes", "v_codes"):
            return buf.view(torch.int32).view(*units, tiles, 32 * 128 * l.bits // 32)
        if name in ("k_scale", "k_zero"):       # one row per group of G tokens
            return buf.view(torch.float16).view(*units, l.cap_q_tokens // l.group, 128)
        if name in ("v_scale", "v_zero"):       # one entry per group of G channels
            return buf.view(torch.float16).view(*units, l.cap_q_tokens, 128 // l.group)
        return buf.view(torch.float16).view(*units, l.cap_r_tokens, 128)


def kivi_quantize_key_groups(layout, k_fp16, n_tokens, cache: Cache, stream=None):
    """k_fp16: CUDA fp16 tensor [b, H_kv, >= n_tokens, 128] (any b/h/t strides)."""
    sb, sh, st = _strides_bht(k_fp16)
    _check(load_library().kivi_quantize_key_groups(
        ctypes.byref(layout), ctypes.c_void_p(k_fp16.data_ptr()), sb, sh, st, n_tokens,
        ctypes.byref(cache.c), _stream_handle(stream)), "kivi_quantize_key_groups")


def kivi_quantize_value_tokens(layout, v_fp16, n_tokens, cache: Cache, stream=None):
    sb, sh, st = _strides_bht(v_fp16)
    _check(load_library().kivi_quantize_value_tokens(
        ctypes.byref(layout), ctypes.c_void_p(v_fp16.data_ptr()), sb, sh, st, n_tokens,
        ctypes.byref(cache.c), _stream_handle(stream)), "kivi_quantize_value_tokens")


def kivi_prefill(layout, k_fp16, v_fp16, n_tokens, cache: Cache, policy=KIVI_FLUSH_WINDOW, stream=None):
    """k_fp16, v_fp16: CUDA fp16 tensors [b, H_kv, >= n_tokens, 128]."""
    ks, vs = _strides_bht(k_fp16), _strides_bht(v_fp16)
    _check(load_library().kivi_prefill(
        ctypes.byref(layout), ctypes.c_void_p(k_fp16.data_ptr()), *ks,
        ctypes.c_void_p(v_fp16.data_ptr()), *vs, n_tokens, policy, ctypes.byref(cache.c),
        _stream_handle(stream)), "kivi_prefill")


def kivi_append_residual(layout, cache: Cache, k_new, v_new, stream=None):
    """k_new, v_new: contiguous CUDA fp16 tensors [b, H_kv, 128]."""
    assert k_new.is_contiguous() and v_new.is_contiguous()
    _check(load_library().kivi_append_residual(
        ctypes.byref(layout), ctypes.byref(cache.c), ctypes.c_void_p(k_new.data_ptr()),
        ctypes.c_void_p(v_new.data_ptr()), _stream_handle(stream)), "kivi_append_residual")


def kivi_flush_residual(layout, cache: Cache, policy=KIVI_FLUSH_WINDOW, stream=None):
    nk, nv = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(load_library().kivi_flush_residual(
        ctypes.byref(layout), ctypes.byref(cache.c), policy, ctypes.byref(nk), ctypes.byref(nv),
        _stream_handle(stream)), "kivi_flush_residual")
    return nk.value, nv.value


def kivi_decode_attention(layout, cache: Cache, q_fp16, softmax_scale, out_fp32, stream=None):
    """q_fp16: contiguous CUDA fp16 [b, H_q, 128]; out_fp32: contiguous CUDA fp32 [b, H_q, 128]."""
    assert q_fp16.is_contiguous() and out_fp32.is_contiguous()
    _check(load_library().kivi_decode_attention(
        ctypes.byref(layout), ctypes.byref(cache.c), ctypes.c_void_p(q_fp16.data_ptr()),
        ctypes.c_float(softmax_scale), ctypes.c_void_p(out_fp32.data_ptr()),
        ctypes.c_void_p(cache.workspace.data_ptr()), cache.workspace.numel(),
        _stream_handle(stream)), "kivi_decode_attention")
    return out_fp32


def kivi_decode_attention_static(layout, cache, q_fp16, softmax_scale, out_fp32, stream=None):
    """kivi_decode_attention on the library's static workspace (no allocation, no workspace argument)."""
    assert q_fp16.is_contiguous() and out_fp32.is_contiguous()
    _check(load_library().kivi_decode_attention_static(
        ctypes.byref(layout), ctypes.byref(cache.c), ctypes.c_void_p(q_fp16.data_ptr()),
        ctypes.c_float(softmax_scale), ctypes.c_void_p(out_fp32.data_ptr()), _stream_handle(stream)),
        "kivi_decode_attention_static")
    return out_fp32


def kivi_decode_step(layout, cache: Cache, k_new, v_new, q_fp16, softmax_scale, out_fp32,
                     policy=KIVI_FLUSH_WINDOW, stream=None):
    """Append + flush + attention of one decoding step.  k_new, v_new: contiguous CUDA fp16
    [b, H_kv, 128] (keep them alive until the launch has run); q_fp16 / out_fp32 as for
    kivi_decode_attention."""
    assert k_new.is_contiguous() and v_new.is_contiguous()
    assert q_fp16.is_contiguous() and out_fp32.is_contiguous()
    _check(load_library().kivi_decode_step(
        ctypes.byref(layout), ctypes.byref(cache.c), ctypes.c_void_p(k_new.data_ptr()),
        ctypes.c_void_p(v_new.data_ptr()), ctypes.c_void_p(q_fp16.data_ptr()),
        ctypes.c_float(softmax_scale), policy, ctypes.c_void_p(out_fp32.data_ptr()),
        ctypes.c_void_p(cache.workspace.data_ptr()), cache.workspace.numel(),
        _stream_handle(stream)), "kivi_decode_step")
    return out_fp32


def kivi_stream_read_probe(src, sink, stream=None):
    """Measurement helper: plain read-only stream over the CUDA tensor `src` (any dtype, contiguous,
    a multiple of 16 bytes); `sink`: CUDA tensor of at least 16 KiB."""
    assert src.is_contiguous() and sink.numel() * sink.element_size() >= 4096 * 4
    _check(load_library().kivi_stream_read_probe(
        ctypes.c_void_p(src.data_ptr()), src.numel() * src.element_size(), ctypes.c_void_p(sink.data_ptr()),
        _stream_handle(stream)), "kivi_stream_read_probe")


class CacheSlice:
    """Batch entries [b0, b0 + nb) of a Cache as a cache of their own (kivi_batch_slice): `layout`
    and `c` can be passed to every entry point, e.g. to prefill one sequence of a ragged batch."""

    def __init__(self, cache: Cache, b0: int, nb: int, state=None):
        self.parent = cache
        self.layout = kivi_layout_t()
        self.c = kivi_cache_t()
        self.workspace = cache.workspace
        _check(load_library().kivi_batch_slice(
            ctypes.byref(cache.layout), ctypes.byref(cache.c), b0, nb,
            ctypes.byref(state) if state is not None else None,
            ctypes.byref(self.layout), ctypes.byref(self.c)), "kivi_batch_slice")

    def state(self) -> kivi_seq_state_t:
        return kivi_seq_state_t(self.c.n_kq, self.c.n_vq, self.c.k_r_start, self.c.n_kr, self.c.v_r_start, self.c.n_vr)


def make_states(batch: int):
    """Host array of per-sequence states (all empty) for the ragged entry points."""
    return (kivi_seq_state_t * batch)()


def kivi_decode_step_ragged(layout, cache: Cache, states, k_new, v_new, q_fp16, softmax_scale, out_fp32,
                            policy=KIVI_FLUSH_WINDOW, stream=None):
    """kivi_decode_step over a batch whose sequences differ in length; `states` from make_states."""
    assert k_new.is_contiguous() and v_new.is_contiguous() and q_fp16.is_contiguous() and out_fp32.is_contiguous()
    _check(load_library().kivi_decode_step_ragged(
        ctypes.byref(layout), ctypes.byref(cache.c), states, ctypes.c_void_p(k_new.data_ptr()),
        ctypes.c_void_p(v_new.data_ptr()), ctypes.c_void_p(q_fp16.data_ptr()), ctypes.c_float(softmax_scale),
        policy, ctypes.c_void_p(out_fp32.data_ptr()), ctypes.c_void_p(cache.workspace.data_ptr()),
        cache.workspace.numel(), _stream_handle(stream)), "kivi_decode_step_ragged")
    return out_fp32


def kivi_decode_launches_ragged(layout, states) -> int:
    """Kernel launches kivi_decode_attention_ragged would enqueue for these sequence states."""
    n = ctypes.c_int32(0)
    _check(load_library().kivi_decode_launches_ragged(ctypes.byref(layout), states, ctypes.byref(n)),
           "kivi_decode_launches_ragged")
    return n.value


def kivi_decode_attention_ragged(layout, cache: Cache, states, q_fp16, softmax_scale, out_fp32, stream=None):
    assert q_fp16.is_contiguous() and out_fp32.is_contiguous()
    _check(load_library().kivi_decode_attention_ragged(
        ctypes.byref(layout), ctypes.byref(cache.c), states, ctypes.c_void_p(q_fp16.data_ptr()),
        ctypes.c_float(softmax_scale), ctypes.c_void_p(out_fp32.data_ptr()),
        ctypes.c_void_p(cache.workspace.data_ptr()), cache.workspace.numel(), _stream_handle(stream)),
        "kivi_decode_attention_ragged")
    return out_fp32


# ---- operators around the cache ----
# Single-token calls take as long as their binding, so these pack the structs' fields directly.

_TENSOR = "Pqqq"
_NO_TENSOR = (0, 0, 0, 0)
_JOB = struct.Struct(_TENSOR * 2 + "Pfiii")
_TWO_JOBS = struct.Struct((_TENSOR * 2 + "Pfiii") * 2)
_ONE_TENSOR = struct.Struct(_TENSOR)
_PROMPT = struct.Struct("iiiiiii4xPPiiiif4x")
_ROWS = struct.Struct(_TENSOR * 4 + "iii4xPP")
_QUERY = struct.Struct("PPiiif")
_ROTATION = struct.Struct("PPiii4x")


_kinds = {}                          # KIVI_TYPE_* by torch type


def _type_of(x) -> int:
    kind = _kinds.get(x.dtype)
    if kind is None:
        import torch
        _kinds.update({torch.float16: KIVI_TYPE_FP16, torch.bfloat16: KIVI_TYPE_BF16})
        if x.dtype not in _kinds:
            raise KiviError(KIVI_ERR_UNSUPPORTED, f"tensor of {x.dtype}")
        return _kinds[x.dtype]
    return kind


def _on_device(*tensors) -> int:
    """All tensors on the current device, which is returned: its stream and launches are the ones the library uses."""
    import torch
    here = torch.cuda.current_device()
    for x in tensors:
        if x is not None and x.get_device() != here:
            raise KiviError(KIVI_ERR_INVALID_ARG, f"tensor on {x.device}, the current device is cuda:{here}")
    return here


def _rows(x, shape):
    """A tensor of this shape, [rows, heads, 128] (any row and head strides), as the fields of a kivi_tensor_t."""
    st, sh, sd = x.stride()
    assert x.shape == shape and sd == 1, f"expected {list(shape)} with contiguous channels"
    return x.data_ptr(), 0, sh, st


def _int32(x, n=None):
    """Device pointer of a contiguous int32 tensor (None: null)."""
    if x is None:
        return None
    import torch
    assert x.dtype is torch.int32 and x.is_contiguous() and (n is None or x.numel() >= n), "expected a contiguous int32 tensor"
    return x.data_ptr()


class Rotation:
    """A table of cosines and sines for the position rotation: CUDA fp32 [n_positions, rotary_dim], the cosines of the
    rotary_dim / 2 channel pairs first.  interleaved: pairs are neighbouring channels."""

    def __init__(self, table, interleaved=False):
        import torch
        assert table.dim() == 2 and table.dtype == torch.float32 and table.is_contiguous(), "expected a contiguous fp32 table"
        self.table = table
        self.interleaved = int(interleaved)
        self._fields = table.data_ptr(), *table.shape, self.interleaved
        self._alone = self.c()

    def c(self, positions=None, rows=0) -> kivi_rotation_t:
        if positions is None and hasattr(self, "_alone"):
            return self._alone
        return kivi_rotation_t(self.table.data_ptr(), _int32(positions, rows), self.table.shape[0], self.table.shape[1], self.interleaved)


def _weight(w, x):
    if w is None:
        return 0
    assert w.dtype is x.dtype and w.numel() == 128 and w.is_contiguous(), "expected a weight [128] of the tensor's type"
    return w.data_ptr()


def kivi_norm_rotate(q, q_out, k=None, k_out=None, q_weight=None, k_weight=None, eps=1e-6, weight_offset=0.0,
                     rotation: Optional[Rotation] = None, positions=None, stream=None):
    """q, k: CUDA fp16 / bf16 [rows, heads, 128] (any row and head strides); q_out, k_out the same shapes, fp16 or bf16, maybe q
    and k themselves; weights: [128] in the type of q / k, or None (no norm); positions: int32 [rows]."""
    here = _on_device(q, q_out, k, k_out, q_weight, k_weight, positions, rotation.table if rotation else None)
    rows, heads, _ = q.shape
    shape = rows, heads, 128
    job = (*_rows(q, shape), *_rows(q_out, shape), _weight(q_weight, q), weight_offset, heads, _type_of(q), _type_of(q_out))
    if k is None:
        n, jobs = 1, _JOB.pack(*job)
    else:
        heads = k.shape[1]
        shape = rows, heads, 128
        n, jobs = 2, _TWO_JOBS.pack(*job, *_rows(k, shape), *_rows(k_out, shape), _weight(k_weight, k), weight_offset, heads,
                                    _type_of(k), _type_of(k_out))
    r = None
    if rotation is not None:
        assert positions is not None, "a rotation needs positions"
        table, *rest = rotation._fields
        r = _ROTATION.pack(table, _int32(positions, rows) or 0, *rest)
    _check(load_library().kivi_norm_rotate(jobs, n, rows, eps, r, _stream_handle(stream, here)), "kivi_norm_rotate")


def kivi_prompt_attention(q, k, v, out, softmax_scale, q_starts=None, k_starts=None, max_q=None, max_k=None, window=0, sinks=0, stream=None):
    """Either q, out [b, H_q, n_q, 128] and k, v [b, H_kv, n_k, 128] (any strides), or, with q_starts and k_starts (int32
    [b + 1]), rows of sequences one after the other: q, out [rows, H_q, 128], k, v [rows, H_kv, 128] and max_q, max_k the longest
    sequence's.  fp16 or bf16, all alike."""
    here = _on_device(q, k, v, out, q_starts, k_starts)
    kind = _type_of(q)
    assert _type_of(k) == _type_of(v) == _type_of(out) == kind, "q, k, v and out have one type"
    if q_starts is not None:
        assert k_starts is not None and max_q is not None and max_k is not None, "both starts, and the longest sequence's lengths"
        batch = q_starts.numel() - 1
        q_rows, heads, _ = q.shape
        k_rows, kv_heads, _ = k.shape
        p = _PROMPT.pack(batch, heads, kv_heads, 128, kind, max_q, max_k, _int32(q_starts), _int32(k_starts, batch + 1), q_rows, k_rows, window, sinks,
                         softmax_scale)
        q_shape, k_shape = (q_rows, heads, 128), (k_rows, kv_heads, 128)
        tensors = _rows(q, q_shape), _rows(k, k_shape), _rows(v, k_shape), _rows(out, q_shape)
    else:
        assert k_starts is None and out.shape == q.shape and v.shape == k.shape, "out is shaped like q, v like k"
        batch, heads, max_q, d = q.shape
        assert k.shape[0] == batch and k.shape[3] == d == 128, "expected [b, h, t, 128]"
        p = _PROMPT.pack(batch, heads, k.shape[1], 128, kind, max_q, k.shape[2], 0, 0, 0, 0, window, sinks, softmax_scale)
        tensors = [(x.data_ptr(), *_strides_bht(x)) for x in (q, k, v, out)]
    lib = load_library()
    need = ctypes.c_size_t(0)
    _check(lib.kivi_prompt_workspace_bytes(p, ctypes.byref(need)), "kivi_prompt_workspace_bytes")
    workspace = None
    if need.value:
        import torch
        with torch.cuda.stream(stream):                 # (the allocator orders its reuse by this stream)
            workspace = torch.empty(need.value, dtype=torch.uint8, device=q.device)
    _check(lib.kivi_prompt_attention(p, *[_ONE_TENSOR.pack(*t) for t in tensors], workspace.data_ptr() if need.value else None, need.value,
                                     _stream_handle(stream, here)), "kivi_prompt_attention")
    return out


def make_paged_layout(max_sequences, n_q_heads, n_kv_heads, bits, residual, page_tokens, n_pages, cap_r_tokens, head_dim=128, group=32) -> kivi_paged_layout_t:
    return kivi_paged_layout_t(max_sequences, n_q_heads, n_kv_heads, head_dim, bits, group, residual, page_tokens, n_pages, cap_r_tokens)


def kivi_paged_sizes(layout: kivi_paged_layout_t) -> kivi_paged_sizes_t:
    sizes = kivi_paged_sizes_t()
    _check(load_library().kivi_paged_sizes(ctypes.byref(layout), ctypes.byref(sizes)), "kivi_paged_sizes")
    return sizes


class PagedCache:
    """Device buffers of a paged cache (or the caller's own: contiguous CUDA tensors of at least those sizes) and the workspace of
    its attention.  Calls of kivi_paged_attention that may overlap need a PagedCache each, over the same buffers."""

    def __init__(self, layout: kivi_paged_layout_t, device="cuda", pages=None, k_resid=None, v_resid=None):
        import torch
        self.layout = layout
        sizes = kivi_paged_sizes(layout)
        self.c = kivi_paged_cache_t()
        self.buffers = {}
        for name, given in (("pages", pages), ("k_resid", k_resid), ("v_resid", v_resid)):
            n = getattr(sizes, name)
            if given is None:
                given = torch.empty(n, dtype=torch.uint8, device=device)
            assert given.is_cuda and given.is_contiguous() and given.numel() * given.element_size() >= n, f"{name}: {n} contiguous bytes"
            self.buffers[name] = given
            setattr(self.c, name, given.data_ptr())
        devices = {x.device for x in self.buffers.values()}
        assert len(devices) == 1, "one device"
        self.workspace = torch.zeros(sizes.workspace, dtype=torch.uint8, device=devices.pop())
        self._refs = ctypes.byref(self.layout), ctypes.byref(self.c)
        self._workspace = self.workspace.data_ptr(), self.workspace.numel()

    def records(self):
        """The pages as int32 words [n_pages, H_kv, records per page, words of a record]."""
        import torch
        l = self.layout
        return self.buffers["pages"].view(torch.uint8).flatten()[:kivi_paged_sizes(l).pages].view(torch.int32).view(
            l.n_pages, l.n_kv_heads, l.page_tokens // 32, -1)

    def rows(self, name):
        """k_resid or v_resid as fp16 [max_sequences, H_kv, cap_r, 128]."""
        import torch
        l = self.layout
        return self.buffers[name].view(torch.uint8).flatten()[:kivi_paged_sizes(l).k_resid].view(torch.float16).view(
            l.max_sequences, l.n_kv_heads, l.cap_r_tokens, 128)


class PagedBatch:
    """The sequences of a call: page_table int32 [b, max_pages] (rows may be strided), lengths int32 [b], slots int32 [b] or None.  The
    tensors are kept, not copied: what they hold when a call runs is what counts."""

    def __init__(self, page_table, lengths, slots=None):
        import torch
        n = lengths.numel()
        assert page_table.dim() == 2 and page_table.shape[0] == n and page_table.dtype == torch.int32 and (page_table.shape[1] < 2 or page_table.stride(1) == 1)
        assert n == 1 or page_table.stride(0) >= page_table.shape[1], "rows of the page table must not overlap"
        assert page_table.device == lengths.device and (slots is None or slots.device == lengths.device), "one device"
        self.page_table, self.lengths, self.slots = page_table, lengths, slots
        self.size = n
        self.c = kivi_paged_batch_t(n, page_table.shape[1], max(page_table.stride(0), page_table.shape[1]), page_table.data_ptr(),
                                    _int32(lengths), _int32(slots, n))
        self._ref = ctypes.byref(self.c)


def kivi_paged_append(cache: PagedCache, batch: PagedBatch, k, v, starts=None, max_new=1, rotation: Optional[Rotation] = None, positions=None,
                      q=None, q_out=None, stream=None):
    """k, v: CUDA fp16 / bf16 [rows, H_kv, 128] (any row and head strides), the new rows of all sequences: those of
    sequence b are rows starts[b] .. starts[b + 1] - 1 (int32 [b + 1]), or max_new of each without starts.  batch.lengths counts them
    already.  q [rows, H_q, 128] is rotated into q_out (fp16)."""
    here = _on_device(k, v, starts, positions, q, q_out, batch.lengths, cache.workspace, rotation.table if rotation else None)
    l, n = cache.layout, k.shape[0]
    shape = n, l.n_kv_heads, 128
    assert v.dtype is k.dtype, "k, v and q have one type"
    qs = _NO_TENSOR * 2
    if q is not None:
        assert q.dtype is k.dtype and _type_of(q_out) == KIVI_TYPE_FP16, "q has the type of k, q_out is fp16"
        q_shape = n, l.n_q_heads, 128
        qs = (*_rows(q, q_shape), *_rows(q_out, q_shape))
    else:
        assert q_out is None, "q_out without q"
    r, at = None, 0
    if rotation is not None:
        r = rotation.c(positions, n)
        at = ctypes.addressof(r)
    rows = _ROWS.pack(*_rows(k, shape), *_rows(v, shape), *qs, _type_of(k), n, max_new, _int32(starts, batch.size + 1) or 0, at)
    _check(load_library().kivi_paged_append(*cache._refs, batch._ref, rows, _stream_handle(stream, here)), "kivi_paged_append")


def kivi_paged_attention(cache: PagedCache, batch: PagedBatch, q_fp16, softmax_scale, out, window=0, sinks=0, stream=None):
    """q_fp16: contiguous CUDA fp16 [b, H_q, 128]; out: the same shape, contiguous, fp16 or bf16."""
    here = _on_device(q_fp16, out, batch.lengths, cache.workspace)
    assert _type_of(q_fp16) == KIVI_TYPE_FP16 and q_fp16.is_contiguous() and out.is_contiguous(), "q is fp16; q and out are contiguous"
    shape = q_fp16.shape
    assert shape == out.shape and shape == (batch.size, cache.layout.n_q_heads, 128), "q and out are [b, H_q, 128]"
    query = _QUERY.pack(q_fp16.data_ptr(), out.data_ptr(), _type_of(out), window, sinks, softmax_scale)
    _check(load_library().kivi_paged_attention(*cache._refs, batch._ref, query, *cache._workspace, _stream_handle(stream, here)), "kivi_paged_attention")
    return out
