"""ctypes binding of libpevlm.so: same names as the C entry points, argument marshalling only.

Tensors are torch tensors in device memory (torch is used to allocate memory and to name the
stream); their data pointers go straight to the C ABI.  Descriptor arrays stay on the host.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libpevlm.so")

PEVLM_OK, PEVLM_ERR_INVALID_ARG, PEVLM_ERR_UNSUPPORTED, PEVLM_ERR_WORKSPACE_TOO_SMALL, PEVLM_ERR_HIP = range(5)
PEVLM_F32, PEVLM_BF16 = 0, 1
PEVLM_MAX_SPLITS = 64


class PevlmError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"pevlm status {status}: {message}")
        self.status = status


class _CLayout(ctypes.Structure):
    _fields_ = [("num_seqs", ctypes.c_int32)] + [
        (n, ctypes.POINTER(ctypes.c_int32)) for n in ("cu_seqlens", "sink_len", "block_len", "ctx_len", "query_len")]


class _CHeads(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("kv_head_of_q", ctypes.POINTER(ctypes.c_int32)), ("dtype", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float)]


class _CCache(ctypes.Structure):
    _fields_ = [("pool", ctypes.c_void_p), ("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("num_seqs", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("block_table", ctypes.c_void_p)]


class WorkItem(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("q_start", "q_rows", "full_start", "full_len", "diag_start",
                                              "diag_len", "seq", "reserved")]


class _StreamSlot(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("q_start", "q_rows", "head", "reserved")]


class StreamItem(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("full_start", "full_len", "diag_start", "diag_len", "kv_head",
                                              "n_full_tiles", "n_tiles", "seq")] + [("slot", _StreamSlot * 8)]


class Fp8Plan(ctypes.Structure):
    _fields_ = [("n_items", ctypes.c_int64), ("n_key_tiles", ctypes.c_int64)] + \
               [(n, ctypes.c_size_t) for n in ("items", "key_tiles", "kv_amax", "q_scales", "q_codes", "k_tiles", "v_tiles", "total")]


_lib = None


def lib_path() -> str:
    return _LIB_PATH


def load_library():
    """Loads libpevlm.so.  Raises if it has not been built: there is no other path."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'` "
                              "(or paper_2506_19651_amd/build.py) first; there is no fallback path")
        lib = ctypes.CDLL(_LIB_PATH)
        vp, i32, f32p = ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p
        LP, HP = ctypes.POINTER(_CLayout), ctypes.POINTER(_CHeads)
        lib.pevlm_rope_seq.restype = ctypes.c_int
        lib.pevlm_rope_seq.argtypes = [vp, vp, LP, HP, ctypes.c_double, vp, vp]
        lib.pevlm_block_prefill_workspace_bytes.restype = ctypes.c_size_t
        lib.pevlm_block_prefill_workspace_bytes.argtypes = [LP, HP]
        lib.pevlm_block_prefill_attn.restype = ctypes.c_int
        lib.pevlm_block_prefill_attn.argtypes = [vp, vp, vp, vp, f32p, LP, HP, vp, ctypes.c_size_t, vp]
        lib.pevlm_query_workspace_bytes.restype = ctypes.c_size_t
        lib.pevlm_query_workspace_bytes.argtypes = [LP, HP, i32]
        lib.pevlm_query_attn.restype = ctypes.c_int
        lib.pevlm_query_attn.argtypes = [vp, vp, vp, vp, f32p, LP, HP, i32, vp, ctypes.c_size_t, vp]
        lib.pevlm_query_attn_static.restype = ctypes.c_int
        lib.pevlm_query_attn_static.argtypes = [vp, vp, vp, vp, f32p, LP, HP, i32, vp]
        lib.pevlm_block_prefill_rope_workspace_bytes.restype = ctypes.c_size_t
        lib.pevlm_block_prefill_rope_workspace_bytes.argtypes = [LP, HP]
        lib.pevlm_block_prefill_attn_rope.restype = ctypes.c_int
        lib.pevlm_block_prefill_attn_rope.argtypes = [vp, vp, vp, vp, f32p, LP, HP, ctypes.c_double, vp, i32, vp, ctypes.c_size_t, vp]
        lib.pevlm_query_rope_workspace_bytes.restype = ctypes.c_size_t
        lib.pevlm_query_rope_workspace_bytes.argtypes = [LP, HP, i32]
        lib.pevlm_query_attn_rope.restype = ctypes.c_int
        lib.pevlm_query_attn_rope.argtypes = [vp, vp, vp, vp, f32p, LP, HP, i32, ctypes.c_double, vp, vp, ctypes.c_size_t, vp]
        i32p = ctypes.POINTER(ctypes.c_int32)
        lib.pevlm_block_prefill_attn_blocks.restype = ctypes.c_int
        lib.pevlm_block_prefill_attn_blocks.argtypes = [vp, vp, vp, vp, f32p, LP, HP, i32p, i32p, i32, vp, ctypes.c_size_t, vp]
        lib.pevlm_query_window_workspace_bytes.restype = ctypes.c_size_t
        lib.pevlm_query_window_workspace_bytes.argtypes = [LP, HP, i32]
        lib.pevlm_query_attn_window.restype = ctypes.c_int
        lib.pevlm_query_attn_window.argtypes = [vp, vp, vp, vp, f32p, LP, HP, i32p, i32, vp, ctypes.c_size_t, vp]
        lib.pevlm_prefill_worklist_blocks_host.restype = ctypes.c_int64
        lib.pevlm_prefill_worklist_blocks_host.argtypes = [LP, i32, i32p, i32p, i32, ctypes.POINTER(WorkItem), ctypes.c_int64]
        lib.pevlm_query_worklist_window_host.restype = ctypes.c_int64
        lib.pevlm_query_worklist_window_host.argtypes = [LP, i32, i32, i32p, ctypes.POINTER(WorkItem), ctypes.c_int64]
        lib.pevlm_block_prefill_attn_mrope.restype = ctypes.c_int
        lib.pevlm_block_prefill_attn_mrope.argtypes = [vp, vp, vp, vp, f32p, LP, HP, ctypes.c_double, vp, i32p, i32, vp,
                                                       ctypes.c_size_t, vp]
        lib.pevlm_query_attn_mrope.restype = ctypes.c_int
        lib.pevlm_query_attn_mrope.argtypes = [vp, vp, vp, vp, f32p, LP, HP, i32, ctypes.c_double, vp, i32p, vp, ctypes.c_size_t, vp]
        lib.pevlm_block_prefill_fp8_plan.restype = ctypes.c_int
        lib.pevlm_block_prefill_fp8_plan.argtypes = [LP, HP, ctypes.POINTER(Fp8Plan)]
        lib.pevlm_block_prefill_fp8_workspace_bytes.restype = ctypes.c_size_t
        lib.pevlm_block_prefill_fp8_workspace_bytes.argtypes = [LP, HP]
        lib.pevlm_block_prefill_attn_fp8.restype = ctypes.c_int
        lib.pevlm_block_prefill_attn_fp8.argtypes = [vp, vp, vp, vp, f32p, LP, HP, vp, ctypes.c_size_t, i32, vp]
        lib.pevlm_last_error.restype = ctypes.c_char_p
        lib.pevlm_version.restype = i32
        lib.pevlm_prefill_tile_rows.restype = i32
        lib.pevlm_prefill_tile_rows.argtypes = [HP]
        lib.pevlm_query_tile_rows.restype = i32
        lib.pevlm_query_tile_rows.argtypes = [HP]
        lib.pevlm_prefill_uses_stream_kernel.restype = ctypes.c_int32
        lib.pevlm_prefill_uses_stream_kernel.argtypes = [LP, HP]
        lib.pevlm_set_prefill_kernel.restype = ctypes.c_int32
        lib.pevlm_set_prefill_kernel.argtypes = [i32]
        lib.pevlm_prefill_stream_items_host.restype = ctypes.c_int64
        lib.pevlm_prefill_stream_items_host.argtypes = [LP, HP, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32), i32,
                                                        ctypes.POINTER(StreamItem), ctypes.c_int64]
        lib.pevlm_prefill_worklist_host.restype = ctypes.c_int64
        lib.pevlm_prefill_worklist_host.argtypes = [LP, i32, ctypes.POINTER(WorkItem), ctypes.c_int64]
        lib.pevlm_query_worklist_host.restype = ctypes.c_int64
        lib.pevlm_query_worklist_host.argtypes = [LP, i32, i32, ctypes.POINTER(WorkItem), ctypes.c_int64]
        lib.pevlm_rope_mrope.restype = ctypes.c_int
        lib.pevlm_rope_mrope.argtypes = [vp, vp, ctypes.c_int64, HP, ctypes.c_double, vp, ctypes.POINTER(ctypes.c_int32), vp]
        lib.pevlm_probe_mfma_bf16.restype = ctypes.c_int
        lib.pevlm_probe_mfma_bf16.argtypes = [vp, i32, i32, ctypes.POINTER(ctypes.c_double), vp]
        lib.pevlm_probe_tile_loop_bf16.restype = ctypes.c_int
        lib.pevlm_probe_tile_loop_bf16.argtypes = [vp, vp, ctypes.c_size_t, i32, i32, i32, ctypes.POINTER(ctypes.c_double), vp]
        lib.pevlm_probe_copy.restype = ctypes.c_int
        lib.pevlm_probe_copy.argtypes = [vp, vp, ctypes.c_size_t, vp]
        CP, i64, size_t = ctypes.POINTER(_CCache), ctypes.c_int64, ctypes.c_size_t
        lib.pevlm_cache_pool_bytes.restype = size_t
        lib.pevlm_cache_pool_bytes.argtypes = [HP, i32, i32]
        lib.pevlm_cache_slots_workspace_bytes.restype = size_t
        lib.pevlm_cache_slots_workspace_bytes.argtypes = [i32]
        lib.pevlm_cache_slots.restype = ctypes.c_int
        lib.pevlm_cache_slots.argtypes = [CP, vp, vp, vp, i32, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, size_t, vp]
        for fn in (lib.pevlm_cache_store_kv4, lib.pevlm_cache_load_kv4):
            fn.restype = ctypes.c_int
            fn.argtypes = [vp, vp, i64, i64, vp, i32, CP, HP, vp]
        lib.pevlm_cache_attn_workspace_bytes.restype = size_t
        lib.pevlm_cache_attn_workspace_bytes.argtypes = [HP, i32, i32]
        lib.pevlm_cache_attn_kv4.restype = ctypes.c_int
        lib.pevlm_cache_attn_kv4.argtypes = [vp, vp, vp, CP, HP, i32, vp, vp, vp, vp, vp, vp, size_t, vp]
        lib.pevlm_visible_pairs.restype = ctypes.c_int
        lib.pevlm_visible_pairs.argtypes = [LP] + [ctypes.POINTER(ctypes.c_int64)] * 3
        _lib = lib
    return _lib


def _i32p(a: np.ndarray):
    return a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


class Layout:
    """Host-side partition descriptor: per sequence sink S, block length B, context length C,
    question length Q; sequences are packed back to back (cu_seqlens)."""

    def __init__(self, cu_seqlens: Sequence[int], sink_len, block_len, ctx_len, query_len):
        self.cu = np.ascontiguousarray(cu_seqlens, dtype=np.int32)
        self.s = np.ascontiguousarray(sink_len, dtype=np.int32)
        self.b = np.ascontiguousarray(block_len, dtype=np.int32)
        self.c = np.ascontiguousarray(ctx_len, dtype=np.int32)
        self.q = np.ascontiguousarray(query_len, dtype=np.int32)
        self.struct = _CLayout(len(self.s), _i32p(self.cu), _i32p(self.s), _i32p(self.b), _i32p(self.c), _i32p(self.q))

    @classmethod
    def from_seqs(cls, seqs):
        a = np.asarray(seqs, dtype=np.int64).reshape(-1, 4)
        cu = np.concatenate([[0], np.cumsum(a[:, 0] + a[:, 2] + a[:, 3])])
        return cls(cu, a[:, 0], a[:, 1], a[:, 2], a[:, 3])

    @property
    def total_tokens(self) -> int:
        return int(self.cu[-1]) if len(self.cu) else 0

    def ref(self):
        return ctypes.byref(self.struct)


class Heads:
    def __init__(self, n_q_heads: int, n_kv_heads: int, head_dim: int, dtype: str,
                 kv_head_of_q: Optional[Sequence[int]] = None, softmax_scale: float = 0.0):
        self.map = None if kv_head_of_q is None else np.ascontiguousarray(kv_head_of_q, dtype=np.int32)
        code = {"f32": PEVLM_F32, "bf16": PEVLM_BF16}.get(dtype, dtype)
        self.struct = _CHeads(n_q_heads, n_kv_heads, head_dim, None if self.map is None else _i32p(self.map),
                              int(code), float(softmax_scale))
        self.n_q_heads, self.n_kv_heads, self.head_dim, self.dtype = n_q_heads, n_kv_heads, head_dim, dtype

    def ref(self):
        return ctypes.byref(self.struct)


def _check(status: int):
    if status != PEVLM_OK:
        raise PevlmError(status, pevlm_last_error())


def _ptr(t):
    """Address of a tensor (anything with data_ptr()) or an integer address, as the C calls take it."""
    if t is None:
        return None
    return t.data_ptr() if hasattr(t, "data_ptr") else int(t)


_current_raw_stream = None


def _find_current_raw_stream():
    """() -> hipStream_t of torch's current stream on the current device.  torch.cuda.current_stream() builds a
    stream object (2.9 us, as long as a kernel launch takes); where torch offers the bare handle (0.3 us)
    that is asked for instead."""
    import torch

    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        return lambda: torch.cuda.current_stream().cuda_stream
    device = torch.cuda.current_device
    return lambda: raw(device())


def _stream_ptr(stream):
    global _current_raw_stream
    if stream is None:
        if _current_raw_stream is None:
            _current_raw_stream = _find_current_raw_stream()
        return _current_raw_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _workspace(nbytes: int, like):
    import torch
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=like.device)


def pevlm_last_error() -> str:
    return load_library().pevlm_last_error().decode()


def pevlm_probe_mfma_bf16(scratch, workgroups: int, iters: int, stream=None) -> float:
    """Enqueues the register-resident bf16 MFMA loop; returns the floating-point operations of the launch."""
    flops = ctypes.c_double(0.0)
    _check(load_library().pevlm_probe_mfma_bf16(_ptr(scratch), int(workgroups), int(iters), ctypes.byref(flops), _stream_ptr(stream)))
    return float(flops.value)


def pevlm_probe_tile_loop_bf16(scratch, kv, workgroups: int, iters: int, with_softmax: bool = True, stream=None) -> float:
    """Enqueues the tile-loop probe on `kv` (a device tensor of finite bf16 data); returns the FLOPs of its MFMAs."""
    flops = ctypes.c_double(0.0)
    _check(load_library().pevlm_probe_tile_loop_bf16(_ptr(scratch), _ptr(kv), int(kv.numel() * kv.element_size()), int(workgroups),
                                                     int(iters), int(bool(with_softmax)), ctypes.byref(flops), _stream_ptr(stream)))
    return float(flops.value)


def pevlm_probe_copy(dst, src, nbytes: int, stream=None) -> None:
    _check(load_library().pevlm_probe_copy(_ptr(dst), _ptr(src), int(nbytes), _stream_ptr(stream)))


def pevlm_version() -> int:
    return int(load_library().pevlm_version())


def pevlm_prefill_tile_rows(heads: "Heads") -> int:
    return int(load_library().pevlm_prefill_tile_rows(heads.ref()))


def pevlm_query_tile_rows(heads: "Heads") -> int:
    return int(load_library().pevlm_query_tile_rows(heads.ref()))


def pevlm_rope_seq(q, k, layout: Layout, heads: Heads, rope_base: float, pos_offset=None, stream=None):
    _off, offp = _offsets(pos_offset)
    _check(load_library().pevlm_rope_seq(_ptr(q), _ptr(k), layout.ref(), heads.ref(), float(rope_base), offp,
                                         _stream_ptr(stream)))


def _offsets(pos_offset):
    return (None, None) if pos_offset is None else _i32_array(pos_offset)


def pevlm_block_prefill_rope_workspace_bytes(layout: Layout, heads: Heads) -> int:
    return int(load_library().pevlm_block_prefill_rope_workspace_bytes(layout.ref(), heads.ref()))


def pevlm_block_prefill_attn_rope(q, k, v, out, layout: Layout, heads: Heads, rope_base: float, pos_offset=None,
                                  k_is_rotated: bool = False, lse=None, workspace=None, stream=None):
    if workspace is None:
        workspace = _workspace(pevlm_block_prefill_rope_workspace_bytes(layout, heads), q)
    _off, offp = _offsets(pos_offset)
    _check(load_library().pevlm_block_prefill_attn_rope(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), layout.ref(),
                                                        heads.ref(), float(rope_base), offp, int(bool(k_is_rotated)),
                                                        _ptr(workspace), workspace.numel(), _stream_ptr(stream)))


def pevlm_query_rope_workspace_bytes(layout: Layout, heads: Heads, num_splits: int = 0) -> int:
    return int(load_library().pevlm_query_rope_workspace_bytes(layout.ref(), heads.ref(), int(num_splits)))


def pevlm_query_attn_rope(q, k, v, out, layout: Layout, heads: Heads, rope_base: float, pos_offset=None, num_splits: int = 0,
                          lse=None, workspace=None, stream=None):
    if workspace is None:
        workspace = _workspace(pevlm_query_rope_workspace_bytes(layout, heads, num_splits), q)
    _off, offp = _offsets(pos_offset)
    _check(load_library().pevlm_query_attn_rope(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), layout.ref(), heads.ref(),
                                                int(num_splits), float(rope_base), offp, _ptr(workspace),
                                                workspace.numel(), _stream_ptr(stream)))


def pevlm_block_prefill_attn_mrope(q, k, v, out, layout: Layout, heads: Heads, rope_base: float, pos_ids, section,
                                   k_is_rotated: bool = False, lse=None, workspace=None, stream=None):
    if workspace is None:
        workspace = _workspace(pevlm_block_prefill_rope_workspace_bytes(layout, heads), q)
    _s, sp = _i32_array(section)
    _check(load_library().pevlm_block_prefill_attn_mrope(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), layout.ref(),
                                                         heads.ref(), float(rope_base), _ptr(pos_ids), sp,
                                                         int(bool(k_is_rotated)), _ptr(workspace), workspace.numel(),
                                                         _stream_ptr(stream)))


def pevlm_query_attn_mrope(q, k, v, out, layout: Layout, heads: Heads, rope_base: float, pos_ids, section, num_splits: int = 0,
                           lse=None, workspace=None, stream=None):
    if workspace is None:
        workspace = _workspace(pevlm_query_rope_workspace_bytes(layout, heads, num_splits), q)
    _s, sp = _i32_array(section)
    _check(load_library().pevlm_query_attn_mrope(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), layout.ref(), heads.ref(),
                                                 int(num_splits), float(rope_base), _ptr(pos_ids), sp, _ptr(workspace),
                                                 workspace.numel(), _stream_ptr(stream)))


def pevlm_rope_mrope(q, k, num_tokens: int, heads: Heads, rope_base: float, pos_ids, section, stream=None):
    """pos_ids: device int32 tensor [3, num_tokens]; section: three host ints adding up to head_dim/2."""
    sec = (ctypes.c_int32 * 3)(*[int(x) for x in section])
    _check(load_library().pevlm_rope_mrope(_ptr(q), _ptr(k), int(num_tokens), heads.ref(), float(rope_base), _ptr(pos_ids),
                                           sec, _stream_ptr(stream)))


def pevlm_block_prefill_workspace_bytes(layout: Layout, heads: Heads) -> int:
    return int(load_library().pevlm_block_prefill_workspace_bytes(layout.ref(), heads.ref()))


def pevlm_block_prefill_attn(q, k, v, out, layout: Layout, heads: Heads, lse=None, workspace=None, stream=None):
    if workspace is None:
        workspace = _workspace(pevlm_block_prefill_workspace_bytes(layout, heads), q)
    _check(load_library().pevlm_block_prefill_attn(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), layout.ref(),
                                                   heads.ref(), _ptr(workspace), workspace.numel(),
                                                   _stream_ptr(stream)))
    return workspace


FP8_QUANTISE, FP8_ATTEND = 1, 2


def pevlm_block_prefill_fp8_plan(layout: Layout, heads: Heads) -> Fp8Plan:
    plan = Fp8Plan()
    _check(load_library().pevlm_block_prefill_fp8_plan(layout.ref(), heads.ref(), ctypes.byref(plan)))
    return plan


def pevlm_block_prefill_fp8_workspace_bytes(layout: Layout, heads: Heads) -> int:
    return int(load_library().pevlm_block_prefill_fp8_workspace_bytes(layout.ref(), heads.ref()))


def pevlm_block_prefill_attn_fp8(q, k, v, out, layout: Layout, heads: Heads, lse=None, workspace=None, stages: int = 0,
                                 stream=None):
    if workspace is None:
        workspace = _workspace(pevlm_block_prefill_fp8_workspace_bytes(layout, heads), q)
    _check(load_library().pevlm_block_prefill_attn_fp8(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), layout.ref(),
                                                       heads.ref(), _ptr(workspace), workspace.numel(), int(stages),
                                                       _stream_ptr(stream)))
    return workspace


def pevlm_query_workspace_bytes(layout: Layout, heads: Heads, num_splits: int = 0) -> int:
    return int(load_library().pevlm_query_workspace_bytes(layout.ref(), heads.ref(), int(num_splits)))


def pevlm_query_attn(q, k, v, out, layout: Layout, heads: Heads, num_splits: int = 0, lse=None, workspace=None,
                     stream=None):
    if workspace is None:
        workspace = _workspace(pevlm_query_workspace_bytes(layout, heads, num_splits), q)
    _check(load_library().pevlm_query_attn(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), layout.ref(),
                                           heads.ref(), int(num_splits), _ptr(workspace), workspace.numel(),
                                           _stream_ptr(stream)))
    return workspace


def pevlm_query_attn_static(q, k, v, out, layout: Layout, heads: Heads, num_splits: int = 0, lse=None, stream=None):
    _check(load_library().pevlm_query_attn_static(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), layout.ref(),
                                                  heads.ref(), int(num_splits), _stream_ptr(stream)))


def _i32_array(values):
    """(owner, what the C call takes) of a host array of int32.  A list of integers becomes a ctypes array at
    once (0.6 us; through numpy 3.1); anything else, integers that int32 does not hold and ctypes has wrapped
    among it, is left to numpy."""
    if isinstance(values, (list, tuple)):
        try:
            a = (ctypes.c_int32 * len(values))(*values)
            if a[:] == list(values):
                return a, a
        except TypeError:
            pass
    a = np.ascontiguousarray(values, dtype=np.int32)
    return a, a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


def pevlm_block_prefill_attn_blocks(q, k, v, out, layout: Layout, heads: Heads, first_block, num_blocks, with_sink: bool,
                                    lse=None, workspace=None, stream=None):
    if workspace is None:
        workspace = _workspace(pevlm_block_prefill_workspace_bytes(layout, heads), q)
    _fb, fbp = _i32_array(first_block)
    _nb, nbp = _i32_array(num_blocks)
    _check(load_library().pevlm_block_prefill_attn_blocks(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), layout.ref(),
                                                          heads.ref(), fbp, nbp, int(bool(with_sink)), _ptr(workspace),
                                                          workspace.numel(), _stream_ptr(stream)))
    return workspace


def pevlm_query_window_workspace_bytes(layout: Layout, heads: Heads, num_splits: int = 0) -> int:
    return int(load_library().pevlm_query_window_workspace_bytes(layout.ref(), heads.ref(), int(num_splits)))


def pevlm_query_attn_window(q, k, v, out, layout: Layout, heads: Heads, window_blocks, num_splits: int = 0, lse=None,
                            workspace=None, stream=None):
    if workspace is None:
        workspace = _workspace(pevlm_query_window_workspace_bytes(layout, heads, num_splits), q)
    _w, wp = _i32_array(window_blocks)
    _check(load_library().pevlm_query_attn_window(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), layout.ref(), heads.ref(),
                                                  wp, int(num_splits), _ptr(workspace), workspace.numel(),
                                                  _stream_ptr(stream)))
    return workspace


def pevlm_prefill_worklist_blocks_host(layout: Layout, tile_rows: int, first_block, num_blocks, with_sink: bool):
    lib = load_library()
    _fb, fbp = _i32_array(first_block)
    _nb, nbp = _i32_array(num_blocks)
    n = lib.pevlm_prefill_worklist_blocks_host(layout.ref(), tile_rows, fbp, nbp, int(bool(with_sink)), None, 0)
    if n < 0:
        raise PevlmError(PEVLM_ERR_INVALID_ARG, pevlm_last_error())
    items = (WorkItem * max(n, 1))()
    lib.pevlm_prefill_worklist_blocks_host(layout.ref(), tile_rows, fbp, nbp, int(bool(with_sink)), items, n)
    return [items[i] for i in range(n)]


def pevlm_query_worklist_window_host(layout: Layout, tile_rows: int, num_splits: int, window_blocks):
    lib = load_library()
    _w, wp = _i32_array(window_blocks)
    n = lib.pevlm_query_worklist_window_host(layout.ref(), tile_rows, num_splits, wp, None, 0)
    if n < 0:
        raise PevlmError(PEVLM_ERR_INVALID_ARG, pevlm_last_error())
    items = (WorkItem * max(n, 1))()
    lib.pevlm_query_worklist_window_host(layout.ref(), tile_rows, num_splits, wp, items, n)
    return [items[i] for i in range(n)]


def pevlm_prefill_worklist_host(layout: Layout, tile_rows: int):
    lib = load_library()
    n = lib.pevlm_prefill_worklist_host(layout.ref(), tile_rows, None, 0)
    if n < 0:
        raise PevlmError(PEVLM_ERR_INVALID_ARG, pevlm_last_error())
    items = (WorkItem * max(n, 1))()
    lib.pevlm_prefill_worklist_host(layout.ref(), tile_rows, items, n)
    return [items[i] for i in range(n)]


def pevlm_prefill_uses_stream_kernel(layout: Layout, heads: Heads) -> bool:
    return bool(load_library().pevlm_prefill_uses_stream_kernel(layout.ref(), heads.ref()))


def pevlm_set_prefill_kernel(mode) -> int:
    """mode: 0 / "auto", 1 / "classic", 2 / "stream"; returns the previous mode (int)."""
    code = {"auto": 0, "classic": 1, "stream": 2}.get(mode, mode)
    prev = int(load_library().pevlm_set_prefill_kernel(int(code)))
    if prev < 0:
        raise PevlmError(PEVLM_ERR_INVALID_ARG, "prefill kernel mode must be 0, 1 or 2")
    return prev


def pevlm_prefill_stream_items_host(layout: Layout, heads: Heads, first_block=None, num_blocks=None, with_sink: bool = True):
    lib = load_library()
    fbp = nbp = None
    if first_block is not None:
        _fb, fbp = _i32_array(first_block)
        _nb, nbp = _i32_array(num_blocks)
    n = lib.pevlm_prefill_stream_items_host(layout.ref(), heads.ref(), fbp, nbp, int(bool(with_sink)), None, 0)
    if n < 0:
        raise PevlmError(PEVLM_ERR_INVALID_ARG, pevlm_last_error())
    items = (StreamItem * max(n, 1))()
    lib.pevlm_prefill_stream_items_host(layout.ref(), heads.ref(), fbp, nbp, int(bool(with_sink)), items, n)
    return [items[i] for i in range(n)]


def pevlm_query_worklist_host(layout: Layout, tile_rows: int, num_splits: int):
    lib = load_library()
    n = lib.pevlm_query_worklist_host(layout.ref(), tile_rows, num_splits, None, 0)
    if n < 0:
        raise PevlmError(PEVLM_ERR_INVALID_ARG, pevlm_last_error())
    items = (WorkItem * max(n, 1))()
    lib.pevlm_query_worklist_host(layout.ref(), tile_rows, num_splits, items, n)
    return [items[i] for i in range(n)]


def pevlm_visible_pairs(layout: Layout):
    a, b, c = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
    _check(load_library().pevlm_visible_pairs(layout.ref(), ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)))
    return a.value, b.value, c.value


# ------------------------------------------------------------------------------------------ paged KV cache in 4 bits
# A step of generation makes these calls once a layer, and its kernels take as long as their checks: those are made in one loop
# over the tensors, and the message is put together only where one fails.
_TORCH = None


def _torch():
    """(torch.int32, {dtype code: torch dtype}, torch.float32, torch.uint8, the current device, a device's current raw stream)."""
    global _TORCH
    if _TORCH is None:
        import torch

        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is None:
            raw = lambda device: torch.cuda.current_stream(device).cuda_stream  # noqa: E731
        _TORCH = (torch.int32, {PEVLM_F32: torch.float32, PEVLM_BF16: torch.bfloat16}, torch.float32, torch.uint8, torch.cuda.current_device, raw)
    return _TORCH


def _refuse(message: str):
    raise PevlmError(PEVLM_ERR_INVALID_ARG, message)


class KvCache:
    """Host-side descriptor of a paged 4-bit KV cache: the pool (device uint8 [num_pages][Hkv][page_size / 16][17 * head_dim], as
    new_pool makes it) and the requests' block table (device int32 [num_seqs][max_pages]).  Holds on to both tensors."""

    def __init__(self, pool, block_table, page_size: int):
        int32, _dtypes, _f32, uint8, _current, _raw = _torch()
        if pool.dtype != uint8 or pool.dim() != 4 or not pool.is_contiguous() or pool.shape[2] * 16 != page_size or pool.shape[3] % 17:
            _refuse(f"the pool must be a contiguous uint8 tensor [num_pages][Hkv][page_size / 16][17 * head_dim], got {tuple(pool.shape)} of "
                    f"{pool.dtype} for pages of {page_size}")
        if block_table.dtype != int32 or block_table.dim() != 2 or not block_table.is_contiguous():
            _refuse("block_table must be a contiguous int32 tensor [num_seqs][max_pages]")
        if pool.device != block_table.device:
            _refuse("the pool and block_table are on different devices")
        self.pool, self.block_table, self.page_size = pool, block_table, int(page_size)
        self.num_pages, self.n_kv_heads, self.head_dim = int(pool.shape[0]), int(pool.shape[1]), int(pool.shape[3]) // 17
        self.num_seqs, self.max_pages = int(block_table.shape[0]), int(block_table.shape[1])
        self.device = pool.get_device()
        self.struct = _CCache(pool.data_ptr(), self.num_pages, self.page_size, self.num_seqs, self.max_pages, block_table.data_ptr())
        self._ref = ctypes.byref(self.struct)

    @staticmethod
    def new_pool(heads: "Heads", num_pages: int, page_size: int, device):
        import torch

        if pevlm_cache_pool_bytes(heads, num_pages, page_size) == 0:
            _refuse(pevlm_last_error())
        return torch.zeros((num_pages, heads.n_kv_heads, page_size // 16, 17 * heads.head_dim), dtype=torch.uint8, device=device)

    def ref(self):
        return self._ref


def _arrays(cache: KvCache, int32, named):
    """Addresses of contiguous int32 arrays on the cache's device: named = ((name, tensor, entries), ...); None may stand for an optional one."""
    device, out = cache.device, []
    for name, t, n in named:
        if t is None:
            if name not in _OPTIONAL:
                _refuse(f"{name} must be given")
            out.append(None)
        else:
            if t.dtype is not int32 or t.numel() != n or not t.is_contiguous():
                _refuse(f"{name} must be a contiguous int32 tensor of {n} entries, got {tuple(t.shape)} of {t.dtype}")
            if t.get_device() != device:
                _refuse(f"{name} is on {t.device}, the cache on device {device}")
            out.append(t.data_ptr())
    return out


_OPTIONAL = frozenset(("new_len", "pos_offset", "pos_ids", "sink_len", "window"))


def _new_scratch(cache: KvCache, nbytes: int, stream):
    """A workspace that belongs to the stream of the call: torch's allocator does not give its memory to other work before that stream is done."""
    import torch

    if cache.device < 0:
        _refuse("the cache is not in device memory")
    if stream is None:
        return _workspace(nbytes, cache.pool)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(_stream_ptr(stream), device=cache.device)
    with torch.cuda.stream(stream):
        return _workspace(nbytes, cache.pool)


def _scratch(cache: KvCache, workspace):
    if not workspace.is_contiguous() or workspace.get_device() != cache.device:
        _refuse(f"the workspace must be contiguous and on the cache's device {cache.device}")
    return workspace.data_ptr(), workspace.numel()


def _on_device(cache: KvCache, fn, args, stream):
    """fn(*args, stream) on the cache's device; stream None: torch's current one there."""
    device, current, raw = cache.device, _TORCH[4], _TORCH[5]
    if device < 0:
        _refuse("the cache is not in device memory")
    if device == current():
        status = fn(*args, raw(device) if stream is None else _stream_ptr(stream))
    else:
        import torch

        with torch.cuda.device(device):
            status = fn(*args, raw(device) if stream is None else _stream_ptr(stream))
    if status != PEVLM_OK:
        _check(status)


def _check_heads_of(cache: KvCache, heads: Heads):
    if heads.n_kv_heads != cache.n_kv_heads or heads.head_dim != cache.head_dim:
        _refuse(f"the cache holds {cache.n_kv_heads} KV heads of {cache.head_dim}, heads has {heads.n_kv_heads} of {heads.head_dim}")


def pevlm_cache_pool_bytes(heads: Heads, num_pages: int, page_size: int) -> int:
    return int(load_library().pevlm_cache_pool_bytes(heads.ref(), int(num_pages), int(page_size)))


def pevlm_cache_slots_workspace_bytes(num_seqs: int) -> int:
    return int(load_library().pevlm_cache_slots_workspace_bytes(int(num_seqs)))


def pevlm_cache_slots(cache: KvCache, seq_len, new_len, free_pages, num_free, seq_len_out, num_free_out, row_start, row_len, slot_map,
                      pos_ids=None, pos_offset=None, workspace=None, stream=None):
    """Pages, slots and positions of the new tokens.  num_rows is slot_map's length; pos_ids: int32 [3][num_rows]."""
    int32 = (_TORCH or _torch())[0]
    n, rows, free = cache.num_seqs, slot_map.numel(), free_pages.numel()
    held, new, pages, left, offset, held_out, left_out, start, length, slots, pos = _arrays(cache, int32, (
        ("seq_len", seq_len, n), ("new_len", new_len, n), ("free_pages", free_pages, free), ("num_free", num_free, 1), ("pos_offset", pos_offset, n),
        ("seq_len_out", seq_len_out, n), ("num_free_out", num_free_out, 1), ("row_start", row_start, n), ("row_len", row_len, n),
        ("slot_map", slot_map, rows), ("pos_ids", pos_ids, 3 * rows)))
    if workspace is None:
        workspace = _new_scratch(cache, pevlm_cache_slots_workspace_bytes(n), stream)
    ws, nbytes = _scratch(cache, workspace)
    _on_device(cache, (_lib or load_library()).pevlm_cache_slots, (cache._ref, held, new, pages, free, left, rows, offset, held_out, left_out, start, length, slots,
                                                         pos, ws, nbytes), stream)
    return workspace


def _kv_rows(cache: KvCache, heads: Heads, k, v, slot_map):
    """Arguments of the calls that move rows: k and v [rows][Hkv][D], whose rows may lie further apart."""
    _check_heads_of(cache, heads)
    int32, dtypes, _f32, _u8, _current, _raw = _TORCH or _torch()
    rows, dtype, inner = slot_map.numel(), dtypes.get(heads.struct.dtype), cache.head_dim
    shape, device, args = (rows, cache.n_kv_heads, inner), cache.device, []
    for name, t in (("k", k), ("v", v)):
        if t.dtype is not dtype or t.shape != shape:
            _refuse(f"{name} must be {shape} of {dtype}, got {tuple(t.shape)} of {t.dtype}")
        stride = t.stride()
        if (stride[2] != 1 or (stride[1] != inner and shape[1] > 1)) and rows:
            _refuse(f"a row of {name} must be contiguous (strides {stride})")
        if rows > 1 and stride[0] < shape[1] * inner:  # 0, of an expanded tensor, would say contiguous to the library
            _refuse(f"rows of {name} must lie at least {shape[1] * inner} elements apart (strides {stride})")
        if t.get_device() != device:
            _refuse(f"{name} is on {t.device}, the cache on device {device}")
        args.append((t.data_ptr(), stride[0] if rows > 1 else 0))
    (slots,) = _arrays(cache, int32, (("slot_map", slot_map, rows),))
    return args[0][0], args[1][0], args[0][1], args[1][1], slots, rows, cache._ref, heads.ref()


def pevlm_cache_store_kv4(k, v, slot_map, cache: KvCache, heads: Heads, stream=None):
    """k, v: [rows][Hkv][D] of the dtype of heads, rows contiguous in themselves; slot_map: int32 [rows]."""
    _on_device(cache, (_lib or load_library()).pevlm_cache_store_kv4, _kv_rows(cache, heads, k, v, slot_map), stream)


def pevlm_cache_load_kv4(k, v, slot_map, cache: KvCache, heads: Heads, stream=None):
    """As pevlm_cache_store_kv4, the other way."""
    _on_device(cache, (_lib or load_library()).pevlm_cache_load_kv4, _kv_rows(cache, heads, k, v, slot_map), stream)


def pevlm_cache_attn_workspace_bytes(heads: Heads, num_seqs: int, num_rows: int) -> int:
    return int(load_library().pevlm_cache_attn_workspace_bytes(heads.ref(), int(num_seqs), int(num_rows)))


def pevlm_cache_attn_kv4(q, out, cache: KvCache, heads: Heads, row_start, row_len, seq_len, sink_len=None, window=None, lse=None,
                         workspace=None, stream=None):
    """q, out: contiguous [rows][Hq][D] of the dtype of heads; lse: float32 [rows][Hq] or None."""
    _check_heads_of(cache, heads)
    int32, dtypes, f32, _u8, _current, _raw = _TORCH or _torch()
    n, rows, device = cache.num_seqs, q.shape[0], cache.device
    shape, dtype = (rows, heads.n_q_heads, heads.head_dim), dtypes.get(heads.struct.dtype)
    for name, t in (("q", q), ("out", out)):
        if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
            _refuse(f"{name} must be contiguous, {shape} of {dtype}, got {tuple(t.shape)} of {t.dtype}")
        if t.get_device() != device:
            _refuse(f"{name} is on {t.device}, the cache on device {device}")
    if lse is not None:
        if lse.dtype is not f32 or lse.shape != shape[:2] or not lse.is_contiguous():
            _refuse(f"lse must be contiguous, {shape[:2]} of {f32}, got {tuple(lse.shape)} of {lse.dtype}")
        if lse.get_device() != device:
            _refuse(f"lse is on {lse.device}, the cache on device {device}")
    start, length, held, sink, near = _arrays(cache, int32, (("row_start", row_start, n), ("row_len", row_len, n), ("seq_len", seq_len, n),
                                                             ("sink_len", sink_len, n), ("window", window, n)))
    if workspace is None:
        workspace = _new_scratch(cache, pevlm_cache_attn_workspace_bytes(heads, n, rows), stream)
    ws, nbytes = _scratch(cache, workspace)
    _on_device(cache, (_lib or load_library()).pevlm_cache_attn_kv4, (q.data_ptr(), out.data_ptr(), None if lse is None else lse.data_ptr(), cache._ref,
                                                                        heads.ref(), rows, start, length, held, sink, near, ws, nbytes), stream)
    return workspace
