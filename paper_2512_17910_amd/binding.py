"""Thin Python binding over libalora_qkv.so (C ABI declared in include/alora_qkv.h).

Argument marshalling only: torch tensors supply device memory and the stream; every step of
the path runs in the library's HIP kernels.  There is no fallback: if the library is missing
the import of any entry point raises.
"""
from __future__ import annotations

import ctypes
import os
from array import array
from typing import List, Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libalora_qkv.so")

ALORA_F32, ALORA_BF16 = 0, 1
ALORA_OK, ALORA_EINVAL, ALORA_ESHAPE, ALORA_EWORKSPACE, ALORA_EHIP, ALORA_EDATA, ALORA_ENOMEM = 0, -1, -2, -3, -4, -5, -6
ALORA_ETOOBIG = -8
ALORA_MAX_ADAPTERS, ALORA_MAX_RANK = 128, 64


class AloraDims(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("T", ctypes.c_int32), ("hidden", ctypes.c_int32),
                ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("n_adapters", ctypes.c_int32), ("rank", ctypes.c_int32), ("n_segments", ctypes.c_int32),
                ("n_slots", ctypes.c_int64), ("token_seg_ids", ctypes.c_void_p),
                ("token_positions", ctypes.c_void_p)]


class AloraWsLayout(ctypes.Structure):
    _fields_ = [("active_off", ctypes.c_size_t), ("perm_off", ctypes.c_size_t),
                ("offsets_off", ctypes.c_size_t), ("total_bytes", ctypes.c_size_t)]


class AloraExtras(ctypes.Structure):
    _fields_ = [("bias", ctypes.c_void_p), ("adapter_ranks", ctypes.c_void_p), ("reuse_grouping", ctypes.c_int32),
                ("rope_cos", ctypes.c_void_p), ("rope_sin", ctypes.c_void_p), ("rope_positions", ctypes.c_int32)]


class AloraAttnDims(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("n_tokens", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("n_seqs", ctypes.c_int32),
                ("max_blocks", ctypes.c_int32), ("block_size", ctypes.c_int32), ("n_slots", ctypes.c_int64),
                ("scale", ctypes.c_float)]


class AloraHeadsDims(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("n_tokens", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("rotary_dim", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("norm", ctypes.c_int32), ("rope_positions", ctypes.c_int32),
                ("eps", ctypes.c_float), ("n_slots", ctypes.c_int64), ("q_stride", ctypes.c_int64),
                ("q_out_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("k_out_stride", ctypes.c_int64),
                ("v_stride", ctypes.c_int64), ("v_out_stride", ctypes.c_int64), ("dq_stride", ctypes.c_int64),
                ("dk_stride", ctypes.c_int64)]


class AloraRopeSpec(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("scaling", ctypes.c_int32), ("base", ctypes.c_double),
                ("factor", ctypes.c_double), ("original", ctypes.c_double), ("low", ctypes.c_double),
                ("high", ctypes.c_double), ("magnitude", ctypes.c_double)]


class AloraCacheDims(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("n_layers", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("block_size", ctypes.c_int32), ("n_slots", ctypes.c_int64),
                ("k_caches", ctypes.c_void_p), ("v_caches", ctypes.c_void_p)]
    on_host = None          # a cache that is no device tensor


class AloraStepDims(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("max_blocks", ctypes.c_int32), ("block_size", ctypes.c_int32),
                ("row_cap", ctypes.c_int32), ("pool_cap", ctypes.c_int32), ("n_slots", ctypes.c_int64)]


class AloraBoundsDims(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("n_rows", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("block_size", ctypes.c_int32), ("n_slots", ctypes.c_int64)]


class AloraError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().alora_status_string(status).decode()
        if status == ALORA_EHIP:
            msg += f" [hipError {lib().alora_last_hip_error()}]"
        super().__init__(f"{where}: {msg} ({status})")


_lib = None


_lib_path = LIB_PATH


def use_probe_library(path: str) -> None:
    """Make this process load a probe build of the library (see probe.py) instead of the product build.  Only
    before the first call into the library, and only the probe script does it: a probe build computes wrong
    results on purpose."""
    global _lib_path
    if _lib is not None:
        raise RuntimeError("the library is already loaded")
    _lib_path = path


def lib() -> ctypes.CDLL:
    """The loaded C-ABI library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_lib_path):
            raise ImportError(f"{_lib_path} is missing: build it with `python -m paper_2512_17910_amd.build` "
                              "(there is no non-HIP fallback)")
        # torch first: its HIP runtime must be the one this process uses (a library loaded before it would
        # bring the system's copy of the runtime in beside torch's, and the two do not share devices)
        import torch  # noqa: F401
        L = ctypes.CDLL(_lib_path)
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        L.alora_qkv_workspace_bytes.argtypes = [ctypes.POINTER(AloraDims), ctypes.POINTER(sz)]
        L.alora_qkv_workspace_layout.argtypes = [ctypes.POINTER(AloraDims), ctypes.POINTER(AloraWsLayout)]
        L.alora_qkv_classify_group.argtypes = [vp, vp, ctypes.POINTER(AloraDims), vp, sz, vp]
        L.alora_qkv_forward.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32,
                                        ctypes.POINTER(AloraDims), vp, sz, vp]
        L.alora_qkv_validate.argtypes = [vp, vp, vp, i32, ctypes.POINTER(AloraDims)]
        L.alora_qkv_forward_ex.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32,
                                           ctypes.POINTER(AloraDims), ctypes.POINTER(AloraExtras), vp, sz, vp]
        L.alora_qkv_graph_create.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32,
                                             ctypes.POINTER(AloraDims), ctypes.POINTER(AloraExtras), vp, sz,
                                             ctypes.POINTER(vp)]
        L.alora_qkv_forward_static.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32,
                                               ctypes.POINTER(AloraDims), ctypes.POINTER(AloraExtras), vp]
        L.alora_qkv_forward_static.restype = ctypes.c_int
        L.alora_qkv_static_scratch_bytes.argtypes = []
        L.alora_qkv_static_scratch_bytes.restype = sz
        L.alora_qkv_graph_launch.argtypes = [vp, vp]
        L.alora_qkv_graph_destroy.argtypes = [vp]
        L.alora_paged_attention.argtypes = [vp, vp, vp, vp, vp, vp, vp, ctypes.POINTER(AloraAttnDims), vp]
        L.alora_paged_attention_validate.argtypes = [vp, vp, vp, ctypes.POINTER(AloraAttnDims)]
        L.alora_paged_attention_suffix.argtypes = [vp, vp, vp, vp, vp, vp, vp, ctypes.POINTER(AloraAttnDims), vp]
        L.alora_paged_attention_split.argtypes = [vp, vp, vp, vp, vp, vp, vp, ctypes.POINTER(AloraAttnDims), vp, sz, vp]
        L.alora_paged_attention_workspace_bytes.argtypes = [ctypes.POINTER(AloraAttnDims), ctypes.POINTER(sz)]
        L.alora_paged_attention_suffix_split.argtypes = [vp, vp, vp, vp, vp, vp, vp, ctypes.POINTER(AloraAttnDims), vp, sz, vp]
        L.alora_paged_attention_suffix_workspace_bytes.argtypes = [ctypes.POINTER(AloraAttnDims), ctypes.POINTER(sz)]
        heads, spec, cache = ctypes.POINTER(AloraHeadsDims), ctypes.POINTER(AloraRopeSpec), ctypes.POINTER(AloraCacheDims)
        L.alora_qk_norm_rope.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, heads, vp]
        L.alora_qk_norm_rope_backward.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, heads, vp, sz, vp]
        L.alora_qk_norm_rope_workspace_bytes.argtypes = [heads, ctypes.POINTER(sz)]
        L.alora_qk_norm_rope_validate.argtypes = [vp, vp, heads]
        L.alora_rope_tables.argtypes = [vp, vp, i64, i64, spec, vp]
        L.alora_cache_copy_blocks.argtypes = [vp, vp, i32, cache, vp]
        L.alora_cache_move_rows.argtypes = [vp, vp, vp, i32, vp, vp, i32, i32, i32, cache, vp]
        L.alora_cache_move_rows_validate.argtypes = [vp, vp, vp, i32, i32, cache]
        attn = ctypes.POINTER(AloraAttnDims)
        L.alora_step_rows.argtypes = [vp] * 14 + [ctypes.POINTER(AloraStepDims), vp]
        L.alora_tree_rows.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, vp]
        L.alora_tree_attention_workspace_bytes.argtypes = [attn, i32, ctypes.POINTER(sz)]
        L.alora_tree_attention.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, vp, attn, vp, sz, vp]
        L.alora_block_bounds.argtypes = [vp, vp, vp, vp, ctypes.POINTER(AloraBoundsDims), vp]
        L.alora_block_select_workspace_bytes.argtypes = [attn, ctypes.POINTER(sz)]
        L.alora_block_select.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, attn, vp, sz, vp]
        L.alora_selected_attention_workspace_bytes.argtypes = [attn, i32, ctypes.POINTER(sz)]
        L.alora_selected_attention.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, vp, attn, vp, sz, vp]
        L.alora_status_string.argtypes = [ctypes.c_int]
        L.alora_status_string.restype = ctypes.c_char_p
        L.alora_qkv_set_tuning.argtypes = [ctypes.c_int, ctypes.c_int]
        L.alora_qkv_set_tuning.restype = ctypes.c_int
        L.alora_qkv_profile_begin.argtypes = [ctypes.c_int]
        L.alora_qkv_profile_begin_every.argtypes = [ctypes.c_int, ctypes.c_int]
        L.alora_qkv_profile_begin_every.restype = ctypes.c_int
        L.alora_qkv_profile_end.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int)]
        for name in ("alora_qkv_profile_begin", "alora_qkv_profile_end", "alora_qkv_workspace_bytes", "alora_qkv_workspace_layout", "alora_qkv_classify_group",
                     "alora_qkv_forward", "alora_qkv_validate", "alora_last_hip_error", "alora_qkv_version",
                     "alora_qkv_forward_ex", "alora_qkv_graph_create", "alora_qkv_graph_launch", "alora_qkv_graph_destroy",
                     "alora_paged_attention", "alora_paged_attention_validate", "alora_paged_attention_split", "alora_paged_attention_suffix",
                     "alora_paged_attention_workspace_bytes", "alora_paged_attention_suffix_split",
                     "alora_paged_attention_suffix_workspace_bytes", "alora_qk_norm_rope", "alora_qk_norm_rope_backward",
                     "alora_qk_norm_rope_workspace_bytes", "alora_qk_norm_rope_validate", "alora_rope_tables", "alora_cache_copy_blocks",
                     "alora_cache_move_rows", "alora_cache_move_rows_validate", "alora_step_rows", "alora_tree_rows", "alora_tree_attention",
                     "alora_tree_attention_workspace_bytes", "alora_block_bounds", "alora_block_select", "alora_block_select_workspace_bytes",
                     "alora_selected_attention", "alora_selected_attention_workspace_bytes"):
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return ALORA_BF16
    if t.dtype == torch.float32:
        return ALORA_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def make_dims(dtype: int, T: int, hidden: int, n_q_heads: int, n_kv_heads: int, head_dim: int,
              n_adapters: int, rank: int, n_segments: int, n_slots: int,
              token_seg_ids=None, token_positions=None) -> AloraDims:
    return AloraDims(dtype, T, hidden, n_q_heads, n_kv_heads, head_dim, n_adapters, rank, n_segments,
                     n_slots, _ptr(token_seg_ids), _ptr(token_positions))


def alora_qkv_workspace_bytes(dims: AloraDims) -> int:
    out = ctypes.c_size_t(0)
    s = lib().alora_qkv_workspace_bytes(ctypes.byref(dims), ctypes.byref(out))
    if s:
        raise AloraError(s, "alora_qkv_workspace_bytes")
    return int(out.value)


def alora_qkv_workspace_layout(dims: AloraDims) -> AloraWsLayout:
    out = AloraWsLayout()
    s = lib().alora_qkv_workspace_layout(ctypes.byref(dims), ctypes.byref(out))
    if s:
        raise AloraError(s, "alora_qkv_workspace_layout")
    return out


# Marshalling is what bounds the smallest calls (one row, a small fp32 layer: a projection's kernels take 10 to 17 us, its arguments took
# about as long), so the common path makes no Python object it can do without: the current stream's handle instead of a
# stream object, pointer tables as machine words, the extras in one constructor call.  Host time of a pass, us, measured in turn on one
# card: a small fp32 projection and its attention 17.0 -> 11.8 (the pass itself 17.8 -> 13.7), one row through four layers 57.7 -> 47.4.
_current_device = _current_raw_stream = None


def _stream_handle(stream) -> Optional[int]:
    global _current_device, _current_raw_stream
    if stream is not None:
        return stream.cuda_stream or None
    if _current_raw_stream is None:
        import torch
        torch.cuda.current_device()         # (initialises the device where nothing has yet, which the plain call does not)
        _current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        _current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda d: torch.cuda.current_stream(d).cuda_stream)
    return _current_raw_stream(_current_device()) or None


def alloc_workspace(dims: AloraDims, device="cuda"):
    import torch
    return torch.empty(alora_qkv_workspace_bytes(dims), dtype=torch.uint8, device=device)


def _ptr_array(tensors: Sequence) -> array:
    """The tensors' addresses; pass _table(arr) and keep arr alive over the call."""
    return array("Q", [t.data_ptr() for t in tensors])


def _table(arr: array) -> Optional[int]:
    return arr.buffer_info()[0] if arr else None


def _extras(bias, adapter_ranks, reuse_grouping, rope):
    """(AloraExtras, what has to stay alive over the call)."""
    ranks = None if adapter_ranks is None else (ctypes.c_int32 * len(adapter_ranks))(*[int(r) for r in adapter_ranks])
    on = rope is not None
    return AloraExtras(None if bias is None else bias.data_ptr(), None if ranks is None else ctypes.cast(ranks, ctypes.c_void_p),
                       1 if reuse_grouping else 0, _ptr(rope[0]) if on else None, _ptr(rope[1]) if on else None,
                       int(rope[0].shape[0]) if on else 0), ranks


def alora_qkv_classify_group(token_adapter_ids, activation_start, dims: AloraDims, workspace, stream=None):
    """Runs the classification/grouping step; returns (active, perm, offsets) views of the workspace.
    perm's first offsets[-1] entries are meaningful."""
    import torch
    s = lib().alora_qkv_classify_group(_ptr(token_adapter_ids), _ptr(activation_start), ctypes.byref(dims),
                                       _ptr(workspace), workspace.numel(), _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_qkv_classify_group")
    return workspace_int_views(dims, workspace)


def workspace_int_views(dims: AloraDims, workspace):
    import torch
    lay = alora_qkv_workspace_layout(dims)
    T, L = dims.T, dims.n_adapters
    active = workspace[lay.active_off: lay.active_off + T]
    perm = workspace[lay.perm_off: lay.perm_off + 4 * T].view(torch.int32)
    offsets = workspace[lay.offsets_off: lay.offsets_off + 4 * (L + 2)].view(torch.int32)
    return active, perm, offsets


def alora_qkv_forward(x, token_adapter_ids, activation_start, W_qkv, A: Sequence, B: Sequence,
                      q_out, k_cache, v_cache, slot_mapping, block_size: int, dims: AloraDims,
                      workspace, stream=None) -> None:
    """Enqueue the whole path on `stream` (default: torch's current stream).  Returns nothing;
    q_out and the mapped cache slots are written asynchronously."""
    a, b = _ptr_array(A), _ptr_array(B)
    p = [None if t is None else t.data_ptr() for t in (x, token_adapter_ids, activation_start, W_qkv, q_out, k_cache, v_cache, slot_mapping)]
    s = lib().alora_qkv_forward(p[0], p[1], p[2], p[3],
                                _table(a), _table(b), p[4], p[5], p[6], p[7], block_size, ctypes.byref(dims), _ptr(workspace),
                                workspace.numel() if workspace is not None else 0, _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_qkv_forward")


def alora_qkv_forward_ex(x, token_adapter_ids, activation_start, W_qkv, A: Sequence, B: Sequence,
                         q_out, k_cache, v_cache, slot_mapping, block_size: int, dims: AloraDims,
                         workspace, bias=None, adapter_ranks=None, stream=None, reuse_grouping: bool = False,
                         rope=None) -> None:
    """alora_qkv_forward with a layer bias [N] (device tensor) and/or one rank per adapter (host ints);
    reuse_grouping: use the classification/grouping an earlier call left in this workspace for the same
    token batch (the per-layer call of a model whose layers share one batch); rope: (cos, sin) fp32 device
    tensors [positions, head_dim / 2]: rotary embedding of q and k fused into the store."""
    ex, keep = _extras(bias, adapter_ranks, reuse_grouping, rope)
    a, b = _ptr_array(A), _ptr_array(B)
    p = [None if t is None else t.data_ptr() for t in (x, token_adapter_ids, activation_start, W_qkv, q_out, k_cache, v_cache, slot_mapping)]
    s = lib().alora_qkv_forward_ex(p[0], p[1], p[2], p[3],
                                   _table(a), _table(b), p[4], p[5], p[6], p[7], block_size, ctypes.byref(dims), ctypes.byref(ex),
                                   _ptr(workspace), workspace.numel() if workspace is not None else 0,
                                   _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_qkv_forward_ex")


def alora_qkv_forward_static(x, token_adapter_ids, activation_start, W_qkv, A: Sequence, B: Sequence,
                             q_out, k_cache, v_cache, slot_mapping, block_size: int, dims: AloraDims,
                             bias=None, adapter_ranks=None, stream=None, rope=None) -> None:
    """alora_qkv_forward_ex on the library's static device scratch: no workspace argument, no allocation."""
    ex, keep = _extras(bias, adapter_ranks, False, rope)
    a, b = _ptr_array(A), _ptr_array(B)
    p = [None if t is None else t.data_ptr() for t in (x, token_adapter_ids, activation_start, W_qkv, q_out, k_cache, v_cache, slot_mapping)]
    s = lib().alora_qkv_forward_static(p[0], p[1], p[2], p[3],
                                       _table(a), _table(b), p[4], p[5], p[6], p[7], block_size, ctypes.byref(dims), ctypes.byref(ex),
                                       _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_qkv_forward_static")


def alora_qkv_static_scratch_bytes() -> int:
    return int(lib().alora_qkv_static_scratch_bytes())


def alora_qkv_graph_create(x, token_adapter_ids, activation_start, W_qkv, A: Sequence, B: Sequence,
                           q_out, k_cache, v_cache, slot_mapping, block_size: int, dims: AloraDims, workspace,
                           bias=None, adapter_ranks=None, rope=None):
    """Record one forward call with these buffers for replay; returns an opaque handle for
    alora_qkv_graph_launch / alora_qkv_graph_destroy.  The caller keeps every tensor alive and rewrites
    their contents in place between launches."""
    h = ctypes.c_void_p(None)
    ex, keep = _extras(bias, adapter_ranks, False, rope)
    a, b = _ptr_array(A), _ptr_array(B)
    p = [None if t is None else t.data_ptr() for t in (x, token_adapter_ids, activation_start, W_qkv, q_out, k_cache, v_cache, slot_mapping)]
    s = lib().alora_qkv_graph_create(p[0], p[1], p[2], p[3],
                                     _table(a), _table(b), p[4], p[5], p[6], p[7], block_size, ctypes.byref(dims), ctypes.byref(ex),
                                     _ptr(workspace),
                                     workspace.numel() if workspace is not None else 0, ctypes.byref(h))
    if s:
        raise AloraError(s, "alora_qkv_graph_create")
    return h


def alora_qkv_graph_launch(graph, stream=None) -> None:
    s = lib().alora_qkv_graph_launch(graph, _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_qkv_graph_launch")


def alora_qkv_graph_destroy(graph) -> None:
    s = lib().alora_qkv_graph_destroy(graph)
    if s:
        raise AloraError(s, "alora_qkv_graph_destroy")


def alora_qkv_validate(token_adapter_ids, activation_start, slot_mapping, block_size: int, dims: AloraDims) -> int:
    return int(lib().alora_qkv_validate(_ptr(token_adapter_ids), _ptr(activation_start), _ptr(slot_mapping),
                                        block_size, ctypes.byref(dims)))


def alora_qkv_profile_begin(max_calls: int, every: int = 1) -> None:
    """Measure the dominant kernel of every `every`-th forward call, at most max_calls of them."""
    s = lib().alora_qkv_profile_begin_every(max_calls, every)
    if s:
        raise AloraError(s, "alora_qkv_profile_begin")


def alora_qkv_profile_end():
    """(average milliseconds of the dominant kernel, number of measured calls)."""
    ms, n = ctypes.c_double(0.0), ctypes.c_int(0)
    s = lib().alora_qkv_profile_end(ctypes.byref(ms), ctypes.byref(n))
    if s:
        raise AloraError(s, "alora_qkv_profile_end")
    return float(ms.value), int(n.value)


def alora_qkv_set_tuning(feature_tiles: int = 0, splits: int = 0) -> None:
    """Override the automatic tiling of the bf16 path (0, 0 restores it); see alora_qkv.h."""
    s = lib().alora_qkv_set_tuning(feature_tiles, splits)
    if s:
        raise AloraError(s, "alora_qkv_set_tuning")


def make_attn_dims(q, k_cache, block_tables, n_q_heads: int, n_kv_heads: int, head_dim: int, block_size: int,
                   scale: float = 0.0) -> AloraAttnDims:
    """Dimensions of an alora_paged_attention call, read off the tensors."""
    return AloraAttnDims(_dtype_code(q), q.shape[0], n_q_heads, n_kv_heads, head_dim, block_tables.shape[0],
                         block_tables.shape[1], block_size, k_cache.shape[0], scale)


def alora_paged_attention(q, k_cache, v_cache, block_tables, token_seq_ids, token_positions, out,
                          dims: AloraAttnDims, stream=None) -> None:
    """Enqueue causal softmax attention of the rows of q over the paged cache (include/alora_attention.h)."""
    s = lib().alora_paged_attention(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_tables), _ptr(token_seq_ids),
                                    _ptr(token_positions), _ptr(out), ctypes.byref(dims), _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_paged_attention")


def alora_paged_attention_validate(block_tables, token_seq_ids, token_positions, dims: AloraAttnDims) -> int:
    return int(lib().alora_paged_attention_validate(_ptr(block_tables), _ptr(token_seq_ids), _ptr(token_positions),
                                                    ctypes.byref(dims)))


def alora_paged_attention_workspace_bytes(dims: AloraAttnDims) -> int:
    out = ctypes.c_size_t(0)
    s = lib().alora_paged_attention_workspace_bytes(ctypes.byref(dims), ctypes.byref(out))
    if s:
        raise AloraError(s, "alora_paged_attention_workspace_bytes")
    return int(out.value)


def alora_paged_attention_split(q, k_cache, v_cache, block_tables, token_seq_ids, token_positions, out,
                                dims: AloraAttnDims, workspace, stream=None) -> None:
    """alora_paged_attention with every row's context cut into parts (small batches, long contexts)."""
    s = lib().alora_paged_attention_split(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_tables), _ptr(token_seq_ids),
                                          _ptr(token_positions), _ptr(out), ctypes.byref(dims), _ptr(workspace),
                                          workspace.numel() if workspace is not None else 0, _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_paged_attention_split")


def alora_paged_attention_suffix(q, k_cache, v_cache, block_tables, token_seq_ids, token_positions, out,
                                 dims: AloraAttnDims, stream=None) -> None:
    """alora_paged_attention for the rows of a projected suffix: consecutive rows of a sequence share the loads
    of their context (bf16, head_dim 128)."""
    s = lib().alora_paged_attention_suffix(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_tables), _ptr(token_seq_ids),
                                           _ptr(token_positions), _ptr(out), ctypes.byref(dims), _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_paged_attention_suffix")


def alora_paged_attention_suffix_workspace_bytes(dims: AloraAttnDims) -> int:
    out = ctypes.c_size_t(0)
    s = lib().alora_paged_attention_suffix_workspace_bytes(ctypes.byref(dims), ctypes.byref(out))
    if s:
        raise AloraError(s, "alora_paged_attention_suffix_workspace_bytes")
    return int(out.value)


def alora_paged_attention_suffix_split(q, k_cache, v_cache, block_tables, token_seq_ids, token_positions, out,
                                       dims: AloraAttnDims, workspace, stream=None) -> None:
    """alora_paged_attention_suffix with every row block's context cut into parts (few row blocks, long contexts)."""
    s = lib().alora_paged_attention_suffix_split(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_tables),
                                                 _ptr(token_seq_ids), _ptr(token_positions), _ptr(out), ctypes.byref(dims),
                                                 _ptr(workspace), workspace.numel() if workspace is not None else 0,
                                                 _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_paged_attention_suffix_split")


# ---- norm and rotary embedding of heads, rotary tables (include/alora_heads.h) -------------------
def _rows_stride(t, name: str, width: int) -> int:
    """Elements from row to row of a tensor whose rows are dense; 0 for None."""
    if t is None:
        return 0
    if t.dim() != 2 or t.stride(1) != 1 or t.shape[1] != width:
        raise ValueError(f"{name}: two dimensions of rows of {width} dense elements expected, got {tuple(t.shape)} with strides {t.stride()}")
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), width)


def _check_rope(rope):
    """(positions, pairs) of tables."""
    cos, sin = rope
    f32, shape = (_types or _torch_types())[0][ALORA_F32], cos.shape
    if cos.dtype is not f32 or sin.dtype is not f32 or len(shape) != 2 or sin.shape != shape or not (cos.is_contiguous() and sin.is_contiguous()):
        raise ValueError("rope: two contiguous fp32 tensors [positions, rotary_dim / 2] expected")
    return shape


_types = None


def _torch_types():
    """(types by the library's codes, int32, int64)"""
    global _types
    import torch
    _types = ((torch.float32, torch.bfloat16), torch.int32, torch.int64)
    return _types


# What a call takes beside the tensors that its dims describe is looked at in every call: a type, size or stride that the kernels do not
# expect would be misread in silence, or read behind its end, and a host address would go to a kernel.  That is 25 attributes of tensors for
# a call with norm and rotation, 1 us of its host time, which is why they stand in few conditions.
def _refuse(name: str, t, dtype, n: int) -> None:
    if t.dtype is not dtype:
        raise TypeError(f"{name}: {dtype} expected, got {t.dtype}")
    raise ValueError(f"{name}: {n} contiguous elements expected, got {tuple(t.shape)} with strides {t.stride()}")


def _refuse_host(**tensors) -> None:
    for name, t in tensors.items():
        if t is not None and not t.is_cuda:
            raise TypeError(f"{name}: a tensor on the GPU expected, got one on {t.device}")


def _check_rows(name: str, t, dtype, n: int) -> None:
    """One dense number a row; more than the call has rows are not read."""
    if t.dtype is not dtype or t.numel() < n or not t.is_contiguous():
        _refuse(name, t, dtype, n)


def _check_weights(name_q: str, wq, name_k: str, wk, dtype, d: int) -> None:
    if wq.dtype is not dtype or wq.numel() != d or not wq.is_contiguous():
        _refuse(name_q, wq, dtype, d)
    if wk.dtype is not dtype or wk.numel() != d or not wk.is_contiguous():
        _refuse(name_k, wk, dtype, d)


def _check_heads(wq, wk, rope, token_positions, dims):
    """What both calls of the heads take; the tables' addresses.  Tables are those that dims was made for, or longer ones."""
    by_code, i32, _ = _types or _torch_types()
    if token_positions is not None and (token_positions.dtype is not i32 or token_positions.numel() < dims.n_tokens or not token_positions.is_contiguous()):
        _refuse("token_positions", token_positions, i32, dims.n_tokens)
    if wq is not None and wk is not None:
        dtype, d = by_code[dims.dtype], dims.head_dim
        if wq.dtype is not dtype or wk.dtype is not dtype or wq.numel() != d or wk.numel() != d or not (wq.is_contiguous() and wk.is_contiguous()):
            _check_weights("wq", wq, "wk", wk, dtype, d)
    if rope is None:
        return None, None
    positions, pairs = _check_rope(rope)
    if positions < dims.rope_positions or 2 * pairs != dims.rotary_dim:
        raise ValueError(f"rope: tables of {dims.rope_positions} positions and {dims.rotary_dim // 2} pairs expected, got {positions} and {pairs}")
    return rope[0].data_ptr(), rope[1].data_ptr()


def make_heads_dims(q, q_out, k, k_out, n_q_heads: int, n_kv_heads: int, head_dim: int, rope=None, interleaved: bool = False,
                    norm: bool = True, eps: float = 1e-6, v=None, v_out=None, dq=None, dk=None) -> AloraHeadsDims:
    """Description of alora_qk_norm_rope calls on these tensors, or on others of the same shapes and strides: q, q_out, k, v
    rows (views of a fused buffer may be given), k_out and v_out the caches; k None: keys are turned where they lie in the cache.  For
    the backward pass q_out and k_out are the outputs' gradients, and dq, dk the gradients where their strides are not q's and k's."""
    nq, nkv = n_q_heads * head_dim, n_kv_heads * head_dim
    if rope is not None:
        _check_rope(rope)
    for name, t in (("q_out", q_out), ("k", k), ("k_out", k_out), ("v", v), ("v_out", v_out), ("dq", dq), ("dk", dk)):
        if t is not None and t.dtype != q.dtype:
            raise ValueError(f"{name}: {t.dtype}, but q is {q.dtype}")
    for name, t in (("q_out", q_out), ("k", k), ("v", v), ("dq", dq), ("dk", dk)):
        if t is not None and t.shape[0] != q.shape[0]:
            raise ValueError(f"{name}: {t.shape[0]} rows, but q has {q.shape[0]}")
    if v_out is not None and v_out.shape[0] != k_out.shape[0]:
        raise ValueError(f"v_out: {v_out.shape[0]} rows, but k_out has {k_out.shape[0]}")
    return AloraHeadsDims(_dtype_code(q), q.shape[0], n_q_heads, n_kv_heads, head_dim, 0 if rope is None else 2 * rope[0].shape[1],
                          1 if interleaved else 0, 1 if norm else 0, 0 if rope is None else rope[0].shape[0], eps, k_out.shape[0],
                          _rows_stride(q, "q", nq), _rows_stride(q_out, "q_out", nq), _rows_stride(k, "k", nkv),
                          _rows_stride(k_out, "k_out", nkv), _rows_stride(v, "v", nkv), _rows_stride(v_out, "v_out", nkv),
                          _rows_stride(dq, "dq", nq), _rows_stride(dk, "dk", nkv))


def alora_qk_norm_rope(q, q_out, k, k_cache, v, v_cache, wq, wk, rope, token_positions, slot_mapping, dims: AloraHeadsDims,
                       stream=None) -> None:
    """Enqueue norm and rotary embedding of the rows' heads (include/alora_heads.h): q to q_out, k (None: in place) to its slots of k_cache,
    v, where given, to v_cache.  The tensors are those that dims was made from, or of the same shapes and strides; wq and wk, of their
    type, are None without norm, rope without rotation."""
    i64 = (_types or _torch_types())[2]
    if slot_mapping.dtype is not i64 or slot_mapping.numel() < dims.n_tokens or not slot_mapping.is_contiguous():
        _refuse("slot_mapping", slot_mapping, i64, dims.n_tokens)
    cos, sin = _check_heads(wq, wk, rope, token_positions, dims)
    if not (q.is_cuda and q_out.is_cuda and k_cache.is_cuda and slot_mapping.is_cuda and (k is None or k.is_cuda) and (v is None or v.is_cuda) and (
            v_cache is None or v_cache.is_cuda) and (wq is None or wq.is_cuda) and (wk is None or wk.is_cuda) and (
            rope is None or rope[0].is_cuda and rope[1].is_cuda) and (token_positions is None or token_positions.is_cuda)):
        _refuse_host(q=q, q_out=q_out, k=k, k_cache=k_cache, v=v, v_cache=v_cache, wq=wq, wk=wk, cos=rope and rope[0], sin=rope and rope[1],
                     token_positions=token_positions, slot_mapping=slot_mapping)
    s = (_lib or lib()).alora_qk_norm_rope(q.data_ptr(), q_out.data_ptr(), None if k is None else k.data_ptr(), k_cache.data_ptr(),
                                           None if v is None else v.data_ptr(), None if v_cache is None else v_cache.data_ptr(),
                                           None if wq is None else wq.data_ptr(), None if wk is None else wk.data_ptr(),
                                           cos, sin, None if token_positions is None else token_positions.data_ptr(), slot_mapping.data_ptr(),
                                           dims, _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_qk_norm_rope")


def alora_qk_norm_rope_workspace_bytes(dims: AloraHeadsDims) -> int:
    """Bytes of workspace of the backward pass."""
    out = ctypes.c_size_t(0)
    s = lib().alora_qk_norm_rope_workspace_bytes(ctypes.byref(dims), ctypes.byref(out))
    if s:
        raise AloraError(s, "alora_qk_norm_rope_workspace_bytes")
    return int(out.value)


def alora_qk_norm_rope_backward(q, dq_out, dq, k, dk_out, dk, wq, wk, dwq, dwk, rope, token_positions, dims: AloraHeadsDims,
                                workspace=None, stream=None) -> None:
    """Enqueue the backward pass of alora_qk_norm_rope: dq, dk and, with norm, the fp32 dwq, dwk from the gradients of its outputs."""
    if dims.n_tokens > 1 and (dq.stride(0) != (dims.dq_stride or dims.q_stride) or dk.stride(0) != (dims.dk_stride or dims.k_stride)):
        raise ValueError("dq, dk: strides other than those of dims (make_heads_dims takes dq and dk)")
    cos, sin = _check_heads(wq, wk, rope, token_positions, dims)
    if dwq is not None and dwk is not None:
        _check_weights("dwq", dwq, "dwk", dwk, _types[0][ALORA_F32], dims.head_dim)
    if not (q.is_cuda and dq_out.is_cuda and dq.is_cuda and k.is_cuda and dk_out.is_cuda and dk.is_cuda and (wq is None or wq.is_cuda) and (
            wk is None or wk.is_cuda) and (dwq is None or dwq.is_cuda) and (dwk is None or dwk.is_cuda) and (
            rope is None or rope[0].is_cuda and rope[1].is_cuda) and (token_positions is None or token_positions.is_cuda) and (workspace is None or workspace.is_cuda)):
        _refuse_host(q=q, dq_out=dq_out, dq=dq, k=k, dk_out=dk_out, dk=dk, wq=wq, wk=wk, dwq=dwq, dwk=dwk, cos=rope and rope[0], sin=rope and rope[1],
                     token_positions=token_positions, workspace=workspace)
    s = (_lib or lib()).alora_qk_norm_rope_backward(
        q.data_ptr(), dq_out.data_ptr(), dq.data_ptr(), k.data_ptr(), dk_out.data_ptr(), dk.data_ptr(), None if wq is None else wq.data_ptr(),
        None if wk is None else wk.data_ptr(), None if dwq is None else dwq.data_ptr(), None if dwk is None else dwk.data_ptr(),
        cos, sin, None if token_positions is None else token_positions.data_ptr(), dims, None if workspace is None else workspace.data_ptr(),
        0 if workspace is None else workspace.nbytes, _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_qk_norm_rope_backward")


def alora_qk_norm_rope_validate(token_positions, slot_mapping, dims: AloraHeadsDims) -> int:
    _, i32, i64 = _types or _torch_types()
    for name, t, dtype in (("token_positions", token_positions, i32), ("slot_mapping", slot_mapping, i64)):
        if t is not None:
            _check_rows(name, t, dtype, dims.n_tokens)
    return int(lib().alora_qk_norm_rope_validate(_ptr(token_positions), _ptr(slot_mapping), ctypes.byref(dims)))


ROPE_SCALINGS = {"none": 0, "linear": 1, "by_parts": 2}


def make_rope_spec(rotary_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, original: float = 0.0, low: float = 1.0,
                   high: float = 32.0, magnitude: float = 1.0) -> AloraRopeSpec:
    """Angles of alora_rope_tables: scaling "none", "linear" or "by_parts" (include/alora_heads.h)."""
    if scaling not in ROPE_SCALINGS:
        raise ValueError(f"scaling {scaling!r}: one of {', '.join(ROPE_SCALINGS)} expected")
    return AloraRopeSpec(rotary_dim, ROPE_SCALINGS[scaling], base, factor, original, low, high, magnitude)


def alora_rope_tables(cos, sin, spec: AloraRopeSpec, first: int = 0, stream=None) -> None:
    """Fill the fp32 tensors cos, sin [rows, rotary_dim / 2] for positions first, first + 1, ..."""
    rows, pairs = cos.shape
    if 2 * pairs != spec.rotary_dim or sin.shape != cos.shape or not (cos.is_contiguous() and sin.is_contiguous()) or _dtype_code(cos) or _dtype_code(sin):
        raise ValueError(f"cos, sin: contiguous fp32 tensors [rows, {spec.rotary_dim // 2}] expected")
    _refuse_host(cos=cos, sin=sin)
    s = (_lib or lib()).alora_rope_tables(cos.data_ptr(), sin.data_ptr(), first, rows, spec, _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_rope_tables")


# ---- what the cache holds, moved (include/alora_cache.h) -----------------------------------------
def make_cache_dims(k_caches: Sequence, v_caches: Sequence, n_kv_heads: int, head_dim: int, block_size: int) -> AloraCacheDims:
    """The layers' caches [n_slots, n_kv_heads * head_dim], as alora_cache_copy_blocks and alora_cache_move_rows take them; it keeps the tensors."""
    if len(k_caches) != len(v_caches) or not k_caches:
        raise ValueError(f"{len(k_caches)} K caches and {len(v_caches)} V caches")
    tensors = [*k_caches, *v_caches]
    dtype, shape = tensors[0].dtype, (tensors[0].shape[0], n_kv_heads * head_dim)
    if not all(t.shape == shape and t.dtype is dtype and t.is_contiguous() for t in tensors):
        raise ValueError(f"caches: contiguous tensors [n_slots, {n_kv_heads * head_dim}] of one type expected")
    ptrs, n = _ptr_array(tensors), len(k_caches)
    at = _table(ptrs)
    d = AloraCacheDims(_dtype_code(tensors[0]), n, n_kv_heads, head_dim, block_size, shape[0], at, at + 8 * n)
    d.keep = (ptrs, tensors)
    d.on_host = next((t for t in tensors if not t.is_cuda), None)
    return d


def _host_int32(a, name: str) -> int:
    if a.dtype.char != "i" or not a.dtype.isnative or a.ndim != 1 or (a.strides != (4,) and a.size > 1):
        raise ValueError(f"{name}: a contiguous int32 array on the host expected")
    try:
        return ctypes.addressof(ctypes.c_char.from_buffer(a))      # (a third of the time of asking numpy)
    except (TypeError, ValueError):                                # read-only, or empty
        return a.__array_interface__["data"][0]


def alora_cache_copy_blocks(src, dst, dims: AloraCacheDims, stream=None) -> None:
    """Enqueue copies of blocks src[i] to dst[i] (src[i] = -1: cleared) in every layer; src, dst: int32 numpy arrays."""
    if len(src) != len(dst):
        raise ValueError(f"{len(src)} sources and {len(dst)} destinations")
    src_at, dst_at = _host_int32(src, "src"), _host_int32(dst, "dst")
    if dims.on_host is not None:
        _refuse_host(caches=dims.on_host)
    s = (_lib or lib()).alora_cache_copy_blocks(src_at, dst_at, len(src), dims, _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_cache_copy_blocks")


def _check_lists(src, dst, shift) -> int:
    """Rows of a move's lists."""
    n = src.shape[0]
    if dst.shape[0] != n or (shift is not None and shift.shape[0] != n):
        raise ValueError("src, dst, shift: one length expected")
    _, i32, i64 = _types or _torch_types()
    if src.dtype is not i64 or dst.dtype is not i64 or (shift is not None and (shift.dtype is not i32 or not shift.is_contiguous())) or not (
            src.is_contiguous() and dst.is_contiguous()):
        raise TypeError("src, dst: contiguous int64, shift: contiguous int32 expected")
    return n


def alora_cache_move_rows(src, dst, shift, rope, dims: AloraCacheDims, interleaved: bool = False, stream=None) -> None:
    """Enqueue moves of rows src[i] to dst[i] (int64 device tensors) in every layer, keys turned by shift[i] positions (int32, with the
    tables rope; both None: rows are only copied)."""
    n = _check_lists(src, dst, shift)
    if rope is None:
        cos = sin = None
        positions = pairs = 0
    else:
        positions, pairs = _check_rope(rope)
        if not (rope[0].is_cuda and rope[1].is_cuda):
            _refuse_host(cos=rope[0], sin=rope[1])
        cos, sin = rope[0].data_ptr(), rope[1].data_ptr()
    if not (src.is_cuda and dst.is_cuda and (shift is None or shift.is_cuda)) or dims.on_host is not None:
        _refuse_host(src=src, dst=dst, shift=shift, caches=dims.on_host)
    s = (_lib or lib()).alora_cache_move_rows(src.data_ptr(), dst.data_ptr(), None if shift is None else shift.data_ptr(), n, cos, sin, positions, 2 * pairs,
                                    1 if interleaved else 0, dims, _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_cache_move_rows")


def alora_cache_move_rows_validate(src, dst, shift, rope, dims: AloraCacheDims) -> int:
    n = _check_lists(src, dst, shift)
    return int(lib().alora_cache_move_rows_validate(_ptr(src), _ptr(dst), _ptr(shift), n, 0 if rope is None else rope[0].shape[0], ctypes.byref(dims)))


# ---- steps from lengths on the device, drafted trees, selected blocks ------------------------------
# (include/alora_steps.h, alora_tree.h, alora_select.h).  Every tensor of a call is looked at: its type, that it is dense and holds what the call's sizes
# say, and that it lies on the device the call goes to, the current one.
def _check_tensors(tensors) -> None:
    """tensors: (name, tensor, dtype, elements; a negative number: at least as many) each."""
    device = _current_device() if _current_device is not None else _device_now()
    for name, t, dtype, n in tensors:
        if t.get_device() != device or t.dtype is not dtype or not t.is_contiguous() or (t.numel() != n if n >= 0 else t.numel() < -n):
            if device >= 0 and not t.is_cuda:
                _refuse_host(**{name: t})
            if t.get_device() != device:
                raise ValueError(f"{name}: a tensor on the current device, cuda:{device}, expected, got one on {t.device}")
            _refuse(name, t, dtype, abs(n))
    if device < 0:
        _refuse_host(**{tensors[0][0]: tensors[0][1]})


def _check_workspace(workspace) -> None:
    """(Of the call's tensors, which are on the current device.)"""
    if workspace is None:
        return
    if not workspace.is_cuda:
        _refuse_host(workspace=workspace)
    if workspace.get_device() != _current_device() or not workspace.is_contiguous():
        raise ValueError("workspace: dense memory on the current device expected")


def _device_now() -> int:
    """The current device, -1 without any."""
    import torch
    if not torch.cuda.is_available():
        return -1
    _stream_handle(None)
    return _current_device()


def _check_reader(q, k_cache, v_cache, block_tables, out, dims: AloraAttnDims):
    """What the readers share, as _check_tensors takes it."""
    dtype = (_types or _torch_types())[0][dims.dtype]
    rows, slots = dims.n_tokens * dims.n_q_heads * dims.head_dim, dims.n_slots * dims.n_kv_heads * dims.head_dim
    return (("q", q, dtype, rows), ("k_cache", k_cache, dtype, slots), ("v_cache", v_cache, dtype, slots),
            ("block_tables", block_tables, _types[1], dims.n_seqs * dims.max_blocks), ("out", out, dtype, rows))


def _bytes(t) -> int:
    return 0 if t is None else t.nbytes


def make_step_dims(block_tables, block_size: int, row_cap: int, pool, n_slots: int) -> AloraStepDims:
    """Description of alora_step_rows calls: block_tables [n_seqs, max_blocks], pool a ring of block ids, row_cap rows of the token arrays."""
    return AloraStepDims(block_tables.shape[0], block_tables.shape[1], block_size, row_cap, pool.shape[0], n_slots)


def alora_step_rows(lengths, change, kept_blocks, seq_adapters, block_tables, pool, state, lengths_out, state_out, row_offsets, token_seq_ids,
                    token_positions, token_adapter_ids, slot_mapping, dims: AloraStepDims, stream=None) -> None:
    """Enqueue the step's rows, slots and block tables from the requests' lengths and changes (include/alora_steps.h); kept_blocks and seq_adapters may
    be None."""
    _, i32, i64 = _types or _torch_types()
    n, rows = dims.n_seqs, dims.row_cap
    _check_tensors((("lengths", lengths, i32, n), ("change", change, i32, n), ("block_tables", block_tables, i32, n * dims.max_blocks),
                    ("pool", pool, i32, dims.pool_cap), ("state", state, i32, 6), ("lengths_out", lengths_out, i32, n), ("state_out", state_out, i32, 6),
                    ("row_offsets", row_offsets, i32, n + 1), ("token_seq_ids", token_seq_ids, i32, rows), ("token_positions", token_positions, i32, rows),
                    ("token_adapter_ids", token_adapter_ids, i32, rows), ("slot_mapping", slot_mapping, i64, rows),
                    ("kept_blocks", lengths if kept_blocks is None else kept_blocks, i32, n),
                    ("seq_adapters", lengths if seq_adapters is None else seq_adapters, i32, n)))
    s = (_lib or lib()).alora_step_rows(lengths.data_ptr(), change.data_ptr(), _ptr(kept_blocks), _ptr(seq_adapters), block_tables.data_ptr(), pool.data_ptr(),
                                        state.data_ptr(), lengths_out.data_ptr(), state_out.data_ptr(), row_offsets.data_ptr(), token_seq_ids.data_ptr(),
                                        token_positions.data_ptr(), token_adapter_ids.data_ptr(), slot_mapping.data_ptr(), dims, _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_step_rows")


def alora_tree_rows(tree_parents, row_offsets, context_lens, tree_mask, token_positions, stream=None) -> None:
    """Enqueue the masks (int64 [rows, words], bit j: the sequence's draft j is seen) and positions of drafted trees (include/alora_tree.h)."""
    _, i32, i64 = _types or _torch_types()
    (rows, words), seqs = tree_mask.shape, context_lens.shape[0]
    _check_tensors((("tree_parents", tree_parents, i32, rows), ("row_offsets", row_offsets, i32, seqs + 1), ("context_lens", context_lens, i32, seqs),
                    ("tree_mask", tree_mask, i64, rows * words), ("token_positions", token_positions, i32, rows)))
    s = (_lib or lib()).alora_tree_rows(tree_parents.data_ptr(), row_offsets.data_ptr(), context_lens.data_ptr(), tree_mask.data_ptr(), token_positions.data_ptr(),
                                        rows, seqs, words, _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_tree_rows")


def alora_tree_attention_workspace_bytes(dims: AloraAttnDims, mask_words: int) -> int:
    out = ctypes.c_size_t(0)
    s = lib().alora_tree_attention_workspace_bytes(ctypes.byref(dims), mask_words, ctypes.byref(out))
    if s:
        raise AloraError(s, "alora_tree_attention_workspace_bytes")
    return int(out.value)


def alora_tree_attention(q, k_cache, v_cache, block_tables, row_offsets, context_lens, tree_mask, out, dims: AloraAttnDims, workspace,
                         stream=None) -> None:
    """Enqueue attention of drafted trees over the paged cache (include/alora_tree.h); dims from make_attn_dims."""
    shared = _check_reader(q, k_cache, v_cache, block_tables, out, dims)
    _, i32, i64 = _types
    words = tree_mask.shape[-1]
    _check_tensors((*shared, ("row_offsets", row_offsets, i32, dims.n_seqs + 1), ("context_lens", context_lens, i32, dims.n_seqs),
                    ("tree_mask", tree_mask, i64, dims.n_tokens * words)))
    _check_workspace(workspace)
    s = (_lib or lib()).alora_tree_attention(q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), block_tables.data_ptr(), row_offsets.data_ptr(),
                                             context_lens.data_ptr(), tree_mask.data_ptr(), words, out.data_ptr(), dims, _ptr(workspace), _bytes(workspace),
                                             _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_tree_attention")


def make_bounds_dims(k_cache, slot_mapping, n_kv_heads: int, head_dim: int, block_size: int) -> AloraBoundsDims:
    """Description of alora_block_bounds calls: k_cache [n_slots, n_kv_heads * head_dim], slot_mapping of the rows that a step wrote."""
    return AloraBoundsDims(_dtype_code(k_cache), slot_mapping.shape[0], n_kv_heads, head_dim, block_size, k_cache.shape[0])


def alora_block_bounds(k_cache, slot_mapping, bounds, scales, dims: AloraBoundsDims, stream=None) -> None:
    """Enqueue the bounds (int8 [blocks, n_kv_heads, 2, head_dim], fp32 scales [blocks, n_kv_heads]) of the blocks that the rows of slot_mapping lie
    in (include/alora_select.h)."""
    by_code, _, i64 = _types or _torch_types()
    global _int8
    if _int8 is None:
        import torch
        _int8 = torch.int8
    heads = dims.n_slots // dims.block_size * dims.n_kv_heads
    _check_tensors((("k_cache", k_cache, by_code[dims.dtype], dims.n_slots * dims.n_kv_heads * dims.head_dim), ("slot_mapping", slot_mapping, i64, -dims.n_rows),
                    ("bounds", bounds, _int8, heads * 2 * dims.head_dim), ("scales", scales, by_code[ALORA_F32], heads)))
    s = (_lib or lib()).alora_block_bounds(k_cache.data_ptr(), slot_mapping.data_ptr(), bounds.data_ptr(), scales.data_ptr(), dims, _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_block_bounds")


_int8 = None


def alora_block_select_workspace_bytes(dims: AloraAttnDims) -> int:
    out = ctypes.c_size_t(0)
    s = lib().alora_block_select_workspace_bytes(ctypes.byref(dims), ctypes.byref(out))
    if s:
        raise AloraError(s, "alora_block_select_workspace_bytes")
    return int(out.value)


def alora_block_select(q, bounds, scales, block_tables, token_seq_ids, token_positions, selected, n_first: int, n_recent: int, dims: AloraAttnDims, workspace,
                       stream=None) -> None:
    """Enqueue the choice of the blocks that every row and K/V head reads: selected, int32 [rows, n_kv_heads, budget] (include/alora_select.h)."""
    by_code, i32, _ = _types or _torch_types()
    global _int8
    if _int8 is None:
        import torch
        _int8 = torch.int8
    t, budget, heads = dims.n_tokens, selected.shape[-1], dims.n_slots // dims.block_size * dims.n_kv_heads
    _check_tensors((("q", q, by_code[dims.dtype], t * dims.n_q_heads * dims.head_dim), ("bounds", bounds, _int8, heads * 2 * dims.head_dim),
                    ("scales", scales, by_code[ALORA_F32], heads), ("block_tables", block_tables, i32, dims.n_seqs * dims.max_blocks),
                    ("token_seq_ids", token_seq_ids, i32, -t), ("token_positions", token_positions, i32, -t),
                    ("selected", selected, i32, t * dims.n_kv_heads * budget)))
    _check_workspace(workspace)
    s = (_lib or lib()).alora_block_select(q.data_ptr(), bounds.data_ptr(), scales.data_ptr(), block_tables.data_ptr(), token_seq_ids.data_ptr(),
                                           token_positions.data_ptr(), selected.data_ptr(), budget, n_first, n_recent, dims, _ptr(workspace), _bytes(workspace),
                                           _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_block_select")


def alora_selected_attention_workspace_bytes(dims: AloraAttnDims, budget: int) -> int:
    out = ctypes.c_size_t(0)
    s = lib().alora_selected_attention_workspace_bytes(ctypes.byref(dims), budget, ctypes.byref(out))
    if s:
        raise AloraError(s, "alora_selected_attention_workspace_bytes")
    return int(out.value)


def alora_selected_attention(q, k_cache, v_cache, block_tables, token_seq_ids, token_positions, selected, out, dims: AloraAttnDims, workspace=None,
                             stream=None) -> None:
    """Enqueue attention over the selected blocks alone (include/alora_select.h); selected as alora_block_select leaves it."""
    shared = _check_reader(q, k_cache, v_cache, block_tables, out, dims)
    i32, t, budget = _types[1], dims.n_tokens, selected.shape[-1]
    _check_tensors((*shared, ("token_seq_ids", token_seq_ids, i32, -t), ("token_positions", token_positions, i32, -t),
                    ("selected", selected, i32, t * dims.n_kv_heads * budget)))
    _check_workspace(workspace)
    s = (_lib or lib()).alora_selected_attention(q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), block_tables.data_ptr(), token_seq_ids.data_ptr(),
                                                 token_positions.data_ptr(), selected.data_ptr(), budget, out.data_ptr(), dims, _ptr(workspace),
                                                 _bytes(workspace), _stream_handle(stream))
    if s:
        raise AloraError(s, "alora_selected_attention")
