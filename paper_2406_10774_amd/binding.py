"""ctypes binding of libquest.so: argument marshalling only.

Every function has the name and argument order of its C entry point in
include/quest.h and does nothing but turn torch tensors into device pointers,
pass the current HIP stream, and raise QuestError on a non-zero status.  All
computation happens in the HIP kernels; there is no fallback path: if the
library has not been built, loading fails."""
from __future__ import annotations

import ctypes
import os

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG_DIR, "libquest.so")

QUEST_OK = 0
QUEST_FLAG_SEPARATE_LAUNCHES = 1
QUEST_FLAG_DEVICE_FENCES = 2
QUEST_FLAG_KEEP_FIRST_PAGE = 4
QUEST_FLAG_KEEP_NEWEST_PAGE = 8
QUEST_FLAG_E4M3_PAGES = 16
STATUS_NAMES = {0: "QUEST_OK", -1: "QUEST_ERR_NULL", -2: "QUEST_ERR_SHAPE",
                -3: "QUEST_ERR_UNSUPPORTED", -4: "QUEST_ERR_WORKSPACE", -5: "QUEST_ERR_HIP"}

EXPORTS = ("quest_workspace_bytes", "quest_build_meta", "quest_append_meta", "quest_estimate",
           "quest_append_estimate", "quest_topk", "quest_topk_workspace_bytes", "quest_sparse_decode",
           "quest_select_decode", "quest_step_workspace_bytes", "quest_decode_step",
           "quest_decode_step_static", "quest_append_tokens", "quest_tokens_workspace_bytes",
           "quest_prompt_attention", "quest_tree_attention", "quest_rotate_tokens",
           "quest_rotate_append_tokens", "quest_last_error")


class QuestError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class quest_cache(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("num_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32),
        ("max_pages_per_seq", ctypes.c_int32), ("flags", ctypes.c_int32),
        ("num_phys_pages", ctypes.c_int64),
        ("k_pool", ctypes.c_void_p), ("v_pool", ctypes.c_void_p), ("meta", ctypes.c_void_p),
        ("page_table", ctypes.c_void_p), ("seq_lens", ctypes.c_void_p),
        ("num_kv_heads", ctypes.c_int32), ("scales", ctypes.c_void_p),
    ]


class quest_rotation(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("num_positions", ctypes.c_int32),
                ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32)]


_lib = None


def load():
    """Load libquest.so (built by paper_2406_10774_amd.build); fail loudly if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2406_10774_amd.build` "
            "(there is no fallback implementation)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float
    cp = ctypes.POINTER(quest_cache)
    lib.quest_workspace_bytes.argtypes = [cp, i32, ctypes.POINTER(ctypes.c_size_t)]
    lib.quest_build_meta.argtypes = [cp, vp]
    lib.quest_append_meta.argtypes = [cp, vp, vp, i32, vp]
    lib.quest_estimate.argtypes = [cp, vp, vp, vp]
    lib.quest_append_estimate.argtypes = [cp, vp, vp, i32, vp, vp, vp]
    lib.quest_topk.argtypes = [cp, vp, i32, vp, vp, vp, ctypes.c_size_t, vp]
    lib.quest_topk_workspace_bytes.argtypes = [cp, i32, ctypes.POINTER(ctypes.c_size_t)]
    lib.quest_sparse_decode.argtypes = [cp, vp, vp, i32, f32, vp, i32, vp, vp, ctypes.c_size_t, vp]
    lib.quest_select_decode.argtypes = [cp, vp, vp, i32, f32, vp, vp, vp, i32, vp, vp, ctypes.c_size_t, vp]
    lib.quest_step_workspace_bytes.argtypes = [cp, i32, ctypes.POINTER(ctypes.c_size_t)]
    lib.quest_decode_step.argtypes = [cp, vp, vp, i32, vp, i32, f32, vp, vp, vp, vp, i32, vp, vp,
                                      ctypes.c_size_t, vp]
    lib.quest_decode_step_static.argtypes = [cp, vp, vp, i32, vp, i32, f32, vp, vp, vp, vp, i32, vp, vp]
    i64 = ctypes.c_int64
    lib.quest_append_tokens.argtypes = [cp, vp, vp, i64, vp, vp, i32, vp]
    lib.quest_tokens_workspace_bytes.argtypes = [cp, i32, ctypes.POINTER(ctypes.c_size_t)]
    lib.quest_prompt_attention.argtypes = [cp, vp, i64, vp, i32, f32, vp, i32, vp, vp, ctypes.c_size_t, vp]
    lib.quest_tree_attention.argtypes = [cp, vp, i64, vp, vp, i64, vp, i32, vp, i32, vp, i32, f32, vp, i32, vp, vp,
                                         ctypes.c_size_t, vp]
    rp = ctypes.POINTER(quest_rotation)
    lib.quest_rotate_tokens.argtypes = [cp, rp, vp, i64, i32, vp, i32, vp, i64, vp]
    lib.quest_rotate_append_tokens.argtypes = [cp, rp, vp, i64, vp, i64, vp, vp, i64, vp, i32, vp]
    for name in EXPORTS[:-1]:
        getattr(lib, name).restype = ctypes.c_int
    lib.quest_last_error.argtypes = []
    lib.quest_last_error.restype = ctypes.c_char_p
    _lib = lib
    return lib


# A step of a short context lasts about 9 us on the GPU, so what happens here in front of the
# launches counts: torch is looked up once, pointers and the stream go to ctypes as plain
# integers, and the stream is read without building a torch.cuda.Stream (0.1 us, not
# 2.7 us).  quest_decode_step at one head, call after call: 12.2 -> 9.6 us, of which the two
# launches themselves take 8.8.
_half = None
_current_device = None
_raw_stream = None


def _bind_torch():
    global _half, _current_device, _raw_stream
    import torch
    _half = torch.float16
    _current_device = torch.cuda.current_device
    _raw_stream = torch._C._cuda_getCurrentRawStream


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    if stream is not None:
        return int(stream)
    if _raw_stream is None:
        _bind_torch()
    return _raw_stream(_current_device())


def _is_half(t):
    if _half is None:
        _bind_torch()
    return int(t.dtype is _half)


def _nbytes(t):
    return 0 if t is None else t.nbytes


def _check(status):
    if status:
        raise QuestError(status, load().quest_last_error().decode())


def _check_e4m3(k_pool, v_pool, scales):
    import torch
    N, Hkv = k_pool.shape[:2]
    for pool in (k_pool, v_pool):
        if pool is None or pool.dtype not in (torch.float8_e4m3fn, torch.uint8) or not pool.is_contiguous() or pool.shape != k_pool.shape:
            raise QuestError(-2, "pools of 8 bits have to be float8_e4m3fn (or uint8), contiguous and of the same shape")
    if (scales is None or scales.dtype is not torch.float32 or not scales.is_contiguous() or tuple(scales.shape) != (N, Hkv, 2)
            or scales.device != k_pool.device or v_pool.device != k_pool.device):
        raise QuestError(-2, f"pages of 8 bits need scales: float32 [{N}][{Hkv}][2], contiguous, on the pools' device")


class Cache:
    """Host-side description of one layer's paged KV cache (see quest_cache in quest.h).

    Holds references to the caller's torch tensors so they outlive the calls."""

    def __init__(self, k_pool, v_pool, meta, page_table, seq_lens, flags=0, num_heads=None, scales=None):
        """num_heads: query heads, if more than the KV heads of the pools (grouped-query
        attention); default: one KV head per query head.  scales: float32 [pages][KV heads][2] of pools of 8 bits
        (torch.float8_e4m3fn, or its bytes as torch.uint8)."""
        N, Hkv, S, D = k_pool.shape
        H = Hkv if num_heads is None else int(num_heads)
        if scales is not None or k_pool.element_size() == 1:
            _check_e4m3(k_pool, v_pool, scales)
            flags = int(flags) | QUEST_FLAG_E4M3_PAGES
        elif int(flags) & QUEST_FLAG_E4M3_PAGES:
            raise QuestError(-2, "pages of 8 bits need scales")
        self.scales = scales
        self.k_pool, self.v_pool, self.meta = k_pool, v_pool, meta
        self.page_table, self.seq_lens = page_table, seq_lens
        self.c = quest_cache(
            batch=page_table.shape[0], num_heads=H, head_dim=D, page_size=S,
            max_pages_per_seq=page_table.shape[1], flags=int(flags), num_phys_pages=N,
            k_pool=k_pool.data_ptr(), v_pool=v_pool.data_ptr() if v_pool is not None else None,
            meta=meta.data_ptr(), page_table=page_table.data_ptr(), seq_lens=seq_lens.data_ptr(),
            num_kv_heads=0 if H == Hkv else Hkv, scales=None if scales is None else scales.data_ptr())
        self.heads, self.kv_heads, self.batch, self.head_dim = H, Hkv, page_table.shape[0], D
        self.device = k_pool.get_device()
        self.ref = ctypes.byref(self.c)


class Rotation:
    """Rotation of queries and keys by their position (see quest_rotation in quest.h).

    table: float32 [positions][rotary_dim], the cosines of a position's angles, then their sines; positions: int32, of
    every packed row, if not where the sequence's length puts it."""

    def __init__(self, table, interleaved=False, positions=None):
        import torch
        if table.dim() != 2 or table.dtype is not torch.float32 or not table.is_contiguous():
            raise QuestError(-2, f"table of shape {tuple(table.shape)} ({table.dtype}): has to be float32 [positions][rotary_dim], contiguous")
        if positions is not None and (positions.dtype is not torch.int32 or not positions.is_contiguous()
                                      or positions.device != table.device):
            raise QuestError(-2, f"positions ({positions.dtype}, {positions.device}): have to be int32, contiguous, on the table's device")
        self.table, self.positions = table, positions
        self.rows = None if positions is None else positions.numel()
        self.device = table.get_device()
        self.c = quest_rotation(table=table.data_ptr(), positions=_ptr(positions), num_positions=table.shape[0],
                                rotary_dim=table.shape[1], interleaved=int(bool(interleaved)))
        self.ref = ctypes.byref(self.c)


def quest_workspace_bytes(cache: Cache, k_pages: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().quest_workspace_bytes(cache.ref, int(k_pages), ctypes.byref(out)))
    return out.value


def quest_build_meta(cache: Cache, stream=None):
    _check(load().quest_build_meta(cache.ref, _stream(stream)))


def quest_append_meta(cache: Cache, k_new, v_new=None, k_pool_write=False, stream=None):
    _check(load().quest_append_meta(cache.ref, _ptr(k_new), _ptr(v_new), int(bool(k_pool_write)),
                                    _stream(stream)))


def quest_estimate(cache: Cache, q, scores, stream=None):
    _check(load().quest_estimate(cache.ref, _ptr(q), _ptr(scores), _stream(stream)))


def quest_append_estimate(cache: Cache, k_new, v_new, k_pool_write, q, scores, stream=None):
    _check(load().quest_append_estimate(cache.ref, _ptr(k_new), _ptr(v_new),
                                        int(bool(k_pool_write)), _ptr(q), _ptr(scores),
                                        _stream(stream)))


def quest_topk(cache: Cache, scores, k_pages, topk_idx, k_eff=None, workspace=None, stream=None):
    ws_bytes = _nbytes(workspace)
    _check(load().quest_topk(cache.ref, _ptr(scores), int(k_pages), _ptr(topk_idx), _ptr(k_eff),
                             _ptr(workspace), ws_bytes, _stream(stream)))


def quest_topk_workspace_bytes(cache: Cache, k_pages: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().quest_topk_workspace_bytes(cache.ref, int(k_pages), ctypes.byref(out)))
    return out.value


def quest_sparse_decode(cache: Cache, q, topk_idx, k_pages, sm_scale, out, lse=None,
                        workspace=None, stream=None):
    ws_bytes = _nbytes(workspace)
    _check(load().quest_sparse_decode(
        cache.ref, _ptr(q), _ptr(topk_idx), int(k_pages), float(sm_scale), _ptr(out),
        _is_half(out), _ptr(lse), _ptr(workspace), ws_bytes, _stream(stream)))


def quest_select_decode(cache: Cache, q, scores, k_pages, sm_scale, topk_idx, out, k_eff=None,
                        lse=None, workspace=None, stream=None):
    ws_bytes = _nbytes(workspace)
    _check(load().quest_select_decode(
        cache.ref, _ptr(q), _ptr(scores), int(k_pages), float(sm_scale), _ptr(topk_idx), _ptr(k_eff),
        _ptr(out), _is_half(out), _ptr(lse), _ptr(workspace), ws_bytes,
        _stream(stream)))


def quest_step_workspace_bytes(cache: Cache, k_pages: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().quest_step_workspace_bytes(cache.ref, int(k_pages), ctypes.byref(out)))
    return out.value


def quest_decode_step(cache: Cache, k_new, v_new, k_pool_write, q, k_pages, sm_scale, scores,
                      topk_idx, out, workspace, k_eff=None, lse=None, stream=None):
    ws_bytes = _nbytes(workspace)
    _check(load().quest_decode_step(
        cache.ref, _ptr(k_new), _ptr(v_new), int(bool(k_pool_write)), _ptr(q), int(k_pages),
        float(sm_scale), _ptr(scores), _ptr(topk_idx), _ptr(k_eff), _ptr(out),
        _is_half(out), _ptr(lse), _ptr(workspace), ws_bytes, _stream(stream)))



def quest_decode_step_static(cache: Cache, k_new, v_new, k_pool_write, q, k_pages, sm_scale, scores,
                             topk_idx, out, k_eff=None, lse=None, stream=None):
    _check(load().quest_decode_step_static(
        cache.ref, _ptr(k_new), _ptr(v_new), int(bool(k_pool_write)), _ptr(q), int(k_pages),
        float(sm_scale), _ptr(scores), _ptr(topk_idx), _ptr(k_eff), _ptr(out),
        _is_half(out), _ptr(lse), _stream(stream)))


# ---- many tokens a sequence.  Packed tensors are [rows][heads][head_dim] with any stride between rows.

# (What is checked here costs 2 to 3 us a call, a part of them a tensor's shape, strides and device.)

_types = None


def _types_of_torch():
    global _types
    import torch
    _bind_torch()
    _types = torch.float32, torch.int32, torch.int64
    return _types


def _rows_of(cache, shape, t, heads, other=None):
    """Elements between the rows of t (its shape, t), and of `other`: fp16 rows whose heads lie next to each other."""
    dim, device = cache.head_dim, cache.device
    if len(shape) == 3 and shape[1] == heads and shape[2] == dim and t.dtype is _half and t.get_device() == device:
        if t.is_contiguous() and (other is None or other.dtype is _half and other.is_contiguous() and other.shape == shape
                                  and other.get_device() == device):
            return heads * dim
        stride = t.stride()
        if stride[2] == 1 and (stride[1] == dim or heads == 1) and (
                other is None or other.dtype is _half and other.stride() == stride and other.shape == shape
                and other.get_device() == device):
            return stride[0] if shape[0] > 1 else heads * dim
    stride = t.stride()
    what = "" if other is None else f", {tuple(other.shape)} and {other.stride()} ({other.dtype}, {other.device})"
    raise QuestError(-2, f"packed rows of shape {tuple(shape)} and strides {stride} ({t.dtype}, {t.device}){what}: they have to "
                         f"be fp16 [rows][{heads}][{dim}] on the cache's device, heads next to each other, keys as values")


def _plain(cache, t, dtype, least, what):
    """Refuses a tensor of another type or device, with gaps, or with fewer elements."""
    if t.dtype is not dtype or t.numel() < least or not t.is_contiguous() or t.get_device() != cache.device:
        raise QuestError(-2, f"{what} of shape {tuple(t.shape)}, strides {t.stride()} ({t.dtype}, {t.device}): has to be {dtype}, "
                             f"contiguous, of at least {least} elements, on the cache's device")


def _outputs(cache, out, lse, workspace, rows):
    _plain(cache, out, _half if out.dtype is _half else _types[0], rows * cache.heads * cache.head_dim, "out")
    if lse is not None:
        _plain(cache, lse, _types[0], rows * cache.heads, "lse")
    if workspace is not None and (workspace.get_device() != cache.device or not workspace.is_contiguous()):
        raise QuestError(-2, f"workspace of strides {workspace.stride()} on {workspace.device}: has to be contiguous, on the "
                             "cache's device")


def _stream_of(cache, stream):
    """The stream, or the current one; the cache's device has to be the current one."""
    device = cache.device
    if device >= 0 and _current_device() != device:
        raise QuestError(-2, f"the cache lies on device {device}, which is not the current one")
    return _stream(stream) if device < 0 or stream is not None else _raw_stream(device)


def quest_append_tokens(cache: Cache, k_new, v_new, cu_tokens, rows=None, stream=None):
    _, i32, _ = _types or _types_of_torch()
    shape = k_new.shape
    stride = _rows_of(cache, shape, k_new, cache.kv_heads, v_new)
    total = shape[0]
    if rows is not None:
        _plain(cache, rows, i32, 0, "rows")
        total = rows.numel()
    _plain(cache, cu_tokens, i32, cache.batch + 1, "cu_tokens")
    _check(load().quest_append_tokens(cache.ref, k_new.data_ptr(), v_new.data_ptr(), stride, _ptr(rows),
                                      cu_tokens.data_ptr(), total, _stream_of(cache, stream)))


def quest_tokens_workspace_bytes(cache: Cache, total_tokens: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().quest_tokens_workspace_bytes(cache.ref, int(total_tokens), ctypes.byref(out)))
    return out.value


def quest_prompt_attention(cache: Cache, q, cu_tokens, sm_scale, out, lse=None, workspace=None, stream=None):
    _, i32, _ = _types or _types_of_torch()
    shape, heads = q.shape, cache.heads
    stride = _rows_of(cache, shape, q, heads)
    total = shape[0]
    _plain(cache, cu_tokens, i32, cache.batch + 1, "cu_tokens")
    _outputs(cache, out, lse, workspace, total)
    _check(load().quest_prompt_attention(
        cache.ref, q.data_ptr(), stride, cu_tokens.data_ptr(), total, float(sm_scale), out.data_ptr(),
        out.dtype is _half, _ptr(lse), _ptr(workspace), _nbytes(workspace), _stream_of(cache, stream)))


def quest_tree_attention(cache: Cache, q, k_new, v_new, cu_tokens, tree_mask, sm_scale, out, topk_idx=None, lse=None,
                         workspace=None, stream=None):
    """tree_mask: int64 [rows][words]; topk_idx: int32 [batch][KV heads][k_pages], or None for all pages."""
    _, i32, i64 = _types or _types_of_torch()
    shape, heads, new_shape = q.shape, cache.heads, k_new.shape
    q_stride = _rows_of(cache, shape, q, heads)
    new_stride = _rows_of(cache, new_shape, k_new, cache.kv_heads, v_new)
    total, k_pages = shape[0], 0
    if tree_mask.dim() != 2 or topk_idx is not None and (topk_idx.dim() != 3 or topk_idx.shape[1] != cache.kv_heads):
        raise QuestError(-2, f"tree_mask of shape {tuple(tree_mask.shape)}{'' if topk_idx is None else f' and topk_idx of {tuple(topk_idx.shape)}'}"
                             f": have to be [rows][words] and [batch][{cache.kv_heads}][k_pages]")
    mask_rows, words = tree_mask.shape
    if new_shape[0] < total or mask_rows < total:
        raise QuestError(-2, f"{new_shape[0]} rows of keys and values and {mask_rows} of masks for {total} of queries")
    _plain(cache, tree_mask, i64, 0, "tree_mask")
    _plain(cache, cu_tokens, i32, cache.batch + 1, "cu_tokens")
    if topk_idx is not None:
        k_pages = topk_idx.shape[2]
        _plain(cache, topk_idx, i32, cache.batch * cache.kv_heads * k_pages, "topk_idx")
    _outputs(cache, out, lse, workspace, total)
    _check(load().quest_tree_attention(
        cache.ref, q.data_ptr(), q_stride, k_new.data_ptr(), v_new.data_ptr(), new_stride, cu_tokens.data_ptr(),
        total, tree_mask.data_ptr(), words, _ptr(topk_idx), k_pages, float(sm_scale), out.data_ptr(),
        out.dtype is _half, _ptr(lse), _ptr(workspace), _nbytes(workspace), _stream_of(cache, stream)))


def _rotation_of(cache, rotation, total):
    if rotation.device != cache.device or rotation.rows is not None and rotation.rows < total:
        raise QuestError(-2, f"rotation on device {rotation.device} with positions of {rotation.rows} rows: has to be on the cache's "
                             f"device, with a position for each of {total} rows")


def quest_rotate_tokens(cache: Cache, rotation: Rotation, x, cu_tokens, out, stream=None):
    _, i32, _ = _types or _types_of_torch()
    shape, out_shape = x.shape, out.shape
    heads = shape[1] if len(shape) == 3 else 0
    stride, out_stride = _rows_of(cache, shape, x, heads), _rows_of(cache, out_shape, out, heads)
    if out_shape[0] < shape[0]:
        raise QuestError(-2, f"{out_shape[0]} rows of results for {shape[0]}")
    _rotation_of(cache, rotation, shape[0])
    _plain(cache, cu_tokens, i32, cache.batch + 1, "cu_tokens")
    _check(load().quest_rotate_tokens(cache.ref, rotation.ref, x.data_ptr(), stride, heads, cu_tokens.data_ptr(), shape[0],
                                      out.data_ptr(), out_stride, _stream_of(cache, stream)))


def quest_rotate_append_tokens(cache: Cache, rotation: Rotation, q, k_new, v_new, cu_tokens, q_out=None, stream=None):
    """q and q_out: None for keys and values only."""
    _, i32, _ = _types or _types_of_torch()
    shape = k_new.shape
    stride = _rows_of(cache, shape, k_new, cache.kv_heads, v_new)
    total, q_stride, out_stride = shape[0], 0, 0
    if q is not None and q_out is not None:
        q_shape, out_shape, heads = q.shape, q_out.shape, cache.heads
        q_stride, out_stride = _rows_of(cache, q_shape, q, heads), _rows_of(cache, out_shape, q_out, heads)
        if q_shape[0] < total or out_shape[0] < total:
            raise QuestError(-2, f"{q_shape[0]} rows of queries and {out_shape[0]} of results for {total} of keys")
    elif q is not None or q_out is not None:
        raise QuestError(-1, "q and q_out: both or neither")
    _rotation_of(cache, rotation, total)
    _plain(cache, cu_tokens, i32, cache.batch + 1, "cu_tokens")
    _check(load().quest_rotate_append_tokens(
        cache.ref, rotation.ref, _ptr(q), q_stride, _ptr(q_out), out_stride, k_new.data_ptr(), v_new.data_ptr(), stride,
        cu_tokens.data_ptr(), total, _stream_of(cache, stream)))
