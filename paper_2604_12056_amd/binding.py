"""ctypes binding of liblosa.so: the same entry points as include/losa.h, taking torch
tensors.  Argument marshalling only: every step of the path runs in the HIP kernels.
torch is used for device memory and the current stream, nothing else.

The library must have been built (python -m paper_2604_12056_amd.build, or
__graft_entry__.build()); there is no fallback path if it is missing."""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

from .build import LIB_PATH

LOSA_OK, LOSA_ERR_INVALID_ARG, LOSA_ERR_UNSUPPORTED, LOSA_ERR_WORKSPACE, LOSA_ERR_HIP = range(5)
LOSA_BF16, LOSA_F32 = 0, 1
LOSA_SEL_TOPK, LOSA_SEL_FRACTION, LOSA_SEL_THRESHOLD, LOSA_SEL_MASS = 0, 1, 2, 3

EXPORTS = ["losa_workspace_bytes", "losa_create", "losa_destroy", "losa_last_error", "losa_select_active",
           "losa_page_bounds", "losa_score_pages", "losa_sparse_attn", "losa_step", "losa_profile_enable",
           "losa_profile_read", "losa_calibration_copy", "losa_block_merge", "losa_score_pages_shared",
           "losa_select_active_static", "losa_set_tuning", "losa_calibration_read", "losa_rotate", "losa_append_kv",
           "losa_append_packed", "losa_read_packed", "losa_sparse_attn_packed", "losa_step_packed"]
(LOSA_TUNE_ATTN_WORKGROUPS, LOSA_TUNE_SELECT_ROUND, LOSA_TUNE_SCORE_ROUND, LOSA_TUNE_RANK_IN_SCORES,
 LOSA_TUNE_UNION_IN_ATTENTION, LOSA_TUNE_SHARED_TILES, LOSA_TUNE_HALF_PRECISION_VALUES) = range(7)
LOSA_ROTATE_HALVES, LOSA_ROTATE_PAIRS = 0, 1
STAGES = ["locality", "score", "topk", "attn", "merge", "bounds", "block"]


class LosaError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"losa status {status}: {text}")
        self.status = status
        self.text = text


class losa_config(C.Structure):
    _fields_ = [("max_batch", C.c_int32), ("num_q_heads", C.c_int32), ("num_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("hidden_size", C.c_int32), ("page_size", C.c_int32),
                ("block_size", C.c_int32), ("max_pages_per_seq", C.c_int32), ("max_topk_pages", C.c_int32),
                ("dtype", C.c_int32), ("sm_scale", C.c_float)]


class losa_kv(C.Structure):
    _fields_ = [("k_pages", C.c_void_p), ("v_pages", C.c_void_p), ("meta", C.c_void_p),
                ("page_indptr", C.c_void_p), ("page_indices", C.c_void_p), ("seq_lens", C.c_void_p),
                ("batch", C.c_int32), ("num_pages", C.c_int32), ("max_seq_pages", C.c_int32)]


class losa_packed_kv(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("v_codes", C.c_void_p), ("scales", C.c_void_p), ("meta", C.c_void_p),
                ("page_indptr", C.c_void_p), ("page_indices", C.c_void_p), ("seq_lens", C.c_void_p),
                ("batch", C.c_int32), ("num_pages", C.c_int32), ("max_seq_pages", C.c_int32)]


class losa_rotation(C.Structure):
    _fields_ = [("cos_sin", C.c_void_p), ("max_positions", C.c_int32), ("rotary_dim", C.c_int32), ("style", C.c_int32)]


class losa_new_tokens(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_stride", C.c_int64), ("v_stride", C.c_int64),
                ("tok_indptr", C.c_void_p), ("positions", C.c_void_p), ("num_tokens", C.c_int32), ("max_new_tokens", C.c_int32)]


_lib = None


def load_library() -> C.CDLL:
    """Loads the in-tree liblosa.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(f"{LIB_PATH} is missing: build it with `python -m paper_2604_12056_amd.build`")
    lib = C.CDLL(LIB_PATH)
    p, i32, f32, vp = C.c_void_p, C.c_int32, C.c_float, C.c_void_p
    lib.losa_workspace_bytes.restype = C.c_size_t
    lib.losa_workspace_bytes.argtypes = [C.POINTER(losa_config)]
    lib.losa_create.restype = C.c_int
    lib.losa_create.argtypes = [C.POINTER(losa_config), vp, C.c_size_t, C.POINTER(vp)]
    lib.losa_destroy.restype = C.c_int
    lib.losa_destroy.argtypes = [vp]
    lib.losa_last_error.restype = C.c_char_p
    lib.losa_last_error.argtypes = [vp]
    lib.losa_select_active.restype = C.c_int
    lib.losa_select_active.argtypes = [vp, vp, i32, p, p, C.c_int, f32, p, p, p, p]
    lib.losa_select_active_static.restype = C.c_int
    lib.losa_select_active_static.argtypes = [vp, i32, i32, i32, i32, p, p, C.c_int, f32, p, p, p, p]
    lib.losa_page_bounds.restype = C.c_int
    lib.losa_page_bounds.argtypes = [vp, vp, C.POINTER(losa_kv), i32, i32]
    lib.losa_score_pages.restype = C.c_int
    lib.losa_score_pages.argtypes = [vp, vp, C.POINTER(losa_kv), p, p, p, i32, p, p, p, i32]
    lib.losa_score_pages_shared.restype = C.c_int
    lib.losa_score_pages_shared.argtypes = [vp, vp, C.POINTER(losa_kv), p, p, p, i32, p, p, i32]
    lib.losa_sparse_attn.restype = C.c_int
    lib.losa_sparse_attn.argtypes = [vp, vp, C.POINTER(losa_kv), p, p, p, p, p, i32, p, p]
    lib.losa_step.restype = C.c_int
    lib.losa_step.argtypes = [vp, vp, C.POINTER(losa_kv), i32, p, p, p, C.c_int, f32, i32, p, p, p, p]
    lib.losa_set_tuning.restype = C.c_int
    lib.losa_set_tuning.argtypes = [vp, C.c_int, C.c_int64]
    lib.losa_profile_enable.restype = C.c_int
    lib.losa_profile_enable.argtypes = [vp, i32]
    lib.losa_profile_read.restype = C.c_int
    lib.losa_profile_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
    lib.losa_block_merge.restype = C.c_int
    lib.losa_block_merge.argtypes = [vp, vp, i32, p, p, p, p, p, p, p, p]
    i64, pk, rot, new = C.c_int64, C.POINTER(losa_packed_kv), C.POINTER(losa_rotation), C.POINTER(losa_new_tokens)
    lib.losa_rotate.restype = C.c_int
    lib.losa_rotate.argtypes = [vp, vp, rot, p, i32, p, i64, p, i64, p, i64, p, i64]
    lib.losa_append_kv.restype = C.c_int
    lib.losa_append_kv.argtypes = [vp, vp, C.POINTER(losa_kv), new, rot]
    lib.losa_append_packed.restype = C.c_int
    lib.losa_append_packed.argtypes = [vp, vp, pk, new, rot]
    lib.losa_read_packed.restype = C.c_int
    lib.losa_read_packed.argtypes = [vp, vp, pk, p, i32, i32, p, p]
    lib.losa_sparse_attn_packed.restype = C.c_int
    lib.losa_sparse_attn_packed.argtypes = [vp, vp, pk, p, p, p, p, p, i32, p, p]
    lib.losa_step_packed.restype = C.c_int
    lib.losa_step_packed.argtypes = [vp, vp, pk, i32, p, p, p, C.c_int, f32, i32, p, p, p, p]
    lib.losa_calibration_copy.restype = C.c_int
    lib.losa_calibration_copy.argtypes = [vp, vp, C.c_size_t, vp]
    lib.losa_calibration_read.restype = C.c_int
    lib.losa_calibration_read.argtypes = [vp, C.c_size_t, vp, i32, vp, vp]
    _lib = lib
    return lib


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


# The handle of the current device's current stream, asked for at every call.  A torch.cuda.Stream object made for each
# call only to read its handle takes 2.8 us of host time, this 0.36, and the smallest steps take as long to issue as to run
# (2048 tokens, 4 heads: 22.6 -> 20.9 us per step).
_current_raw_stream = None


def _stream(stream) -> Optional[int]:
    if stream is not None:
        return int(stream) or None
    global _current_raw_stream
    if _current_raw_stream is None:
        import torch
        current_device, raw_stream = torch.cuda.current_device, getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw_stream is not None:
            _current_raw_stream = lambda: raw_stream(current_device())
        else:   # not part of torch's public interface: without it, the public way
            _current_raw_stream = lambda: torch.cuda.current_stream().cuda_stream
    return _current_raw_stream() or None


class PagedKV:
    """Device tensors of one layer's paged prefix cache plus the host-side counts."""

    def __init__(self, k_pages, v_pages, meta, page_indptr, page_indices, seq_lens, max_seq_pages: int = 0):
        self.k_pages, self.v_pages, self.meta = k_pages, v_pages, meta
        self.page_indptr, self.page_indices, self.seq_lens = page_indptr, page_indices, seq_lens
        self.batch = int(seq_lens.numel())
        self.num_pages = int(k_pages.shape[0])
        self.max_seq_pages = int(max_seq_pages)

    def as_struct(self) -> losa_kv:
        return losa_kv(_ptr(self.k_pages), _ptr(self.v_pages), _ptr(self.meta), _ptr(self.page_indptr),
                       _ptr(self.page_indices), _ptr(self.seq_lens), self.batch, self.num_pages, self.max_seq_pages)


class PackedKV:
    """Device tensors of one layer's prefix cache in 4 bits (uint8 pools) plus the host-side counts."""

    def __init__(self, k_codes, v_codes, scales, meta, page_indptr, page_indices, seq_lens, max_seq_pages: int = 0):
        self.k_codes, self.v_codes, self.scales, self.meta = k_codes, v_codes, scales, meta
        self.page_indptr, self.page_indices, self.seq_lens = page_indptr, page_indices, seq_lens
        self.batch = int(seq_lens.numel())
        self.num_pages = int(k_codes.shape[0])
        self.max_seq_pages = int(max_seq_pages)

    def as_struct(self) -> losa_packed_kv:
        meta = self.meta
        return losa_packed_kv(self.k_codes.data_ptr(), self.v_codes.data_ptr(), self.scales.data_ptr(),
                              None if meta is None else meta.data_ptr(), self.page_indptr.data_ptr(), self.page_indices.data_ptr(),
                              self.seq_lens.data_ptr(), self.batch, self.num_pages, self.max_seq_pages)

    def for_scoring(self) -> PagedKV:
        """The cache as losa_score_pages and losa_score_pages_shared take it: they read its page table and bounds only."""
        return PagedKV(self.k_codes, self.v_codes, self.meta, self.page_indptr, self.page_indices, self.seq_lens, self.max_seq_pages)


class Rotation:
    """A rotation's table (float32 [positions, rotary_dim]: cosines, then sines) and which channels make a pair."""

    def __init__(self, cos_sin, style: int = LOSA_ROTATE_HALVES):
        self.cos_sin, self.style = cos_sin, int(style)
        self.max_positions, self.rotary_dim = int(cos_sin.shape[0]), int(cos_sin.shape[1])

    def as_struct(self) -> losa_rotation:
        return losa_rotation(_ptr(self.cos_sin), self.max_positions, self.rotary_dim, self.style)


class Context:
    """Owns the losa_ctx handle and the torch tensor that backs its workspace."""

    def __init__(self, handle: int, workspace, cfg: losa_config):
        self.handle, self.workspace, self.cfg = handle, workspace, cfg
        # what every call with rows of heads asks for (a structure's field takes as long as a launch's tenth)
        self.q_heads, self.kv_heads, self.head_dim = cfg.num_q_heads, cfg.num_kv_heads, cfg.head_dim
        self.element_size = 2 if cfg.dtype == LOSA_BF16 else 4

    def close(self):
        if self.handle:
            load_library().losa_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _check(ctx: Optional[Context], status: int):
    if status != LOSA_OK:
        text = load_library().losa_last_error(ctx.handle if ctx else None)
        raise LosaError(status, text.decode() if text else "")


def make_config(*, max_batch, num_q_heads, num_kv_heads, head_dim, hidden_size, page_size, block_size,
                max_pages_per_seq, max_topk_pages, dtype=LOSA_BF16, sm_scale=0.0) -> losa_config:
    return losa_config(max_batch, num_q_heads, num_kv_heads, head_dim, hidden_size, page_size, block_size,
                       max_pages_per_seq, max_topk_pages, dtype, sm_scale)


def losa_workspace_bytes(cfg: losa_config) -> int:
    return int(load_library().losa_workspace_bytes(C.byref(cfg)))


def losa_create(cfg: losa_config, device="cuda:0") -> Context:
    """Allocates the workspace with torch on `device` and creates the context."""
    import torch
    lib = load_library()
    nbytes = lib.losa_workspace_bytes(C.byref(cfg))
    if nbytes == 0:
        # let the library say what is wrong with the configuration
        out = C.c_void_p()
        _check(None, lib.losa_create(C.byref(cfg), None, 0, C.byref(out)))
    ws = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
    off = (-ws.data_ptr()) % 256
    out = C.c_void_p()
    _check(None, lib.losa_create(C.byref(cfg), ws.data_ptr() + off, nbytes, C.byref(out)))
    return Context(out.value, ws, cfg)


def losa_destroy(ctx: Context):
    ctx.close()


def losa_select_active(ctx: Context, h_cur, h_prev, mode: int, param: float, delta, mask, active_idx, active_count,
                       batch: Optional[int] = None, stream=None):
    batch = int(active_count.numel()) if batch is None else batch
    _check(ctx, load_library().losa_select_active(ctx.handle, _stream(stream), batch, _ptr(h_cur), _ptr(h_prev),
                                                 mode, param, _ptr(delta), _ptr(mask), _ptr(active_idx),
                                                 _ptr(active_count)))


def losa_select_active_static(dtype: int, batch: int, block_size: int, hidden_size: int, h_cur, h_prev, mode: int,
                              param: float, delta, mask, active_idx, active_count, stream=None):
    """The allocation-free variant: no context, no workspace (ticket counters live in the library)."""
    _check(None, load_library().losa_select_active_static(_stream(stream), dtype, batch, block_size, hidden_size,
                                                         _ptr(h_cur), _ptr(h_prev), mode, param, _ptr(delta),
                                                         _ptr(mask), _ptr(active_idx), _ptr(active_count)))


def losa_page_bounds(ctx: Context, kv: PagedKV, first_logical_page: int = 0, num_logical_pages: int = -1, stream=None):
    s = kv.as_struct()
    _check(ctx, load_library().losa_page_bounds(ctx.handle, _stream(stream), C.byref(s), first_logical_page,
                                               num_logical_pages))


def losa_score_pages(ctx: Context, kv: PagedKV, q, active_idx, active_count, topk_pages: int, topk_out, sel_pages,
                     sel_count, cap: int, stream=None):
    s = kv.as_struct()
    _check(ctx, load_library().losa_score_pages(ctx.handle, _stream(stream), C.byref(s), _ptr(q), _ptr(active_idx),
                                               _ptr(active_count), topk_pages, _ptr(topk_out), _ptr(sel_pages),
                                               _ptr(sel_count), cap))


def losa_score_pages_shared(ctx: Context, kv: PagedKV, q, active_idx, active_count, topk_pages: int, sel_pages,
                            sel_count, cap: int, stream=None):
    s = kv.as_struct()
    _check(ctx, load_library().losa_score_pages_shared(ctx.handle, _stream(stream), C.byref(s), _ptr(q),
                                                      _ptr(active_idx), _ptr(active_count), topk_pages,
                                                      _ptr(sel_pages), _ptr(sel_count), cap))


def losa_sparse_attn(ctx: Context, kv: PagedKV, q, active_idx, active_count, sel_pages, sel_count, cap: int, o_p,
                     lse_p, stream=None):
    s = kv.as_struct()
    _check(ctx, load_library().losa_sparse_attn(ctx.handle, _stream(stream), C.byref(s), _ptr(q), _ptr(active_idx),
                                               _ptr(active_count), _ptr(sel_pages), _ptr(sel_count), cap, _ptr(o_p),
                                               _ptr(lse_p)))


def losa_step(ctx: Context, kv: PagedKV, step_index: int, h_cur, h_prev, q, mode: int, param: float,
              topk_pages: int, o_p, lse_p, mask=None, sel_count=None, stream=None):
    s = kv.as_struct()
    _check(ctx, load_library().losa_step(ctx.handle, _stream(stream), C.byref(s), step_index, _ptr(h_cur),
                                        _ptr(h_prev), _ptr(q), mode, param, topk_pages, _ptr(o_p), _ptr(lse_p),
                                        _ptr(mask), _ptr(sel_count)))


def _row_stride(t, ctx: Context, tokens: int, heads: int, what: str) -> int:
    """Elements between consecutive tokens of a [tokens, heads, d] tensor of the context's type, whose heads have to lie together."""
    d = ctx.head_dim
    if t.shape != (tokens, heads, d) or t.element_size() != ctx.element_size:
        raise LosaError(LOSA_ERR_INVALID_ARG, f"{what} is not a [{tokens}, {heads}, {d}] tensor of the context's type")
    if tokens == 0:
        return 0
    if t.is_contiguous():
        return heads * d if tokens > 1 else 0
    row, head, channel = t.stride()
    if channel != 1 or (head != d and heads > 1):
        raise LosaError(LOSA_ERR_INVALID_ARG, f"{what}: the heads of a token do not lie one behind the other")
    if tokens == 1:
        return 0
    if row == 0:
        raise LosaError(LOSA_ERR_INVALID_ARG, f"{what}: all tokens are the same row")
    return row


def losa_rotate(ctx: Context, rotation: Rotation, positions, q=None, q_out=None, k=None, k_out=None, stream=None):
    """q [tokens, Hq, d] and / or k [tokens, Hkv, d], turned by the positions (int32 [tokens]) into q_out / k_out (the inputs
    themselves, if need be)."""
    n, qs, qo, ks, ko = positions.numel(), 0, 0, 0, 0
    if q is not None:
        qs = _row_stride(q, ctx, n, ctx.q_heads, "q")
    if q_out is not None:
        qo = _row_stride(q_out, ctx, n, ctx.q_heads, "q_out")
    if k is not None:
        ks = _row_stride(k, ctx, n, ctx.kv_heads, "k")
    if k_out is not None:
        ko = _row_stride(k_out, ctx, n, ctx.kv_heads, "k_out")
    _check(ctx, load_library().losa_rotate(ctx.handle, _stream(stream), C.byref(rotation.as_struct()), positions.data_ptr(), n, _ptr(q), qs,
                                          _ptr(q_out), qo, _ptr(k), ks, _ptr(k_out), ko))


def _new_tokens(ctx: Context, k, v, tok_indptr, positions, max_new_tokens: int) -> losa_new_tokens:
    n = k.shape[0]
    if positions is not None and positions.numel() != n:
        raise LosaError(LOSA_ERR_INVALID_ARG, f"{positions.numel()} positions for {n} tokens")
    return losa_new_tokens(k.data_ptr(), v.data_ptr(), _row_stride(k, ctx, n, ctx.kv_heads, "k"), _row_stride(v, ctx, n, ctx.kv_heads, "v"),
                           tok_indptr.data_ptr(), _ptr(positions), n, max_new_tokens)


def losa_append_kv(ctx: Context, kv: PagedKV, k, v, tok_indptr, rotation: Optional[Rotation] = None, positions=None,
                   max_new_tokens: int = 0, stream=None):
    """Tokens k, v [tokens, Hkv, d] (row strides as they are) into the pages and bounds of `kv`, whose seq_lens count them already."""
    _check(ctx, load_library().losa_append_kv(ctx.handle, _stream(stream), C.byref(kv.as_struct()),
                                             C.byref(_new_tokens(ctx, k, v, tok_indptr, positions, max_new_tokens)),
                                             None if rotation is None else C.byref(rotation.as_struct())))


def losa_append_packed(ctx: Context, kv: PackedKV, k, v, tok_indptr, rotation: Optional[Rotation] = None, positions=None,
                       max_new_tokens: int = 0, stream=None):
    """The same into a 4-bit cache."""
    _check(ctx, load_library().losa_append_packed(ctx.handle, _stream(stream), C.byref(kv.as_struct()),
                                                 C.byref(_new_tokens(ctx, k, v, tok_indptr, positions, max_new_tokens)),
                                                 None if rotation is None else C.byref(rotation.as_struct())))


def losa_read_packed(ctx: Context, kv: PackedKV, tok_indptr, k_out, v_out, max_tokens: int = 0, stream=None):
    """The last tokens of every sequence of a 4-bit cache into k_out / v_out [tokens, Hkv, d] (contiguous; either may be None)."""
    one = k_out if k_out is not None else v_out
    n = 0 if one is None else one.shape[0]
    shape = (n, ctx.kv_heads, ctx.head_dim)
    for t in (k_out, v_out):
        if t is not None and (t.shape != shape or t.element_size() != ctx.element_size or not t.is_contiguous()):
            raise LosaError(LOSA_ERR_INVALID_ARG, f"an output is not a contiguous {list(shape)} tensor of the context's type")
    _check(ctx, load_library().losa_read_packed(ctx.handle, _stream(stream), C.byref(kv.as_struct()), tok_indptr.data_ptr(), n, max_tokens,
                                               _ptr(k_out), _ptr(v_out)))


def losa_sparse_attn_packed(ctx: Context, kv: PackedKV, q, active_idx, active_count, sel_pages, sel_count, cap: int, o_p, lse_p,
                            stream=None):
    s = kv.as_struct()
    _check(ctx, load_library().losa_sparse_attn_packed(ctx.handle, _stream(stream), C.byref(s), _ptr(q), _ptr(active_idx),
                                                      _ptr(active_count), _ptr(sel_pages), _ptr(sel_count), cap, _ptr(o_p),
                                                      _ptr(lse_p)))


def losa_step_packed(ctx: Context, kv: PackedKV, step_index: int, h_cur, h_prev, q, mode: int, param: float, topk_pages: int, o_p, lse_p,
                     mask=None, sel_count=None, stream=None):
    s = kv.as_struct()
    _check(ctx, load_library().losa_step_packed(ctx.handle, _stream(stream), C.byref(s), step_index, _ptr(h_cur), _ptr(h_prev), _ptr(q),
                                               mode, param, topk_pages, _ptr(o_p), _ptr(lse_p), _ptr(mask), _ptr(sel_count)))


def losa_set_tuning(ctx: Context, knob: int, value: int):
    _check(ctx, load_library().losa_set_tuning(ctx.handle, knob, int(value)))


def losa_profile_enable(ctx: Context, enable: bool):
    _check(ctx, load_library().losa_profile_enable(ctx.handle, 1 if enable else 0))


def losa_profile_read(ctx: Context):
    """-> ({stage: milliseconds}, {stage: launches}) since the last read."""
    ms = (C.c_double * len(STAGES))()
    cnt = (C.c_int64 * len(STAGES))()
    _check(ctx, load_library().losa_profile_read(ctx.handle, ms, cnt))
    return dict(zip(STAGES, list(ms))), dict(zip(STAGES, list(cnt)))


def losa_calibration_copy(dst, src, stream=None):
    """Plain copy of src into dst (same byte size): the known-size reference for byte counters."""
    nbytes = src.numel() * src.element_size()
    _check(None, load_library().losa_calibration_copy(_ptr(dst), _ptr(src), nbytes, _stream(stream)))


def losa_calibration_read(pool, tile_bytes: int, tile_ids, sink, stream=None):
    """Read-only stream over the tiles of `pool` listed in tile_ids (int32 tensor); nothing is written."""
    _check(None, load_library().losa_calibration_read(_ptr(pool), tile_bytes, _ptr(tile_ids), int(tile_ids.numel()),
                                                     _ptr(sink), _stream(stream)))


def losa_block_merge(ctx: Context, q, k_b, v_b, o_p, lse_p, out, o_b=None, lse_b=None, batch: Optional[int] = None,
                     stream=None):
    batch = int(lse_p.shape[0] // ctx.cfg.block_size) if batch is None else batch
    _check(ctx, load_library().losa_block_merge(ctx.handle, _stream(stream), batch, _ptr(q), _ptr(k_b), _ptr(v_b),
                                               _ptr(o_p), _ptr(lse_p), _ptr(out), _ptr(o_b), _ptr(lse_b)))
