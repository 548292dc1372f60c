"""ctypes binding of libsagekv.so (include/sagekv.h).

Argument marshalling only (the hot calls' in C, csrc/marshal.cpp): every function below has the name and the meaning of
the C entry point it calls, takes torch CUDA tensors for the device buffers and
passes their pointers, strides and the current CUDA stream through.  Nothing is
computed here, and there is no fallback: importing this module raises if the
library has not been built (`python -m paper_2503_08879_b200.build`), and every
call raises `SagekvError` on a non-zero return code.
"""

from __future__ import annotations

import ctypes as C
import os

import torch

# SAGEKV_LIB selects another build of the same interface (the checked build, libsagekv_checked.so)
_LIB_PATH = os.environ.get("SAGEKV_LIB") or os.path.join(os.path.dirname(os.path.abspath(__file__)), "libsagekv.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError(
        f"{_LIB_PATH} is missing: build it with `python -m paper_2503_08879_b200.build` "
        "(nvcc, sm_100a). There is no CPU or PyTorch fallback.")
lib = C.CDLL(_LIB_PATH)

try:
    from . import _marshal
except ImportError as e:
    raise ImportError("paper_2503_08879_b200/_marshal is missing for this interpreter: build it with "
                      "`python -m paper_2503_08879_b200.build`") from e

OK, ERR_INVALID, ERR_ALIGN, ERR_UNSUPPORTED, ERR_CUDA, ERR_NOMEM = 0, -1, -2, -3, -4, -5
ERR_TOO_LARGE, ERR_TIMEOUT, ERR_BOUNDS, ERR_DEVICE = -6, -7, -8, -9


class Shape(C.Structure):
    _fields_ = [("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("batch", C.c_int32), ("softmax_scale", C.c_float)]


class Strides(C.Structure):
    _fields_ = [("batch_stride", C.c_int64), ("head_stride", C.c_int64), ("token_stride", C.c_int64)]


class CacheState(C.Structure):
    _fields_ = [("n_init", C.c_int32), ("k_q", C.c_int32), ("n_sel", C.c_int32), ("n_recent", C.c_int32),
                ("ring_len", C.c_int32), ("len", C.c_int32), ("d_step", C.c_void_p)]


class Rows(C.Structure):
    _fields_ = [("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class RopePlan(C.Structure):
    """Rotary positions as the kernels take them (sagekv_rope_plan); made by sagekv_rope_plan or sagekv_rope_plan_from."""
    _fields_ = [("rotary_dim", C.c_int32), ("interleaved", C.c_int32), ("amplitude", C.c_float), ("reserved", C.c_int32),
                ("turns", C.c_uint64 * 64)]


class RopeScaling(C.Structure):
    _fields_ = [("kind", C.c_int32), ("reserved", C.c_int32), ("factor", C.c_double), ("low", C.c_double), ("high", C.c_double),
                ("original_ctx", C.c_double), ("amplitude", C.c_double)]


ROPE_KINDS = {"none": 0, "linear": 1, "base": 2, "bands": 3, "yarn": 4}
CACHE_BF16, CACHE_E4M3 = 0, 1

_vp, _i32, _i64 = C.c_void_p, C.c_int32, C.c_int64


class PagedCache(C.Structure):
    """One layer's full cache in pages: the C struct sagekv_paged_cache, and the tensors that it points to.

      k_pages, v_pages   [n_pages, H_kv, page_size, 128], torch.bfloat16 or torch.float8_e4m3fn, last dimension contiguous, the same
                         strides (other orders of the first three dimensions by a permuted view)
      block_table        int32 [n_seqs, max_pages], last dimension contiguous
      seq_lens           int32 [n_seqs], contiguous; wanted by paged_attn alone
      k_scale, v_scale   fp32 [H_kv], contiguous; 8-bit caches, value = code * scale (None: 1)
    """
    _fields_ = [("k_pages", _vp), ("v_pages", _vp), ("page_stride", _i64), ("head_stride", _i64), ("token_stride", _i64),
                ("block_table", _vp), ("table_stride", _i64), ("seq_lens", _vp), ("k_scale", _vp), ("v_scale", _vp),
                ("n_pages", _i32), ("page_size", _i32), ("max_pages", _i32), ("n_seqs", _i32), ("dtype", _i32)]

    def __init__(self, k_pages, v_pages, block_table, seq_lens=None, k_scale=None, v_scale=None):
        if k_pages.dim() != 4 or k_pages.stride(3) != 1 or k_pages.shape[3] != 128:
            raise ValueError("expected pages [n_pages, H_kv, page_size, 128] with contiguous last dimension")
        if v_pages.shape != k_pages.shape or v_pages.stride() != k_pages.stride() or v_pages.dtype != k_pages.dtype:
            raise ValueError("expected v_pages with the shape, the strides and the type of k_pages")
        if k_pages.dtype not in (torch.bfloat16, torch.float8_e4m3fn):
            raise ValueError("expected pages of torch.bfloat16 or torch.float8_e4m3fn")
        if block_table.dim() != 2 or block_table.dtype != torch.int32 or (block_table.shape[1] > 1 and block_table.stride(1) != 1):
            raise ValueError("expected an int32 block table [n_seqs, max_pages] with contiguous rows")
        n_seqs, max_pages = block_table.shape
        if seq_lens is not None and (seq_lens.dtype != torch.int32 or tuple(seq_lens.shape) != (n_seqs,) or not seq_lens.is_contiguous()):
            raise ValueError("expected contiguous int32 seq_lens, one per row of the block table")
        for s in (k_scale, v_scale):
            if s is not None and (s.dtype != torch.float32 or tuple(s.shape) != (k_pages.shape[1],) or not s.is_contiguous()):
                raise ValueError("expected contiguous float32 scales, one per KV head")
        self.tensors = (k_pages, v_pages, block_table, seq_lens, k_scale, v_scale)
        self.n_kv_heads = k_pages.shape[1]
        if any(t is not None and t.device != k_pages.device for t in self.tensors):
            raise ValueError("expected all tensors of a cache on one device")
        self.device_index = k_pages.get_device()
        ptr = lambda t: None if t is None else t.data_ptr()
        super().__init__(ptr(k_pages), ptr(v_pages), k_pages.stride(0), k_pages.stride(1), k_pages.stride(2), ptr(block_table),
                         block_table.stride(0) if n_seqs > 1 else max_pages, ptr(seq_lens), ptr(k_scale), ptr(v_scale), k_pages.shape[0],
                         k_pages.shape[2], max_pages, n_seqs, CACHE_BF16 if k_pages.dtype == torch.bfloat16 else CACHE_E4M3)


lib.sagekv_create.argtypes = [C.POINTER(_vp), C.POINTER(Shape), _i64, _i32]
lib.sagekv_destroy.argtypes = [_vp]
lib.sagekv_budget_split.argtypes = [_i32, _i32, C.POINTER(_i32), C.POINTER(_i32), C.POINTER(_i32)]
lib.sagekv_score.argtypes = [_vp, _vp, _vp, Strides, _i64, _i32, _i32, _vp, _i64, _vp]
lib.sagekv_select_compact.argtypes = [_vp, _vp, _i64, _vp, _vp, Strides, _i64, _i32, _i32, _i32,
                                      _vp, _vp, _vp, Strides, C.POINTER(CacheState), _vp]
lib.sagekv_decode_attn.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, Strides, C.POINTER(CacheState), _vp, _vp, _vp]
lib.sagekv_score_static.argtypes = [C.POINTER(Shape), _vp, _vp, Strides, _i64, _i32, _i32, _vp, _i64, _vp]
lib.sagekv_score_static.restype = C.c_int
lib.sagekv_set_overlap.argtypes = [_vp, C.c_int]
lib.sagekv_set_overlap.restype = C.c_int
lib.sagekv_set_decode_variant.argtypes = [_vp, C.c_int]
lib.sagekv_set_decode_variant.restype = C.c_int
lib.sagekv_set_select_overlap.argtypes = [_vp, C.c_int]
lib.sagekv_set_select_overlap.restype = C.c_int
lib.sagekv_set_select_hint.argtypes = [_vp, C.c_int, _i32]
lib.sagekv_set_select_hint.restype = C.c_int
lib.sagekv_scores_row_stride.argtypes = [_vp, _i64, _i32, _i32]
lib.sagekv_scores_row_stride.restype = _i64
lib.sagekv_set_group_mode.argtypes = [_vp, C.c_int]
lib.sagekv_set_group_mode.restype = C.c_int
lib.sagekv_pool_scores.argtypes = [_vp, _vp, _i64, _i64, _i32, _i32, _vp, _i64, _vp]
lib.sagekv_pool_scores.restype = C.c_int
lib.sagekv_compact_window_rope.argtypes = [_vp, _vp, _vp, Strides, _i64, _i32, _i32, C.c_float, _vp, _vp, Strides,
                                           C.POINTER(CacheState), _vp]
lib.sagekv_compact_window_rope.restype = C.c_int
lib.sagekv_quest_build.argtypes = [_vp, _vp, Strides, _i64, _i32, _i32, _vp, _vp, _vp]
lib.sagekv_quest_build.restype = C.c_int
lib.sagekv_quest_bounds.argtypes = [_vp, _vp, _vp, _vp, _i64, _vp, _i64, _vp]
lib.sagekv_quest_bounds.restype = C.c_int
lib.sagekv_select_topk.argtypes = [_vp, _vp, _i64, _i64, _i32, _vp, _vp]
lib.sagekv_select_topk.restype = C.c_int
lib.sagekv_paged_check.argtypes = [C.POINTER(Shape), C.POINTER(PagedCache)]
lib.sagekv_paged_check.restype = C.c_int
lib.sagekv_paged_offset.argtypes = [C.POINTER(PagedCache), _i32, _i32, _i64]
lib.sagekv_paged_offset.restype = _i64
lib.sagekv_rope_plan_init.argtypes = [C.POINTER(RopePlan), _i32, _i32, C.c_double, C.POINTER(RopeScaling), C.POINTER(C.c_double)]
lib.sagekv_rope_plan_init.restype = C.c_int
lib.sagekv_rope_plan_from.argtypes = [C.POINTER(RopePlan), _i32, _i32, C.POINTER(C.c_double), C.c_float]
lib.sagekv_rope_plan_from.restype = C.c_int
lib.sagekv_rope.argtypes = [_vp, C.POINTER(RopePlan), _vp, Rows, _i64, _i32, _vp, _vp, Rows, _vp]
lib.sagekv_rope.restype = C.c_int
lib.sagekv_paged_append.argtypes = [_vp, C.POINTER(PagedCache), _vp, _vp, Rows, _i64, _vp, _vp, C.POINTER(RopePlan), _vp, Rows, _vp, Rows, _vp]
lib.sagekv_paged_append.restype = C.c_int
lib.sagekv_paged_attn.argtypes = [_vp, _vp, _i64, C.POINTER(PagedCache), _vp, _vp, _vp]
lib.sagekv_paged_attn.restype = C.c_int
lib.sagekv_paged_score.argtypes = [_vp, _vp, C.POINTER(PagedCache), _i64, _i32, _i32, _vp, _i64, _vp]
lib.sagekv_paged_score.restype = C.c_int
lib.sagekv_paged_compact.argtypes = [_vp, _vp, C.POINTER(PagedCache), _i64, _i32, _i32, _i32, _vp, _vp, Strides, C.POINTER(CacheState), _vp]
lib.sagekv_paged_compact.restype = C.c_int
lib.sagekv_status.argtypes = [_vp, C.POINTER(_i32)]
lib.sagekv_status.restype = C.c_int
lib.sagekv_status_code.argtypes = [_i32]
lib.sagekv_status_code.restype = C.c_int
lib.sagekv_checked_build.argtypes = []
lib.sagekv_checked_build.restype = C.c_int
lib.sagekv_strerror.argtypes = [C.c_int]
lib.sagekv_strerror.restype = C.c_char_p
lib.sagekv_last_cuda_error.argtypes = [_vp]
for _f in (lib.sagekv_create, lib.sagekv_destroy, lib.sagekv_budget_split, lib.sagekv_score,
           lib.sagekv_select_compact, lib.sagekv_decode_attn, lib.sagekv_last_cuda_error):
    _f.restype = C.c_int


class SagekvError(RuntimeError):
    def __init__(self, code: int, where: str, cuda_error: int = 0):
        self.code = code
        msg = f"{where}: {lib.sagekv_strerror(code).decode()} ({code})"
        if cuda_error:
            msg += f", cudaError {cuda_error}"
        super().__init__(msg)


def _check(code: int, where: str, ctx=None):
    if code != OK:
        raise SagekvError(code, where, lib.sagekv_last_cuda_error(ctx) if ctx else 0)


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


try:        # the handle alone: torch.cuda.current_stream() builds a stream object first
    _device_now, _stream_of_device = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
except AttributeError:
    def _stream_handle() -> int:
        return torch.cuda.current_stream().cuda_stream
else:
    def _stream_handle() -> int:
        return _stream_of_device(_device_now())


def _stream():
    return C.c_void_p(_stream_handle())


_marshal.bind(*(C.cast(f, _vp).value for f in (lib.sagekv_score, lib.sagekv_select_compact, lib.sagekv_decode_attn,
                                               lib.sagekv_pool_scores, lib.sagekv_quest_bounds, lib.sagekv_select_topk)),
              _stream_handle, C.ArgumentError)


_marshal.bind_paged(*(C.cast(f, _vp).value for f in (lib.sagekv_rope, lib.sagekv_paged_append, lib.sagekv_paged_attn, lib.sagekv_paged_score,
                                                     lib.sagekv_paged_compact)))


def _kv_strides(t: torch.Tensor) -> Strides:
    """Strides of a [B, H_kv, tokens, 128] tensor whose last dimension is contiguous."""
    if t.dim() != 4 or t.stride(3) != 1:
        raise ValueError("expected a [B, H_kv, tokens, head_dim] tensor with contiguous head_dim")
    return Strides(t.stride(0), t.stride(1), t.stride(2))


def sagekv_budget_split(B: int, G: int):
    a, b, c = _i32(), _i32(), _i32()
    _check(lib.sagekv_budget_split(B, G, C.byref(a), C.byref(b), C.byref(c)), "sagekv_budget_split")
    return a.value, b.value, c.value


def sagekv_create(n_q_heads: int, n_kv_heads: int, head_dim: int, batch: int, max_ctx: int, max_len: int,
                  softmax_scale: float = 0.0):
    h = _vp()
    shape = Shape(n_q_heads, n_kv_heads, head_dim, batch, softmax_scale)
    _check(lib.sagekv_create(C.byref(h), C.byref(shape), max_ctx, max_len), "sagekv_create")
    return h


def sagekv_destroy(ctx):
    _check(lib.sagekv_destroy(ctx), "sagekv_destroy")


def sagekv_score(ctx, q_last, K, n_ctx: int, n_init: int, n_recent: int, scores, scores_row_stride: int):
    code = _marshal.score(ctx, q_last, K, n_ctx, n_init, n_recent, scores, scores_row_stride)
    if code:
        _check(code, "sagekv_score", ctx)


def sagekv_set_overlap(ctx, mode: int):
    _check(lib.sagekv_set_overlap(ctx, mode), "sagekv_set_overlap", ctx)


def sagekv_set_decode_variant(ctx, variant: int):
    _check(lib.sagekv_set_decode_variant(ctx, variant), "sagekv_set_decode_variant", ctx)


def sagekv_set_select_overlap(ctx, mode: int):
    _check(lib.sagekv_set_select_overlap(ctx, mode), "sagekv_set_select_overlap", ctx)


def sagekv_set_select_hint(ctx, mode: int, k: int = 0):
    _check(lib.sagekv_set_select_hint(ctx, mode, k), "sagekv_set_select_hint", ctx)


def sagekv_scores_row_stride(ctx, n_ctx: int, n_init: int, n_recent: int) -> int:
    r = lib.sagekv_scores_row_stride(ctx, n_ctx, n_init, n_recent)
    if r < 0:
        _check(int(r), "sagekv_scores_row_stride", ctx)
    return int(r)


def sagekv_set_group_mode(ctx, mode: int):
    _check(lib.sagekv_set_group_mode(ctx, mode), "sagekv_set_group_mode", ctx)


def sagekv_pool_scores(ctx, scores, scores_row_stride: int, n_ctx: int, n_init: int, n_recent: int, pooled,
                       pooled_row_stride: int):
    code = _marshal.pool_scores(ctx, scores, scores_row_stride, n_ctx, n_init, n_recent, pooled, pooled_row_stride)
    if code:
        _check(code, "sagekv_pool_scores", ctx)


def sagekv_compact_window_rope(ctx, K_pre, V, n_ctx: int, n_init: int, n_recent: int, rope_theta: float, Kc, Vc,
                               state: CacheState):
    _check(lib.sagekv_compact_window_rope(ctx, _ptr(K_pre), _ptr(V), _kv_strides(K_pre), n_ctx, n_init, n_recent,
                                          rope_theta, _ptr(Kc), _ptr(Vc), _kv_strides(Kc), C.byref(state), _stream()),
           "sagekv_compact_window_rope", ctx)


def sagekv_quest_build(ctx, K, n_ctx: int, n_init: int, n_recent: int, kmin, kmax):
    _check(lib.sagekv_quest_build(ctx, _ptr(K), _kv_strides(K), n_ctx, n_init, n_recent, _ptr(kmin), _ptr(kmax), _stream()),
           "sagekv_quest_build", ctx)


def sagekv_quest_bounds(ctx, q, kmin, kmax, n_blocks: int, bounds, bounds_row_stride: int):
    code = _marshal.quest_bounds(ctx, q, kmin, kmax, n_blocks, bounds, bounds_row_stride)
    if code:
        _check(code, "sagekv_quest_bounds", ctx)


def sagekv_select_topk(ctx, scores, scores_row_stride: int, n: int, k_q: int, idx):
    code = _marshal.select_topk(ctx, scores, scores_row_stride, n, k_q, idx)
    if code:
        _check(code, "sagekv_select_topk", ctx)


def sagekv_status(ctx) -> int:
    """The context's device status word (0 = clean); raises SagekvError if any bit is set."""
    bits = _i32(0)
    code = lib.sagekv_status(ctx, C.byref(bits))
    if code != OK:
        e = SagekvError(code, "sagekv_status (word %d)" % bits.value, lib.sagekv_last_cuda_error(ctx))
        e.bits = bits.value
        raise e
    return bits.value


def sagekv_score_static(shape: Shape, q_last, K, n_ctx: int, n_init: int, n_recent: int, scores,
                        scores_row_stride: int):
    """sagekv_score without a context or any allocation: the partials live in the library's fixed array."""
    _check(lib.sagekv_score_static(C.byref(shape), _ptr(q_last), _ptr(K), _kv_strides(K), n_ctx, n_init, n_recent,
                                   _ptr(scores), scores_row_stride, _stream()), "sagekv_score_static")


def sagekv_rope_plan(rotary_dim: int, interleaved: bool, theta: float, scaling: dict = None) -> RopePlan:
    """A rotary plan from a base and a scaling rule: dict(kind="linear" | "base" | "bands" | "yarn", factor=...,
    low=..., high=..., original_ctx=..., amplitude=...), the entries its kind takes (None: unscaled)."""
    plan, rule = RopePlan(), None
    if scaling is not None:
        extra = set(scaling) - {"kind", "factor", "low", "high", "original_ctx", "amplitude"}
        if extra or scaling.get("kind") not in ROPE_KINDS:
            raise ValueError("unknown scaling rule: %r" % (scaling,))
        rule = RopeScaling(ROPE_KINDS[scaling["kind"]], 0, scaling.get("factor", 1.0), scaling.get("low", 0.0), scaling.get("high", 0.0),
                           scaling.get("original_ctx", 0.0), scaling.get("amplitude", 0.0))
    _check(lib.sagekv_rope_plan_init(C.byref(plan), rotary_dim, bool(interleaved), theta, None if rule is None else C.byref(rule), None),
           "sagekv_rope_plan_init")
    return plan


def sagekv_rope_plan_from(rotary_dim: int, interleaved: bool, inv_freq, amplitude: float = 1.0) -> RopePlan:
    """A rotary plan from rotary_dim / 2 frequencies in radians per position."""
    f = [float(x) for x in inv_freq]
    if len(f) != rotary_dim // 2:
        raise ValueError("expected rotary_dim / 2 frequencies")
    plan = RopePlan()
    _check(lib.sagekv_rope_plan_from(C.byref(plan), rotary_dim, bool(interleaved), (C.c_double * len(f))(*f), amplitude), "sagekv_rope_plan_from")
    return plan


def sagekv_paged_check(shape: Shape, cache: PagedCache):
    _check(lib.sagekv_paged_check(C.byref(shape), C.byref(cache)), "sagekv_paged_check")


def sagekv_paged_offset(cache: PagedCache, page: int, head: int, position: int) -> int:
    at = lib.sagekv_paged_offset(C.byref(cache), page, head, position)
    if at < 0:
        _check(int(at), "sagekv_paged_offset")
    return int(at)


def sagekv_rope(ctx, plan: RopePlan, x, n_tokens: int, n_heads: int, positions, out):
    code = _marshal.rope(ctx, plan, x, n_tokens, n_heads, positions, out)
    if code:
        _check(code, "sagekv_rope", ctx)


def sagekv_paged_append(ctx, cache: PagedCache, k, v, n_tokens: int, positions, seqs=None, plan: RopePlan = None, q=None, q_out=None):
    code = _marshal.paged_append(ctx, cache, k, v, n_tokens, positions, seqs, plan, q, q_out)
    if code:
        _check(code, "sagekv_paged_append", ctx)


def sagekv_paged_attn(ctx, q, cache: PagedCache, out, lse=None):
    code = _marshal.paged_attn(ctx, q, cache, out, lse)
    if code:
        _check(code, "sagekv_paged_attn", ctx)


def sagekv_paged_score(ctx, q_last, cache: PagedCache, n_ctx: int, n_init: int, n_recent: int, scores, scores_row_stride: int):
    code = _marshal.paged_score(ctx, q_last, cache, n_ctx, n_init, n_recent, scores, scores_row_stride)
    if code:
        _check(code, "sagekv_paged_score", ctx)


def sagekv_paged_compact(ctx, idx, cache: PagedCache, n_ctx: int, n_init: int, n_recent: int, k: int, Kc, Vc, state: CacheState):
    code = _marshal.paged_compact(ctx, idx, cache, n_ctx, n_init, n_recent, k, Kc, Vc, state)
    if code:
        _check(code, "sagekv_paged_compact", ctx)


def sagekv_select_compact(ctx, scores, scores_row_stride: int, K, V, n_ctx: int, n_init: int, n_recent: int, k: int,
                          idx, Kc, Vc, state: CacheState):
    code = _marshal.select_compact(ctx, scores, scores_row_stride, K, V, n_ctx, n_init, n_recent, k, idx, Kc, Vc, state)
    if code:
        _check(code, "sagekv_select_compact", ctx)


def sagekv_decode_attn(ctx, q, k_new, v_new, Kc, Vc, state: CacheState, out, lse=None):
    code = _marshal.decode_attn(ctx, q, k_new, v_new, Kc, Vc, state, out, lse)
    if code:
        _check(code, "sagekv_decode_attn", ctx)


_INT32, _BF16, _FP32 = torch.int32, torch.bfloat16, torch.float32
_placed, _placed_row, _holds_rows = _marshal.placed, _marshal.placed_row, _marshal.holds_rows


def _holds(Kc, Vc, sk, rows: int) -> bool:
    """Are Kc and Vc bf16 [B, H_kv, >= rows, 128] on the context's device, laid out alike?"""
    return _holds_rows(Kc, Vc, sk.shape[3], sk.shape[1], rows) and _placed(_BF16, sk.device_index, Kc, Vc)


class Layer:
    """Buffers of one layer's reduced cache (allocated with torch) plus the C state struct."""

    def __init__(self, batch, n_q_heads, n_kv_heads, head_dim, L_cap, k_q_cap, device):
        self.Kc = torch.zeros(batch, n_kv_heads, L_cap, head_dim, dtype=torch.bfloat16, device=device)
        self.Vc = torch.zeros_like(self.Kc)
        self.idx = torch.zeros(batch, n_q_heads, max(1, k_q_cap), dtype=torch.int32, device=device)
        self.step = torch.zeros(1, dtype=torch.int32, device=device)
        self.state = CacheState(0, 0, 0, 0, 0, 0, self.step.data_ptr())
        self._made = (self.Kc, self.Vc, batch, n_kv_heads, self.Kc.get_device(), L_cap)

    def holds(self, sk, rows: int) -> bool:
        """Has it `rows` rows for every head of the context, on its device?  (Told from how it was made, as long as the tensors are those: a
        call of few rows would spend a third of its host time on looking at them.)"""
        Kc, Vc, batch, heads, device, room = self._made
        if Kc is not self.Kc or Vc is not self.Vc:
            return _holds(self.Kc, self.Vc, sk, rows)
        return room >= rows and sk.shape[3] == batch and sk.shape[1] == heads and sk.device_index == device

    def indices(self) -> torch.Tensor:
        """Selected positions as [B, H_q, k_q] for the k_q the last select_compact call used."""
        B, Hq = self.idx.shape[0], self.idx.shape[1]
        k_q = self.state.k_q
        return self.idx.flatten()[: B * Hq * k_q].view(B, Hq, k_q)

    def cache(self):
        """(Kc, Vc) cut to the L rows in use."""
        return self.Kc[:, :, : self.state.len], self.Vc[:, :, : self.state.len]


class SageKV:
    """Convenience wrapper: one context, the caller's tensors, the four steps in order."""

    def __init__(self, n_q_heads, n_kv_heads, head_dim=128, batch=1, max_ctx=131072, max_len=8193,
                 softmax_scale=0.0, device="cuda"):
        self.device = torch.device(device)
        self.shape = (n_q_heads, n_kv_heads, head_dim, batch)
        self.G = n_q_heads // n_kv_heads
        with torch.cuda.device(self.device):
            self.device_index = torch.cuda.current_device()
            self.ctx = sagekv_create(n_q_heads, n_kv_heads, head_dim, batch, max_ctx, max_len, softmax_scale)

    def set_overlap(self, mode: int):
        sagekv_set_overlap(self.ctx, mode)

    def set_decode_variant(self, variant: int):
        sagekv_set_decode_variant(self.ctx, variant)

    def set_select_overlap(self, mode: int):
        sagekv_set_select_overlap(self.ctx, mode)

    def set_select_hint(self, mode: int, k: int = 0):
        sagekv_set_select_hint(self.ctx, mode, k)

    def status(self) -> int:
        return sagekv_status(self.ctx)

    def close(self):
        if self.ctx is not None:
            sagekv_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def score_stride(self, n_ctx: int, n_init: int, n_recent: int) -> int:
        """Row stride of a score buffer for this context's hint mode (sagekv_scores_row_stride)."""
        return sagekv_scores_row_stride(self.ctx, n_ctx, n_init, n_recent)

    def new_scores(self, n_ctx: int, n_init: int, n_recent: int) -> torch.Tensor:
        Hq, _, _, B = self.shape
        return torch.empty(B * Hq, self.score_stride(n_ctx, n_init, n_recent), dtype=torch.float32,
                           device=self.device)

    def new_layer(self, n_init: int, n_recent: int, k: int, spare_rows: int = 0) -> Layer:
        """Buffers for a reduced cache of L = n_init + k + n_recent + 1 rows (plus `spare_rows` unused ones)."""
        Hq, Hkv, d, B = self.shape
        return Layer(B, Hq, Hkv, d, n_init + k + n_recent + 1 + spare_rows, k // self.G, self.device)

    def score(self, q_last, K, n_init, n_recent, scores=None):
        n_ctx = K.shape[2]
        if scores is None:
            scores = self.new_scores(n_ctx, n_init, n_recent)
        sagekv_score(self.ctx, q_last, K, n_ctx, n_init, n_recent, scores, scores.stride(0))
        return scores

    def select_compact(self, scores, K, V, n_init, n_recent, k, layer: Layer = None):
        if layer is None:
            layer = self.new_layer(n_init, n_recent, k)
        sagekv_select_compact(self.ctx, scores, scores.stride(0) if scores is not None else 0, K, V, K.shape[2],
                              n_init, n_recent, k, layer.idx, layer.Kc, layer.Vc, layer.state)
        return layer

    def decode_attn(self, q, k_new, v_new, layer: Layer, out=None, lse=None):
        if out is None:
            out = torch.empty_like(q)
        sagekv_decode_attn(self.ctx, q, k_new, v_new, layer.Kc, layer.Vc, layer.state, out, lse)
        return out

    # ---- the full cache in pages ----

    def rope(self, x, positions, plan: RopePlan, out=None):
        """Rows x [tokens, heads, 128] rotated by their positions (int32 [tokens]); out may be x."""
        shape = x.shape
        if out is None:
            out = torch.empty(shape, dtype=x.dtype, device=x.device)
        elif out.shape != shape:
            raise ValueError("expected out with the shape of x")
        n, heads, d = shape
        if d != 128 or not _placed(_BF16, self.device_index, x, out):
            raise ValueError("expected bf16 rows [tokens, heads, 128] on the context's device")
        if positions is None or not _placed_row(_INT32, self.device_index, n, False, positions):
            raise ValueError("expected contiguous int32 positions on the context's device, one per token")
        code = _marshal.rope(self.ctx, plan, x, n, heads, positions, out)
        if code:
            _check(code, "sagekv_rope", self.ctx)
        return out

    def paged_append(self, cache: PagedCache, k, v, positions, seqs=None, plan: RopePlan = None, q=None, q_out=None):
        """Keys and values [tokens, H_kv, 128] (with the same strides) into their pages, keys (and queries q, into q_out) rotated by the
        plan.  Without seqs token t belongs to sequence t.  Returns the rotated queries, or None."""
        shape = k.shape
        n, heads, d = shape
        device = self.device_index
        if heads != self.shape[1] or d != 128 or v.shape != shape or cache.n_kv_heads != heads or cache.device_index != device or \
                not _placed(_BF16, device, k, v, q, q_out):
            raise ValueError("expected bf16 k and v [tokens, H_kv, 128], bf16 q and q_out and pages of H_kv heads on the context's device")
        if positions is None or not _placed_row(_INT32, device, n, False, positions, seqs):
            raise ValueError("expected contiguous int32 positions and seqs on the context's device, one per token")
        if q is not None:
            shape = q.shape
            if q_out is None:
                q_out = torch.empty(shape, dtype=q.dtype, device=q.device)
            elif q_out is not q and q_out.shape != shape:
                raise ValueError("expected q_out with the shape of q")
            if shape != (n, self.shape[0], 128):
                raise ValueError("expected q [tokens, H_q, 128]")
        code = _marshal.paged_append(self.ctx, cache, k, v, n, positions, seqs, plan, q, q_out)
        if code:
            _check(code, "sagekv_paged_append", self.ctx)
        return q_out

    def paged_attn(self, q, cache: PagedCache, out=None, lse=None):
        """Attention of one new token per sequence, q [>= n_seqs, H_q, 128], over its cache."""
        shape, n, device = q.shape, cache.n_seqs, self.device_index
        if len(shape) != 3 or shape[0] < n or shape[1] != self.shape[0] or shape[2] != 128 or not _placed(_BF16, device, q) or \
                cache.n_kv_heads != self.shape[1] or cache.device_index != device:
            raise ValueError("expected bf16 q [n_seqs, H_q, 128] and pages of H_kv heads on the context's device")
        rows = n * shape[1]
        if out is None:
            out = torch.empty(shape, dtype=q.dtype, device=q.device)
        elif not _placed_row(_BF16, device, rows * 128, True, out):
            raise ValueError("expected contiguous bf16 out [n_seqs, H_q, 128] on the context's device")
        if not _placed_row(_FP32, device, rows, True, lse):
            raise ValueError("expected contiguous fp32 lse [n_seqs, H_q] on the context's device")
        code = _marshal.paged_attn(self.ctx, q, cache, out, lse)
        if code:
            _check(code, "sagekv_paged_attn", self.ctx)
        return out

    def paged_score(self, q_last, cache: PagedCache, n_ctx: int, n_init: int, n_recent: int, scores=None):
        """score() on a paged cache whose sequences have n_ctx tokens each."""
        (Hq, Hkv, d, batch), device = self.shape, self.device_index
        if q_last is None or not _placed_row(_BF16, device, batch * Hq * d, False, q_last) or cache.n_kv_heads != Hkv or cache.device_index != device:
            raise ValueError("expected contiguous bf16 q_last [B, H_q, 128] and pages of H_kv heads on the context's device")
        if scores is None:
            scores = self.new_scores(n_ctx, n_init, n_recent)
        shape, strides = scores.shape, scores.stride()
        if len(shape) != 2 or shape[0] < batch * Hq or shape[1] < n_ctx - 1 - n_init - n_recent or strides[1] != 1 or not _placed(_FP32, device, scores):
            raise ValueError("expected fp32 scores [B * H_q, >= n_ctx - 1 - n_init - n_recent] with contiguous rows on the context's device")
        code = _marshal.paged_score(self.ctx, q_last, cache, n_ctx, n_init, n_recent, scores, strides[0])
        if code:
            _check(code, "sagekv_paged_score", self.ctx)
        return scores

    def paged_compact(self, idx, cache: PagedCache, n_ctx: int, n_init: int, n_recent: int, k: int, layer: Layer = None):
        """The reduced cache from lists of offsets into the eviction region, int32 [B, H_q, k_q], as sagekv_select_topk writes
        them (layer.idx is not touched).  A layer that the caller brings has to hold the rows."""
        device = self.device_index
        if cache.n_kv_heads != self.shape[1] or cache.device_index != device:
            raise ValueError("expected pages of H_kv heads on the context's device")
        k_q = max(0, min(k // self.G, n_ctx - 1 - n_init - n_recent))
        if not _placed_row(_INT32, device, self.shape[3] * self.shape[0] * k_q, False, idx):
            raise ValueError("expected contiguous int32 lists [B, H_q, min(k / G, E)] on the context's device")
        if layer is None:
            layer = self.new_layer(n_init, n_recent, k)
        else:                                          # the library is given Kc's strides for both, and no number of rows
            rows = n_init + self.G * k_q + n_recent + 1
            fits = layer.holds(self, rows) if type(layer) is Layer else _holds(layer.Kc, layer.Vc, self, rows)
            if not fits:
                raise ValueError("expected a layer whose bf16 Kc and Vc are [B, H_kv, >= n_init + G * k_q + n_recent + 1, 128] on the context's "
                                 "device, laid out alike")
        code = _marshal.paged_compact(self.ctx, idx, cache, n_ctx, n_init, n_recent, k, layer.Kc, layer.Vc, layer.state)
        if code:
            _check(code, "sagekv_paged_compact", self.ctx)
        return layer
