"""What the wrapper's paged methods refuse by themselves, before the library is called (needs no device: the context is none,
so a call that is let through comes back from the library as INVALID)."""

import ctypes as C
from types import SimpleNamespace

import pytest
import torch

HQ, HKV, BATCH = 8, 2, 3
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def B():
    from paper_2503_08879_b200 import build
    build.build()
    from paper_2503_08879_b200 import binding as B
    names = ("score", "select_compact", "decode_attn", "pool_scores", "quest_bounds", "select_topk")
    bind = lambda stream: B._marshal.bind(*(C.cast(getattr(B.lib, "sagekv_" + n), C.c_void_p).value for n in names), stream, C.ArgumentError)
    bind(lambda: 0)                                                  # there is no current stream without a device
    yield B
    bind(B._stream_handle)


def wrapper(B, device_index=-1):
    """A SageKV without a context; -1 is the index that host tensors give."""
    sk = B.SageKV.__new__(B.SageKV)
    sk.ctx, sk.shape, sk.G, sk.device, sk.device_index = None, (HQ, HKV, 128, BATCH), HQ // HKV, torch.device("cpu"), device_index
    return sk


def cache(B, lens=True, **kw):
    k = torch.zeros(12, HKV, 16, 128, dtype=BF16)
    return B.PagedCache(k, torch.zeros_like(k), torch.zeros(BATCH, 4, dtype=torch.int32), torch.zeros(BATCH, dtype=torch.int32) if lens else None, **kw)


def reaches_the_library(B, call, *a, **kw):
    with pytest.raises(B.SagekvError) as e:
        call(*a, **kw)
    assert e.value.code == B.ERR_INVALID


def refused(call, *a, **kw):
    with pytest.raises(ValueError):
        call(*a, **kw)


# ---- paged_compact: the caller's layer -------------------------------------------------------------------------------------

N, S, R, KQ = 60, 4, 10, 5
L = S + HQ // HKV * KQ + R + 1


def layer_of(B, Kc, Vc):
    return SimpleNamespace(Kc=Kc, Vc=Vc, state=B.CacheState(0, 0, 0, 0, 0, 0, None))


def compact(B, layer, sk=None):
    idx = torch.zeros(BATCH, HQ, KQ, dtype=torch.int32)
    return (sk or wrapper(B)).paged_compact, idx, cache(B), N, S, R, HQ // HKV * KQ, layer


def test_layers_that_hold_the_rows_are_taken(B):
    for rows in (L, L + 7):
        Kc = torch.zeros(BATCH, HKV, rows, 128, dtype=BF16)
        reaches_the_library(B, *compact(B, layer_of(B, Kc, torch.zeros_like(Kc))))
    wide = torch.zeros(BATCH, HKV, L, 136, dtype=BF16)
    reaches_the_library(B, *compact(B, layer_of(B, wide[..., :128], wide.clone()[..., :128])))
    reaches_the_library(B, *compact(B, None))


@pytest.mark.parametrize("shape", [(BATCH, HKV, L - 1, 128), (BATCH - 1, HKV, L, 128), (BATCH, HKV - 1, L, 128), (BATCH, HKV, L, 64),
                                   (BATCH, HKV, L * 128), (HKV, L, 128)])
def test_layers_too_small_for_the_rows_are_refused(B, shape):
    """A layer of a smaller budget, or of another batch: the rows would go into the next head's, and past the end."""
    small, full = torch.zeros(shape, dtype=BF16), torch.zeros(BATCH, HKV, L, 128, dtype=BF16)
    for Kc, Vc in ((small, small.clone()), (full, small), (small, full)):
        refused(*compact(B, layer_of(B, Kc, Vc)))


def test_a_layer_whose_tensors_are_laid_out_differently_is_refused(B):
    """One set of strides goes to the library, Kc's."""
    Kc = torch.zeros(BATCH, HKV, L, 128, dtype=BF16)
    refused(*compact(B, layer_of(B, Kc, torch.zeros(BATCH, L, HKV, 128, dtype=BF16).transpose(1, 2))))
    refused(*compact(B, layer_of(B, torch.zeros(BATCH, HKV, L + 1, 128, dtype=BF16), Kc)))


# ---- rows of 128 -----------------------------------------------------------------------------------------------------------


def rows(*shape, dtype=BF16):
    return torch.zeros(*shape, dtype=dtype)


def int32(n):
    return torch.zeros(n, dtype=torch.int32)


def test_calls_with_whole_rows_reach_the_library(B):
    sk, c, plan = wrapper(B), cache(B), B.sagekv_rope_plan(128, False, 1e4)
    reaches_the_library(B, sk.rope, rows(5, 3, 128), int32(5), plan)
    reaches_the_library(B, sk.rope, rows(5, 3, 136)[..., 8:], int32(5), plan, rows(5, 4, 128)[:, :3])
    reaches_the_library(B, sk.paged_append, c, rows(5, HKV, 128), rows(5, HKV, 128), int32(5), int32(5), plan, rows(5, HQ, 128))
    reaches_the_library(B, sk.paged_append, c, rows(5, HKV, 128), rows(5, HKV, 128), int32(5))
    reaches_the_library(B, sk.paged_attn, rows(BATCH, HQ, 128), c)
    reaches_the_library(B, sk.paged_attn, rows(BATCH + 2, HQ, 128), c, rows(BATCH, HQ, 128), torch.zeros(BATCH, HQ))
    reaches_the_library(B, sk.paged_score, rows(BATCH, HQ, 128), c, N, S, R, torch.zeros(BATCH * HQ, 60))


def test_rows_that_are_shorter_are_refused(B):
    """128 elements are read and written per row: half a row of a wider tensor has the strides of a whole one, and the result that the
    wrapper would make for it is too short."""
    sk, c, plan = wrapper(B), cache(B), B.sagekv_rope_plan(64, False, 1e4)
    half = lambda *shape: rows(*shape)[..., :64]
    refused(sk.paged_attn, half(BATCH, HQ, 128), c)
    refused(sk.paged_attn, rows(BATCH, HQ, 64), c)
    refused(sk.rope, rows(1, 1, 64), int32(1), plan)
    refused(sk.rope, half(5, 3, 128), int32(5), plan)
    k, q = rows(1, HKV, 128), rows(1, HQ, 128)
    refused(sk.paged_append, c, half(1, HKV, 128), half(1, HKV, 128), int32(1))
    refused(sk.paged_append, c, k, k, int32(1), None, plan, half(1, HQ, 128))
    refused(sk.paged_append, c, k, k, int32(1), None, plan, q, half(1, HQ, 128))


# ---- types -------------------------------------------------------------------------------------------------------------------


def test_tensors_of_other_types_are_refused(B):
    """Pointers carry no type: 16-bit floats of another kind would be taken for bf16, and an lse of 2-byte elements be written past its end."""
    sk, c, plan = wrapper(B), cache(B), B.sagekv_rope_plan(128, False, 1e4)
    for dtype in (torch.float16, torch.float32):
        x = rows(5, 3, 128, dtype=dtype)
        refused(sk.rope, x, int32(5), plan)
        refused(sk.rope, x, int32(5), plan, x)
        refused(sk.rope, rows(5, 3, 128), int32(5), plan, x)
        k, q, other = rows(5, HKV, 128), rows(5, HQ, 128), rows(5, HKV, 128, dtype=dtype)
        refused(sk.paged_append, c, other, other, int32(5))
        refused(sk.paged_append, c, k, other, int32(5))
        refused(sk.paged_append, c, other, k, int32(5))
        refused(sk.paged_append, c, k, k, int32(5), None, plan, rows(5, HQ, 128, dtype=dtype))
        refused(sk.paged_append, c, k, k, int32(5), None, plan, q, rows(5, HQ, 128, dtype=dtype))
        q = rows(BATCH, HQ, 128)
        refused(sk.paged_attn, q.to(dtype), c)
        refused(sk.paged_attn, q, c, q.to(dtype))
        refused(sk.paged_score, q.to(dtype), c, N, S, R, torch.zeros(BATCH * HQ, 60))
        full = torch.zeros(BATCH, HKV, L, 128, dtype=dtype)
        refused(*compact(B, layer_of(B, full, full.clone())))
        refused(*compact(B, layer_of(B, full.to(BF16), full)))
    for dtype in (BF16, torch.float16, torch.float64):
        refused(sk.paged_attn, q, c, None, torch.zeros(BATCH, HQ, dtype=dtype))
        refused(sk.paged_score, q, c, N, S, R, torch.zeros(BATCH * HQ, 60, dtype=dtype))


# ---- devices -----------------------------------------------------------------------------------------------------------------


def test_tensors_on_another_device_than_the_context_are_refused(B):
    """Host pointers, or those of another device, would reach the kernels.  (A context of device 0 here, tensors of the host.)"""
    c, plan = cache(B), B.sagekv_rope_plan(128, False, 1e4)
    k, q = rows(5, HKV, 128), rows(BATCH, HQ, 128)
    for call in (lambda sk: sk.rope(rows(5, 3, 128), int32(5), plan), lambda sk: sk.paged_append(c, k, k, int32(5)),
                 lambda sk: sk.paged_attn(q, c), lambda sk: sk.paged_score(q, c, N, S, R, torch.zeros(BATCH * HQ, 60))):
        reaches_the_library(B, call, wrapper(B))
        refused(call, wrapper(B, 0))
    layer = B.Layer(BATCH, HQ, HKV, 128, L, KQ, "cpu")
    reaches_the_library(B, *compact(B, layer))
    refused(*compact(B, layer, wrapper(B, 0)))


class Elsewhere:
    """A tensor that says it is on another device."""

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return 1


def test_every_tensor_of_a_call_is_looked_at(B):
    sk, plan, far = wrapper(B), B.sagekv_rope_plan(128, False, 1e4), Elsewhere
    c, k, q, pos = cache(B), rows(5, HKV, 128), rows(5, HQ, 128), int32(5)
    moved = cache(B)
    moved.device_index = 1                                           # as of pages on that device
    refused(sk.rope, far(q), pos, plan, q)
    refused(sk.rope, q, far(pos), plan)
    refused(sk.rope, q, pos, plan, far(q))
    for bad in ((moved, k, k, pos, pos, plan, q, q), (c, far(k), k, pos, pos, plan, q, q), (c, k, far(k), pos, pos, plan, q, q),
                (c, k, k, far(pos), pos, plan, q, q), (c, k, k, pos, far(pos), plan, q, q), (c, k, k, pos, pos, plan, far(q), q),
                (c, k, k, pos, pos, plan, q, far(q))):
        refused(sk.paged_append, *bad)
    q, out, lse, scores = rows(BATCH, HQ, 128), rows(BATCH, HQ, 128), torch.zeros(BATCH, HQ), torch.zeros(BATCH * HQ, 60)
    for bad in ((q, moved, out, lse), (far(q), c, out, lse), (q, c, far(out), lse), (q, c, out, far(lse))):
        refused(sk.paged_attn, *bad)
    for bad in ((q, moved, N, S, R, scores), (far(q), c, N, S, R, scores), (q, c, N, S, R, far(scores))):
        refused(sk.paged_score, *bad)
    call, idx, c, *sizes, layer = compact(B, B.Layer(BATCH, HQ, HKV, 128, L, KQ, "cpu"))
    refused(call, idx, moved, *sizes, layer)
    refused(call, far(idx), c, *sizes, layer)
    refused(call, idx, c, *sizes, layer_of(B, far(layer.Kc), layer.Vc))
    refused(call, idx, c, *sizes, layer_of(B, layer.Kc, far(layer.Vc)))


def test_layers_of_the_wrapper_are_judged_by_how_they_were_made_unless_their_tensors_were_exchanged(B):
    made = lambda batch=BATCH, heads=HKV, rows=L: B.Layer(batch, HQ, heads, 128, rows, KQ, "cpu")
    reaches_the_library(B, *compact(B, made()))
    for small in (made(rows=L - 1), made(batch=BATCH - 1), made(heads=HKV - 1)):
        refused(*compact(B, small))
    layer = made()
    layer.Vc = layer.Vc[:, :, : L - 1]
    refused(*compact(B, layer))
    layer = made(rows=L - 1)
    layer.Kc, layer.Vc = torch.zeros(BATCH, HKV, L, 128, dtype=BF16), torch.zeros(BATCH, HKV, L, 128, dtype=BF16)
    reaches_the_library(B, *compact(B, layer))


# ---- the scores' rows ----------------------------------------------------------------------------------------------------------


def test_scores_without_a_row_per_query_head_are_refused(B):
    """The library is given the distance of the rows and no number: a buffer of fewer rows, or of shorter ones, would be written past its end."""
    sk, c, q, E = wrapper(B), cache(B), rows(BATCH, HQ, 128), N - 1 - S - R
    for good in (torch.zeros(BATCH * HQ, E + 3), torch.zeros(BATCH * HQ + 1, 64), torch.zeros(BATCH * HQ, 80)[:, :E]):
        reaches_the_library(B, sk.paged_score, q, c, N, S, R, good)
    for bad in (torch.zeros(BATCH * HQ - 1, 64), torch.zeros(HQ, 64), torch.zeros(BATCH * HQ, E - 1), torch.zeros(64, BATCH * HQ).t(),
                torch.zeros(BATCH, HQ, 64), torch.zeros(BATCH * HQ * 64)):
        refused(sk.paged_score, q, c, N, S, R, bad)


# ---- strides that are never stepped along ---------------------------------------------------------------------------------------


def test_one_token_of_k_and_v_out_of_different_tensors(B):
    """Of a single token the distance of the tokens means nothing: k by itself and v out of a fused projection go together."""
    sk, c = wrapper(B), cache(B)
    fused = rows(1, HQ + 2 * HKV, 128)
    reaches_the_library(B, sk.paged_append, c, rows(1, HKV, 128), fused[:, HQ + HKV:], int32(1))
    fused = rows(2, HQ + 2 * HKV, 128)
    refused(sk.paged_append, c, rows(2, HKV, 128), fused[:, HQ + HKV:], int32(2))
    refused(sk.paged_append, c, rows(1, HKV, 128), rows(1, HKV, 136)[..., :128], int32(1))
