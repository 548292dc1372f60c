"""The paged cache's host side: argument checks, addresses and rotary plans (needs no device)."""

import ctypes as C
import math

import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2503_08879_b200 import build
    build.build()
    from paper_2503_08879_b200 import binding
    return binding


def shape(B, **kw):
    return B.Shape(**(dict(n_q_heads=32, n_kv_heads=8, head_dim=128, batch=4, softmax_scale=0.0) | kw))


def described(B, dtype=torch.bfloat16, n_seqs=4, max_pages=5, page=16, n_pages=30):
    k = torch.zeros(n_pages, 8, page, 128, dtype=dtype)
    return B.PagedCache(k, torch.zeros_like(k), torch.zeros(n_seqs, max_pages, dtype=torch.int32))


def refusal(B, c, s=None):
    with pytest.raises(B.SagekvError) as e:
        B.sagekv_paged_check(s or shape(B), c)
    return e.value.code


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
def test_a_good_cache_passes(B, dtype):
    B.sagekv_paged_check(shape(B), described(B, dtype))
    c = described(B, dtype, n_seqs=0)
    B.sagekv_paged_check(shape(B), c)


@pytest.mark.parametrize("field, value", [("k_pages", None), ("v_pages", None), ("block_table", None), ("n_pages", 0), ("page_size", 0),
                                          ("max_pages", -1), ("n_seqs", -1), ("dtype", 2), ("dtype", -1), ("table_stride", 4),
                                          ("token_stride", 120), ("head_stride", 0), ("page_stride", -128), ("k_scale", 64), ("v_scale", 64)])
def test_invalid_fields(B, field, value):
    c = described(B)
    setattr(c, field, value)
    assert refusal(B, c) == B.ERR_INVALID


@pytest.mark.parametrize("field, value", [("page_size", 8), ("page_size", 24), ("n_seqs", 5), ("max_pages", 1 << 27), ("page_stride", 1 << 39),
                                          ("head_stride", 1 << 40), ("token_stride", 1 << 60)])
def test_unsupported_sizes(B, field, value):
    c = described(B)
    c.table_stride = 1 << 28
    setattr(c, field, value)
    assert refusal(B, c) == B.ERR_UNSUPPORTED


def test_the_list_of_tiles_must_fit_32_bits(B):
    c = described(B, n_seqs=3, max_pages=1 << 26)
    c.page_size, c.table_stride = 16, 1 << 26
    s = shape(B, n_kv_heads=16, batch=3)                          # 3 * 16 * 2^26 tiles
    assert refusal(B, c, s) == B.ERR_UNSUPPORTED
    c.max_pages = ((1 << 31) - 1) // 48
    B.sagekv_paged_check(s, c)
    c.max_pages += 1
    assert refusal(B, c, s) == B.ERR_UNSUPPORTED


@pytest.mark.parametrize("dtype, step", [(torch.bfloat16, 8), (torch.float8_e4m3fn, 16)])
def test_alignment(B, dtype, step):
    for f in ("page_stride", "head_stride", "token_stride"):
        c = described(B, dtype)
        setattr(c, f, getattr(c, f) + step)
        B.sagekv_paged_check(shape(B), c)
        setattr(c, f, getattr(c, f) - step // 2)
        assert refusal(B, c) == B.ERR_ALIGN
    for f in ("k_pages", "v_pages"):
        c = described(B, dtype)
        setattr(c, f, getattr(c, f) + 8)
        assert refusal(B, c) == B.ERR_ALIGN


def test_null_context_and_null_cache(B):
    assert B.lib.sagekv_paged_check(None, None) == B.ERR_INVALID
    assert B.lib.sagekv_paged_attn(None, None, 0, None, None, None, None) == B.ERR_INVALID
    assert B.lib.sagekv_paged_append(None, None, None, None, B.Rows(), 1, None, None, None, None, B.Rows(), None, B.Rows(), None) == B.ERR_INVALID
    assert B.lib.sagekv_rope(None, None, None, B.Rows(), 1, 1, None, None, B.Rows(), None) == B.ERR_INVALID
    assert B.lib.sagekv_paged_score(None, None, None, 1, 0, 0, None, 0, None) == B.ERR_INVALID
    assert B.lib.sagekv_paged_compact(None, None, None, 1, 0, 0, 0, None, None, B.Strides(), None, None) == B.ERR_INVALID


def test_the_python_description_refuses_what_the_struct_cannot_say(B):
    k = torch.zeros(4, 8, 16, 128, dtype=torch.bfloat16)
    t = torch.zeros(2, 2, dtype=torch.int32)
    for args in [(k, k[:, :, ::2], t), (k.float(), k.float(), t), (k, k, t.long()), (k, k, t, torch.zeros(2)), (k, k, t, torch.zeros(3, dtype=torch.int32)),
                 (k[..., ::2], k[..., ::2], t), (k, k, t.t().contiguous().t()),
                 (k, k, t, None, torch.zeros(7))]:
        with pytest.raises(ValueError):
            B.PagedCache(*args)


def test_rows_of_the_table_must_lie_apart(B):
    """A row expanded to several sequences has stride 0: refused, and not taken for rows one behind the other."""
    k = torch.zeros(4, 8, 16, 128, dtype=torch.bfloat16)
    assert refusal(B, B.PagedCache(k, k, torch.zeros(1, 3, dtype=torch.int32).expand(3, 3))) == B.ERR_INVALID
    B.sagekv_paged_check(shape(B), B.PagedCache(k, k, torch.zeros(1, 3, dtype=torch.int32).expand(1, 3)))
    B.sagekv_paged_check(shape(B), B.PagedCache(k, k, torch.zeros(5, 9, dtype=torch.int32)[:3, :4]))


@pytest.mark.parametrize("page_size", [16, 48, 64, 80, 1008, 65536])
def test_offsets(B, page_size):
    """Addresses against a plain division, beyond 32 bits too; pages that are none have no address."""
    c = described(B)
    c.page_size, c.n_pages = page_size, 1 << 20
    c.token_stride, c.head_stride, c.page_stride = 136, 136 * page_size, 136 * page_size * 8
    rng = np.random.default_rng(page_size)
    positions = [0, 1, page_size - 1, page_size, 2 * page_size - 1, 2 ** 31 - 1, 2 ** 30] + rng.integers(0, 2 ** 31, 2000).tolist()
    for pos in positions:
        page, head = int(rng.integers(0, 1 << 20)), int(rng.integers(0, 8))
        assert B.sagekv_paged_offset(c, page, head, pos) == page * c.page_stride + head * c.head_stride + (pos % page_size) * 136
    assert B.sagekv_paged_offset(c, (1 << 20) - 1, 7, 5) > 2 ** 32
    for page, head, pos in [(-1, 0, 0), (1 << 20, 0, 0), (2 ** 31 - 1, 0, 0), (-2 ** 31, 0, 0), (0, -1, 0), (0, 0, -1), (0, 0, 2 ** 31)]:
        with pytest.raises(B.SagekvError):
            B.sagekv_paged_offset(c, page, head, pos)


# ---- rotary plans ---------------------------------------------------------------------------------------------------


def turns(f):
    """f / (2 pi) as a fraction of 2^64, in exact arithmetic on a long expansion of pi."""
    from fractions import Fraction
    two_pi = 2 * Fraction(314159265358979323846264338327950288419716939937510582097494459, 10 ** 62)
    x = Fraction(f) / two_pi
    return (x - math.floor(x)) * 2 ** 64


def test_a_plan_holds_the_frequencies_as_fractions_of_a_revolution(B):
    f = [1.0, 0.5, 1e-3, 3.7e-7, 6.0, 7.0, 100.0, 0.0]
    p = B.sagekv_rope_plan_from(16, True, f, 1.5)
    assert (p.rotary_dim, p.interleaved, p.amplitude) == (16, 1, 1.5)
    for i, x in enumerate(f):
        # the long double quotient has 64 bits: half a unit of its last place, and the rounding to 2^-64
        assert abs(p.turns[i] - turns(x)) <= 1 + float(x) / (2 * math.pi) * 2
    assert not any(p.turns[i] for i in range(8, 64))


def test_a_fraction_that_rounds_up_to_a_revolution_carries(B):
    f = [math.nextafter(2 * math.pi, 0), 2 * math.pi] + [1.0] * 6
    p = B.sagekv_rope_plan_from(16, False, f)
    for i in (0, 1):
        d = abs(p.turns[i] - turns(f[i]))
        assert min(d, 2 ** 64 - d) <= 4


def frequencies_of(B, r, theta, rule=None):
    plan, f = B.RopePlan(), (C.c_double * 64)()
    code = B.lib.sagekv_rope_plan_init(C.byref(plan), r, 0, theta, None if rule is None else C.byref(rule), f)
    assert code == 0
    return np.array(f[: r // 2]), plan


@pytest.mark.parametrize("r", [16, 32, 64, 96, 128])
def test_unscaled_linear_and_base(B, r):
    i = np.arange(r // 2)
    f, plan = frequencies_of(B, r, 10000.0)
    np.testing.assert_allclose(f, 10000.0 ** (-2 * i / r), rtol=1e-14)
    assert plan.amplitude == 1.0 and plan.rotary_dim == r
    g, _ = frequencies_of(B, r, 10000.0, B.RopeScaling(1, 0, 4.0, 0, 0, 0, 0))
    np.testing.assert_allclose(g, f / 4, rtol=1e-14)
    h, plan = frequencies_of(B, r, 10000.0, B.RopeScaling(2, 0, 4.0, 0, 0, 0, 0.75))
    np.testing.assert_allclose(h, (10000.0 * 4 ** (r / (r - 2))) ** (-2 * i / r), rtol=1e-13)
    assert plan.amplitude == 0.75
    np.testing.assert_allclose(h[-1], f[-1] / 4, rtol=1e-12)      # the lowest frequency is interpolated in full


@pytest.mark.parametrize("kind, name, low, high", [(3, "llama3", 1.0, 4.0), (4, "yarn", 1.0, 32.0)])
@pytest.mark.parametrize("factor", [2.0, 8.0, 40.0])
def test_bands_and_yarn_against_a_library(B, kind, name, low, high, factor):
    """The library computes in 32 bits, powers and divisions: relative 1e-5."""
    from transformers.modeling_rope_utils import ROPE_INIT_FUNCTIONS

    class Config:
        rope_theta, hidden_size, num_attention_heads, head_dim, partial_rotary_factor = 500000.0, 4096, 32, 128, 1.0
        max_position_embeddings = int(8192 * factor)
        rope_parameters = rope_scaling = {"rope_type": name, "factor": factor, "low_freq_factor": low, "high_freq_factor": high, "beta_slow": low,
                                          "beta_fast": high, "original_max_position_embeddings": 8192, "rope_theta": 500000.0}

        def standardize_rope_params(self):
            pass

    want, amplitude = ROPE_INIT_FUNCTIONS[name](Config(), torch.device("cpu"))
    got, plan = frequencies_of(B, 128, 500000.0, B.RopeScaling(kind, 0, factor, low, high, 8192, 0))
    np.testing.assert_allclose(got, want.double().numpy(), rtol=1e-5)
    assert plan.amplitude == pytest.approx(amplitude, rel=1e-6)


def test_plans_refuse(B):
    code = lambda *a, **kw: pytest.raises(B.SagekvError, B.sagekv_rope_plan, *a, **kw).value.code
    for r in (0, 8, 24, 144, -16):
        assert code(r, False, 10000.0) == B.ERR_UNSUPPORTED
    for theta in (1.0, 0.0, -5.0, math.inf, math.nan):
        assert code(128, False, theta) == B.ERR_INVALID
    for rule in (dict(kind="linear", factor=0.5), dict(kind="linear", factor=math.nan), dict(kind="base", factor=math.inf),
                 dict(kind="bands", factor=8, low=4, high=4, original_ctx=8192), dict(kind="bands", factor=8, low=1, high=4),
                 dict(kind="yarn", factor=8, low=0, high=4, original_ctx=8192), dict(kind="linear", factor=2, amplitude=-1.0)):
        assert code(128, False, 10000.0, rule) == B.ERR_INVALID
    with pytest.raises(ValueError):
        B.sagekv_rope_plan(128, False, 1e4, dict(kind="cubic"))
    with pytest.raises(ValueError):
        B.sagekv_rope_plan(128, False, 1e4, dict(kind="linear", faktor=2))
    for f in ([-1.0] * 8, [math.nan] * 8, [math.inf] * 8):
        with pytest.raises(B.SagekvError):
            B.sagekv_rope_plan_from(16, False, f)
    with pytest.raises(ValueError):
        B.sagekv_rope_plan_from(16, False, [1.0] * 7)
    assert B.lib.sagekv_rope_plan_init(None, 128, 0, 1e4, None, None) == B.ERR_INVALID
    assert B.lib.sagekv_rope_plan_init(C.byref(B.RopePlan()), 128, 0, 1e4, C.byref(B.RopeScaling(5)), None) == B.ERR_INVALID
