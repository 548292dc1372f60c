"""What fills and reduces a paged cache (rotary positions, append, score, compaction) against 64 bits, and the operators together."""

import pytest
import torch

import paged_oracle as O

pytestmark = pytest.mark.gpu
BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn
# (dimensions that turn, neighbours paired, scaling rule)
TURNS = [(128, False, None), (128, True, None), (64, False, None), (16, False, None), (16, True, None), (96, True, None), (112, False, None),
         (32, True, dict(kind="linear", factor=4.0)), (128, False, dict(kind="yarn", factor=4.0, low=1.0, high=32.0, original_ctx=4096)),
         (128, False, dict(kind="bands", factor=8.0, low=1.0, high=4.0, original_ctx=8192))]
NAMES = ["%d%s%s" % (r, "n" if i else "h", s["kind"] if s else "") for r, i, s in TURNS]


def context(Hq, Hkv, batch, max_ctx=1024, max_len=64, **kw):
    from paper_2503_08879_b200 import binding as B
    return B, B.SageKV(Hq, Hkv, 128, batch, max_ctx=max_ctx, max_len=max_len, device="cuda", **kw)


def plan_of(B, turn, theta=10000.0):
    """(plan, its frequencies in 64 bits, its amplitude): the rules themselves are tested in test_paged_host.py"""
    import ctypes as C
    r, interleaved, rule = turn
    plan, f = B.sagekv_rope_plan(r, interleaved, theta, rule), (C.c_double * 64)()
    args = None if rule is None else B.RopeScaling(B.ROPE_KINDS[rule["kind"]], 0, *(rule.get(k, 0.0) for k in ("factor", "low", "high", "original_ctx", "amplitude")))
    assert B.lib.sagekv_rope_plan_init(C.byref(B.RopePlan()), r, int(interleaved), theta, None if args is None else C.byref(args), f) == 0
    return plan, torch.tensor(f[: r // 2], dtype=torch.float64), plan.amplitude


def random(*shape, seed=0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * spread).to(BF16)


def assert_rotated(got, x, pos, freq, interleaved, amplitude):
    """Two products and a sum in 32 bits of sines and cosines that are off by at most 2^-22 (the angle is known to 2^-33 of a revolution and
    rounded to 24 bits, 2^-24 * pi; sincospi 2 units): 2^-21 of |x_u| + |x_w|; then half a step of bf16."""
    want = O.rotate(x, pos, freq, interleaved, amplitude)
    tol = 2.0 ** -8 * want.abs() + 2.0 ** -21 * (1 + 2.0 ** -8) * O.pair_size(x, freq, interleaved, amplitude)
    r = 2 * len(freq)
    assert torch.all((got.double() - want).abs()[..., :r] <= tol[..., :r]), float(((got.double() - want).abs() - tol)[..., :r].max())
    assert torch.equal(got[..., r:], x[..., r:])


# ---- rope -----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("turn", TURNS, ids=NAMES)
@pytest.mark.parametrize("tokens, heads", [(1, 1), (1, 32), (3, 5), (130, 8), (700, 28)])
def test_rope(tokens, heads, turn):
    B, sk = context(1, 1, 1)
    plan, freq, amp = plan_of(B, turn)
    x = random(tokens, heads, 128)
    pos = torch.randint(-3, 2000, (tokens,), device="cuda", dtype=torch.int32)
    got = sk.rope(x, pos, plan)
    assert_rotated(got, x, pos, freq, turn[1], amp)
    sk.close()


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_far_positions(interleaved):
    """Angles of 2^31 revolutions' order: in 64 bits the oracle's own angle is off by 2^31 * 2^-53 radians."""
    B, sk = context(1, 1, 1)
    pos = torch.tensor([0, 1, -1, 131071, 1 << 20, 987654321, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    plan, freq, amp = plan_of(B, (128, interleaved, None), 500000.0)
    x = random(len(pos), 3, 128)
    assert_rotated(sk.rope(x, pos, plan), x, pos, freq, interleaved, amp)
    sk.close()


def test_rope_strides_in_place_and_what_lies_beside():
    B, sk = context(1, 1, 1)
    plan, freq, amp = plan_of(B, TURNS[0])
    pos = torch.arange(50, dtype=torch.int32, device="cuda") * 17
    wide = random(50, 9, 136)
    x = wide[:, 2:7, 8:]
    out = torch.full((50, 6, 128), 7.0, dtype=BF16, device="cuda")
    sk.rope(x, pos, plan, out[:, :5])
    assert_rotated(out[:, :5], x, pos, freq, False, amp)
    assert torch.all(out[:, 5] == 7)
    before = wide.clone()
    sk.rope(x, pos, plan, x)                                        # in place
    assert torch.equal(x, out[:, :5])
    wide[:, 2:7, 8:] = before[:, 2:7, 8:]
    assert torch.equal(wide, before)
    sideways = random(7, 50, 128).transpose(0, 1)                   # heads outside tokens
    assert_rotated(sk.rope(sideways, pos, plan), sideways, pos, freq, False, amp)
    sk.close()


def test_rope_gradient():
    """Turned back by negated positions: the gradient of <w, rope(x)> with respect to x is rope(w) at the negated positions
    (against the transposed formula, and against differences of the oracle)."""
    B, sk = context(1, 1, 1)
    for turn in TURNS:
        plan, freq, amp = plan_of(B, turn)
        pos = torch.randint(0, 3000, (20,), device="cuda", dtype=torch.int32)
        w = random(20, 2, 128, seed=1)
        x = random(20, 2, 128, seed=2).double().requires_grad_()
        grad, = torch.autograd.grad((O_rotate_graph(x, pos, freq, turn[1], amp) * w.double()).sum(), x)
        got = sk.rope(w, -pos, plan)
        assert torch.all((got.double() - grad).abs() <= 2.0 ** -8 * grad.abs() + 2.0 ** -20 * O.pair_size(w, freq, turn[1], amp) + 1e-30)
        e = torch.zeros_like(x)
        e[3, 1, 5] = 0.5                                            # (linear: a difference of any size will do)
        rise = ((O.rotate(x.detach() + e, pos, freq, turn[1], amp) - O.rotate(x.detach() - e, pos, freq, turn[1], amp)) * w.double()).sum()
        assert abs(float(rise) - float(got[3, 1, 5])) <= 2.0 ** -7 * abs(float(rise)) + 2.0 ** -18 * float(w.abs().max())
    sk.close()


def O_rotate_graph(x, pos, freq, interleaved, amplitude):
    r = 2 * len(freq)
    angle = pos.double()[:, None, None] * freq.to(x.device)
    c, s = angle.cos() * amplitude, angle.sin() * amplitude
    u, w = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., : r // 2], x[..., r // 2: r])
    a, b = u * c - w * s, w * c + u * s
    turned = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., r:]], -1)


def test_rope_refusals_and_nothing_to_do():
    B, sk = context(2, 1, 1)
    plan, x, pos = B.sagekv_rope_plan(128, False, 1e4), random(4, 2, 128), torch.zeros(4, dtype=torch.int32, device="cuda")
    out = torch.full_like(x, 7.0)
    code = lambda *a: pytest.raises(B.SagekvError, B.sagekv_rope, sk.ctx, *a).value.code
    assert code(None, x, 4, 2, pos, out) == B.ERR_INVALID
    assert code(B.RopePlan(), x, 4, 2, pos, out) == B.ERR_INVALID                 # a plan that no call filled
    assert code(plan, None, 4, 2, pos, out) == B.ERR_INVALID
    assert code(plan, x, 4, 2, None, out) == B.ERR_INVALID
    assert code(plan, x, 4, 2, pos, None) == B.ERR_INVALID
    assert code(plan, x, -1, 2, pos, out) == B.ERR_INVALID
    assert code(plan, x, 4, -1, pos, out) == B.ERR_INVALID
    assert code(plan, x[:, :1].expand(4, 2, 128), 4, 2, pos, out) == B.ERR_INVALID
    assert code(plan, x, 1 << 31, 2, pos, out) == B.ERR_UNSUPPORTED
    odd = torch.empty(4 * 256 + 8, dtype=BF16, device="cuda")
    assert code(plan, odd[4: 4 + 1024].view(4, 2, 128), 4, 2, pos, out) == B.ERR_ALIGN
    assert code(plan, torch.as_strided(odd, (4, 2, 128), (252, 128, 1)), 4, 2, pos, out) in (B.ERR_ALIGN, B.ERR_INVALID)
    for bad in ((x, pos.long(), plan), (x, pos[:3], plan), (x, pos, plan, out[:3])):
        with pytest.raises(ValueError):
            sk.rope(*bad)
    with pytest.raises(ValueError):
        B.sagekv_rope(sk.ctx, plan, x.transpose(1, 2), 4, 2, pos, out)
    B.sagekv_rope(sk.ctx, plan, x, 0, 2, pos, out)
    B.sagekv_rope(sk.ctx, plan, x, 4, 0, pos, out)
    torch.cuda.synchronize()
    assert torch.all(out == 7) and sk.status() == 0
    sk.close()


# ---- append -----------------------------------------------------------------------------------------------------------


def assert_stored(pool, which, s, tokens, want, slack):
    """want [n, H, 128] in 64 bits, known to `slack` before the one rounding: half a step of the cache's type.  (The 32-bit division by
    the scale of an 8-bit cache, as a product with its rounded reciprocal: 2^-23 more.)"""
    got = pool.rows(which, s, tokens, scaled=False)
    if pool.dtype == BF16:
        assert torch.all((got - want).abs() <= 2.0 ** -8 * want.abs() + slack * (1 + 2.0 ** -8)), float((got - want).abs().max())
        return
    scale = getattr(pool, which + "_scale")
    scale = torch.ones(pool.H, 1, device="cuda").double() if scale is None else scale.double()[:, None]
    code, slack = (want / scale).clamp(-448, 448), slack / scale + 2.0 ** -22 * (want / scale).abs()
    # a step of e4m3 is 2^(e - 3) in [2^e, 2^(e+1)), 2^-9 below 2^-6; what the slack carries over a power of two has at most twice the step there
    half = torch.maximum(2.0 ** -4 * (code.abs() + slack), torch.full_like(code, 2.0 ** -10))
    assert torch.all((got - code).abs() <= half + slack), float(((got - code).abs() - half).max())


def appended(Hq, Hkv, lens, page, dtype, turn, order=(0, 1, 2), queries=True, first=None, padding=0, fused=False, batch=None, scaled=True):
    """Tokens first[s] .. first[s] + lens[s] - 1 of every sequence appended in random order, with padding in between."""
    n = len(lens)
    first = first or [0] * n
    B, sk = context(Hq, Hkv, batch or n)
    pool = O.Pool(Hkv, page, n, max(1, -(-max(a + b for a, b in zip(first, lens)) // page)), dtype, "cuda", order, scaled=scaled)
    plan, freq, amp = plan_of(B, turn) if turn else (None, torch.zeros(0, dtype=torch.float64), 1.0)
    interleaved = bool(turn and turn[1])
    seq = torch.cat([torch.full((m,), s) for s, m in enumerate(lens)] + [torch.zeros(padding)]).to(torch.int32)
    pos = torch.cat([torch.arange(f, f + m) for f, m in zip(first, lens)] + [torch.full((padding,), -1)]).to(torch.int32)
    mix = torch.randperm(len(seq))
    seq, pos = seq[mix].cuda(), pos[mix].cuda()
    T = len(seq)
    if fused:
        wide = random(T, Hq + 2 * Hkv, 128)
        q, k, v = wide[:, :Hq], wide[:, Hq: Hq + Hkv], wide[:, Hq + Hkv:]
    else:
        q, k, v = random(T, Hq, 128, seed=1), random(T, Hkv, 128, seed=2), random(T, Hkv, 128, seed=3)
    raw_k, raw_v = pool.raw("k").clone(), pool.raw("v").clone()
    cache = pool.cache(B)
    q_out = torch.full((T, Hq, 128), 7.0, dtype=BF16, device="cuda") if queries else None
    sk.paged_append(cache, k, v, pos, seq, plan, q if queries else None, q_out)
    torch.cuda.synchronize()
    assert sk.status() == 0
    real = pos >= 0
    for s, m in enumerate(lens):
        mine = real & (seq == s)
        t = pos[mine].long()
        assert len(t) == m
        if m == 0:
            continue
        slack = 2.0 ** -21 * O.pair_size(k[mine], freq, interleaved, amp) if turn else torch.zeros(())
        if turn is None and dtype == BF16:
            assert torch.equal(pool.rows("k", s, t), k[mine].double())
        else:
            assert_stored(pool, "k", s, t, O.rotate(k[mine], t, freq, interleaved, amp), slack * torch.ones_like(k[mine]).double())
        if dtype == BF16:
            assert torch.equal(pool.rows("v", s, t), v[mine].double())
        else:
            assert_stored(pool, "v", s, t, v[mine].double(), torch.zeros_like(v[mine]).double())
        # the slots of these tokens are the only ones that changed
        pages = pool.table[s, t // page].long()
        for raw, now in ((raw_k, pool.raw("k")), (raw_v, pool.raw("v"))):
            raw[pages, :, t % page] = now[pages, :, t % page]
    assert torch.equal(raw_k, pool.raw("k")) and torch.equal(raw_v, pool.raw("v"))
    if queries:
        if turn:
            assert_rotated(q_out[real], q[real], pos[real], freq, interleaved, amp)
        else:
            assert torch.equal(q_out[real], q[real])
        assert torch.all(q_out[~real] == 7)
    sk.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("turn", TURNS + [None], ids=NAMES + ["none"])
def test_append_rotations(turn, dtype):
    appended(8, 4, [33, 0, 70], 16, dtype, turn, padding=5)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (2, 1), (28, 4), (32, 8), (5, 5), (6, 3), (42, 6), (7, 7)])
@pytest.mark.parametrize("queries", [True, False])
def test_append_heads(Hq, Hkv, queries, dtype):
    appended(Hq, Hkv, [1, 50, 17], 32, dtype, TURNS[0], queries=queries)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("page, order", [(16, (0, 2, 1)), (48, (0, 1, 2)), (80, (2, 0, 1)), (1024, (1, 0, 2))])
@pytest.mark.parametrize("fused", [False, True])
def test_append_layouts(page, order, fused, dtype):
    appended(8, 2, [100, 31, 200], page, dtype, TURNS[1], order=order, fused=fused, first=[0, 1000, 77])


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_append_many_tokens(dtype):
    """As many as give every warp several groups of heads."""
    appended(28, 4, [4000, 0, 9, 2500], 64, dtype, TURNS[0])


def test_append_without_scales():
    appended(4, 2, [40], 16, E4M3, TURNS[0], scaled=False)


def test_append_one_token_each_without_a_list_of_sequences():
    B, sk = context(8, 2, 40)
    n = 37                                                          # of a batch of 40
    pool = O.Pool(2, 16, n, 9, BF16, "cuda").fill([0] * n)
    plan, freq, amp = plan_of(B, TURNS[0])
    k, v = random(n, 2, 128), random(n, 2, 128, seed=1)
    pos = torch.randint(0, 9 * 16, (n,), device="cuda", dtype=torch.int32)
    pos[5] = -1
    q = random(n, 8, 128, seed=2)
    mine = q.clone()
    got = sk.paged_append(pool.cache(B), k, v, pos, plan=plan, q=mine, q_out=mine)      # queries in place
    assert got is mine and sk.status() == 0
    for s in range(n):
        if s == 5:
            assert torch.equal(mine[5], q[5])
            continue
        t = pos[s: s + 1].long()
        assert torch.equal(pool.rows("v", s, t), v[s: s + 1].double())
        assert_stored(pool, "k", s, t, O.rotate(k[s: s + 1], t, freq), 2.0 ** -21 * O.pair_size(k[s: s + 1], freq))
        assert_rotated(mine[s: s + 1], q[s: s + 1], t, freq, False, amp)
    sk.close()


def test_append_e4m3_limits():
    """Every step, ties, the largest value, beyond it, infinities and NaN."""
    B, sk = context(1, 1, 1)
    pool = O.Pool(1, 16, 1, 40, E4M3, "cuda", scaled=False)
    x = torch.cat([torch.linspace(-500, 500, 30001), torch.linspace(-0.05, 0.05, 30001), torch.tensor([448.0, 464, 480, 1e30, -1e30, float("inf"), -float("inf"), float("nan"), 0.0, -0.0]),
                   torch.zeros(128)])
    x = x[: len(x) // 128 * 128].to(BF16).view(-1, 1, 128).cuda()
    x = torch.cat([x[:600], x[-30:]])[: 40 * 16]
    pos = torch.arange(len(x), dtype=torch.int32, device="cuda")
    sk.paged_append(pool.cache(B), x, x, pos, torch.zeros_like(pos))
    want = x.float().clamp(-448, 448).to(E4M3).double()             # one rounding, to nearest even
    for which in "kv":
        got = pool.rows(which, 0, pos.long())
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(got[~torch.isnan(got)], want[~torch.isnan(want)])
    sk.close()


def test_append_beyond_32_bits():
    B, sk = context(2, 2, 1)
    n_pages = (2 ** 32 + 2 ** 26) // (2 * 16 * 128)
    pool = O.Pool(2, 16, 1, 3, E4M3, "cuda")
    for w in ("k", "v"):
        setattr(pool, w, torch.zeros(n_pages, 2, 16, 128, dtype=torch.uint8, device="cuda").view(E4M3))
    pool.table = torch.tensor([[n_pages - 1, 1, 2 ** 32 // 4096]], dtype=torch.int32, device="cuda")
    k, pos = random(48, 2, 128), torch.arange(48, dtype=torch.int32, device="cuda")
    sk.paged_append(pool.cache(B), k, k, pos, torch.zeros_like(pos))
    for w in ("k", "v"):
        assert_stored(pool, w, 0, pos.long(), k.double(), torch.zeros_like(k).double())
        assert int((getattr(pool, w).view(torch.int32) != 0).sum()) <= 48 * 2 * 32
    sk.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_append_out_of_range_is_left_out_and_reported(dtype):
    B, sk = context(2, 1, 4)
    pool = O.Pool(1, 16, 3, 2, dtype, "cuda").fill([0] * 3)
    good = pool.table.clone()
    pool.table[1, 0], pool.table[2, 1] = pool.k.shape[0], -7
    k, q = random(9, 1, 128), random(9, 2, 128)
    seq = torch.tensor([0, 0, 1, 1, 2, 2, 3, -1, 0], dtype=torch.int32, device="cuda")
    pos = torch.tensor([0, 32, 5, 20, 15, 16, 0, 0, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    before = pool.raw("k").clone()
    out = sk.paged_append(pool.cache(B), k, k, pos, seq, None, q)
    with pytest.raises(B.SagekvError) as e:
        sk.status()
    assert e.value.code == B.ERR_BOUNDS and e.value.bits == 2
    assert torch.equal(out, q)
    for t, there in enumerate([True, False, False, True, True, False, False, False, False]):
        if there:
            page, slot = int(good[seq[t], pos[t] // 16]), int(pos[t]) % 16
            row = pool.raw("k")[page, 0, slot].view(dtype).double() * (1 if dtype == BF16 else pool.k_scale.double())
            assert torch.allclose(row, k[t, 0].double(), rtol=2.0 ** -4 * 1.01 if dtype == E4M3 else 0, atol=2.0 ** -9 * 0.03 if dtype == E4M3 else 0)
            before[page, 0, slot] = pool.raw("k")[page, 0, slot]
    assert torch.equal(before, pool.raw("k"))
    sk.close()


def test_a_cache_of_another_number_of_heads_is_refused():
    """The C structure cannot say how many heads its pages have; the binding knows, and compares."""
    B, sk = context(4, 2, 2, max_ctx=40, max_len=40)
    pool = O.Pool(1, 16, 2, 2, BF16, "cuda")
    cache, k, q, pos = pool.cache(B, [5, 5]), random(2, 2, 128), random(2, 4, 128), torch.zeros(2, dtype=torch.int32, device="cuda")
    idx = torch.zeros(2, 4, 3, dtype=torch.int32, device="cuda")
    for call in (lambda: sk.paged_append(cache, k, k, pos), lambda: sk.paged_attn(q, cache), lambda: sk.paged_score(q, cache, 32, 4, 5),
                 lambda: sk.paged_compact(idx, cache, 32, 4, 5, 6)):
        with pytest.raises(ValueError):
            call()
    sk.close()


def test_append_refusals():
    B, sk = context(4, 2, 3)
    pool = O.Pool(2, 16, 3, 2, BF16, "cuda")
    k, q, pos = random(3, 2, 128), random(3, 4, 128), torch.zeros(3, dtype=torch.int32, device="cuda")
    cache, plan = pool.cache(B), B.sagekv_rope_plan(128, False, 1e4)
    before = pool.raw("k").clone()
    code = lambda *a: pytest.raises(B.SagekvError, B.sagekv_paged_append, sk.ctx, *a).value.code
    assert code(None, k, k, 3, pos) == B.ERR_INVALID
    assert code(cache, k, k, -1, pos) == B.ERR_INVALID
    assert code(cache, k, k, 1 << 31, pos) == B.ERR_UNSUPPORTED
    assert code(cache, k, k, 3, None) == B.ERR_INVALID
    assert code(cache, k, k, 3, pos, None, B.RopePlan()) == B.ERR_INVALID
    assert code(cache, k, k, 3, pos, None, plan, q, None) == B.ERR_INVALID
    assert code(cache, k, k, 3, pos, None, plan, None, q) == B.ERR_INVALID
    same = k[:1].expand(3, 2, 128)
    assert code(cache, same, same, 3, pos) == B.ERR_INVALID
    assert code(cache, k, k, 3, pos, None, plan, q[:1].expand(3, 4, 128), q) == B.ERR_INVALID
    odd = torch.empty(3 * 2 * 128 + 8, dtype=BF16, device="cuda")[4:-4].view(3, 2, 128)
    assert code(cache, odd, odd, 3, pos) == B.ERR_ALIGN
    for bad in (dict(k=k, v=k, positions=pos.long()), dict(k=k, v=k[:2], positions=pos), dict(k=k, v=k, positions=pos[:2]),
                dict(k=k, v=k, positions=pos, seqs=pos.long()), dict(k=k, v=k, positions=pos, q=q[:, :2]),
                dict(k=q, v=q, positions=pos), dict(k=k, v=random(3, 4, 128)[:, :2], positions=pos)):
        with pytest.raises(ValueError):
            sk.paged_append(cache, **bad)
    B.sagekv_paged_append(sk.ctx, cache, k, k, 0, pos)
    torch.cuda.synchronize()
    assert torch.equal(before, pool.raw("k")) and sk.status() == 0
    sk.close()


# ---- score and compaction ------------------------------------------------------------------------------------------------


def contiguous(pool, which, n_seqs, N):
    """[B, H, N, 128] in the type of the pool's values (bf16)."""
    t = torch.arange(N, device="cuda")
    return torch.stack([pool.rows(which, s, t) for s in range(n_seqs)]).transpose(1, 2)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("Hq, Hkv, n, N, page, order", [
    (32, 8, 1, 4096, 16, (0, 1, 2)), (28, 4, 2, 1003, 48, (0, 2, 1)), (1, 1, 1, 12, 16, (0, 1, 2)), (3, 1, 3, 777, 64, (1, 0, 2)),
    (16, 2, 1, 20000, 128, (2, 0, 1)), (8, 8, 2, 390, 16, (0, 1, 2)), (8, 1, 1, 770, 32, (0, 1, 2))])
def test_score(Hq, Hkv, n, N, page, order, dtype):
    """Against 64 bits, and against sagekv_score on the same rows without pages (which sums in another order: both are within tol)."""
    B, sk = context(Hq, Hkv, n, max_ctx=N)
    S, R = 4, 5
    E = N - 1 - S - R
    pool = O.Pool(Hkv, page, n, -(-N // page) + 1, dtype, "cuda", order).fill([N] * n)
    q = random(n, Hq, 128, spread=2.0)
    scores = torch.full((n * Hq, E + 20 - E % 4), 7.0, device="cuda")
    sk.paged_score(q, pool.cache(B), N, S, R, scores)
    assert sk.status() == 0 and torch.all(scores[:, E:] == 7)
    K = contiguous(pool, "k", n, N)
    s = torch.einsum("bhgd,bhtd->bhgt", q.double().view(n, Hkv, Hq // Hkv, 128), K[:, :, S: S + E]) * 128 ** -0.5
    sizes = torch.einsum("bhgd,bhtd->bhgt", q.double().abs().view(n, Hkv, Hq // Hkv, 128), K[:, :, S: S + E].abs()).amax(-1, keepdim=True) * 128 ** -0.5
    want = torch.softmax(s, -1).view(n * Hq, E)
    # as in assert_attention: a score is off by 2^-21 of its size, the exponential by 2^-22, a weight by twice that in all; the sums 2^-24 a term
    tol = (2 * (2.0 ** -21 * sizes + 2.0 ** -22)).view(n * Hq, 1) + 2.0 ** -24 * (E / 2048 + 64)
    assert torch.all((scores[:, :E].double() - want).abs() <= tol * want + 1e-38)
    if dtype == BF16:
        plain = sk.score(q, K.to(BF16).contiguous(), S, R, torch.empty_like(scores))
        assert torch.all((plain[:, :E].double() - scores[:, :E].double()).abs() <= 2 * tol * want + 1e-38)
    sk.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("hint", [0, 1, 2])
def test_score_hints_select_the_same(hint, dtype):
    """The hints behind the rows serve sagekv_select_topk's sibling on a contiguous cache as those of sagekv_score do."""
    N, S, R, G, k_q = 20011, 4, 128, 4, 100
    B, sk = context(8, 2, 1, max_ctx=N, max_len=2048)
    pool = O.Pool(2, 64, 1, -(-N // 64), dtype, "cuda").fill([N])
    q = random(1, 8, 128, spread=2.0)
    K, V = (contiguous(pool, w, 1, N).to(BF16).contiguous() for w in "kv")
    E = N - 1 - S - R
    plain = sk.paged_score(q, pool.cache(B), N, S, R)
    sk.set_select_hint(hint, G * k_q)
    scores = sk.paged_score(q, pool.cache(B), N, S, R)
    assert torch.allclose(scores[:, :E], plain[:, :E], rtol=1e-5, atol=0)
    layer = sk.select_compact(scores, K, V, S, R, G * k_q)
    want = scores[:, :E].topk(k_q, dim=1).indices.sort(dim=1).values + S
    assert torch.equal(layer.indices()[0].long(), want) and sk.status() == 0
    sk.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("Hq, Hkv, n, N, S, R, k_q, page, order", [
    (32, 8, 1, 3000, 4, 128, 60, 16, (0, 1, 2)), (28, 4, 2, 1003, 0, 0, 33, 48, (0, 2, 1)), (1, 1, 1, 20, 3, 4, 100, 16, (0, 1, 2)),
    (3, 1, 3, 777, 100, 1, 1, 64, (1, 0, 2)), (8, 2, 1, 500, 4, 10, 0, 32, (2, 0, 1)), (8, 2, 1, 30, 20, 9, 5, 16, (0, 1, 2))])
def test_compact(Hq, Hkv, n, N, S, R, k_q, page, order, dtype):
    B, sk = context(Hq, Hkv, n, max_ctx=N, max_len=3000)
    G, E = Hq // Hkv, N - 1 - S - R
    pool = O.Pool(Hkv, page, n, -(-N // page), dtype, "cuda", order).fill([N] * n)
    kept = min(k_q, E)
    idx = torch.rand(n * Hq, max(E, 1), device="cuda").topk(kept, dim=1).indices.view(n, Hq, kept).to(torch.int32) if kept else None
    layer = sk.new_layer(S, R, G * k_q, spare_rows=3)
    layer.Kc.fill_(7.0), layer.Vc.fill_(7.0), layer.step.fill_(9)
    sk.paged_compact(idx, pool.cache(B), N, S, R, G * k_q, layer)
    assert sk.status() == 0 and layer.step.item() == 0
    st = layer.state
    L = S + G * kept + R + 1
    assert (st.n_init, st.k_q, st.n_sel, st.n_recent, st.ring_len, st.len) == (S, kept, G * kept, R, R + 1, L)
    K, V = (contiguous(pool, w, n, N) for w in "kv")
    for b in range(n):
        for h in range(Hkv):
            mine = idx[b, h * G: (h + 1) * G].reshape(-1).long() + S if kept else torch.zeros(0, dtype=torch.long, device="cuda")
            t = torch.cat([torch.arange(S, device="cuda"), mine, torch.arange(S + E, N, device="cuda")])
            for got, all_rows in ((layer.Kc, K), (layer.Vc, V)):
                want = all_rows[b, h, t]
                if dtype == BF16:
                    assert torch.equal(got[b, h, :L].double(), want)
                else:   # code * scale in 32 bits (exact to 2^-24), rounded to bf16
                    assert torch.all((got[b, h, :L].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -23) * want.abs())
                assert torch.all(got[b, h, L:] == 7)
    sk.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_score_and_compact_with_bad_pages_and_positions(dtype):
    N, S, R, k_q = 200, 4, 10, 6
    B, sk = context(2, 1, 2, max_ctx=N, max_len=100)
    E = N - 1 - S - R
    pool = O.Pool(1, 16, 2, 13, dtype, "cuda").fill([N, N])
    q = random(2, 2, 128)
    cache = pool.cache(B)
    good, n_pages = pool.table.clone(), pool.k.shape[0]
    pool.table[0, 3], pool.table[0, 12], pool.table[1, 0] = -1, n_pages, 2 ** 31 - 1
    scores = sk.paged_score(q, cache, N, S, R)
    with pytest.raises(B.SagekvError) as e:
        sk.status()
    assert e.value.bits == 2
    p = scores[:, :E].view(2, 2, E)
    gone = torch.zeros(2, N, dtype=torch.bool, device="cuda")
    gone[0, 48:64] = gone[0, 192:] = gone[1, :16] = True
    assert torch.equal(p == 0, gone[:, None, S: S + E].expand(2, 2, E))
    assert torch.allclose(p.double().sum(-1), torch.ones(2, 2, device="cuda").double(), atol=1e-5)
    pool.table[1] = -1                                              # no page at all: the row stays finite, for a selection that may follow
    none = sk.paged_score(q, cache, N, S, R)[2:, :E]
    assert torch.allclose(none, torch.full_like(none, 1 / E), rtol=1e-5)
    with pytest.raises(B.SagekvError):
        sk.status()
    pool.table[1], pool.table[1, 0] = good[1], 2 ** 31 - 1
    idx = torch.tensor([[[0, 44, 45, 50, 90, 91], [1, 2, 3, -1, E, 2 ** 31 - 1]]] * 2, dtype=torch.int32, device="cuda")
    layer = sk.new_layer(S, R, 2 * k_q)
    layer.Kc.fill_(7.0), layer.Vc.fill_(7.0)
    sk.paged_compact(idx, cache, N, S, R, 2 * k_q, layer)
    with pytest.raises(B.SagekvError) as e:
        sk.status()
    assert e.value.bits == 2
    pool.table.copy_(good)
    K = contiguous(pool, "k", 2, N)
    for b in range(2):
        toks = list(range(S)) + [S + int(i) for i in idx[b].flatten()] + list(range(S + E, N))
        for r, t in enumerate(toks):
            row = layer.Kc[b, 0, r].double()
            off = r - S
            listed = not 0 <= off < 2 * k_q or 0 <= int(idx[b].flatten()[off]) < E
            if not listed or gone[b, t]:
                assert torch.all(row == 7), (b, r)
            else:
                assert torch.all((row - K[b, 0, t]).abs() <= (2.0 ** -8 + 2.0 ** -23) * K[b, 0, t].abs()), (b, r)
    sk.close()


def test_score_and_compact_refusals():
    N = 200
    B, sk = context(4, 2, 2, max_ctx=N, max_len=60)
    pool = O.Pool(2, 16, 2, 13, BF16, "cuda").fill([N, N])
    cache, q = pool.cache(B), random(2, 4, 128)
    scores = torch.full((8, 200), 7.0, device="cuda")
    code = lambda *a: pytest.raises(B.SagekvError, B.sagekv_paged_score, sk.ctx, *a).value.code
    assert code(None, cache, N, 4, 10, scores, 200) == B.ERR_INVALID
    assert code(q, None, N, 4, 10, scores, 200) == B.ERR_INVALID
    assert code(q, cache, N, 4, 10, None, 200) == B.ERR_INVALID
    assert code(q, cache, N, -1, 10, scores, 200) == B.ERR_INVALID
    assert code(q, cache, N, 190, 10, scores, 200) == B.ERR_INVALID                # sink + recent + 1 > n_ctx
    assert code(q, cache, 209, 4, 10, scores, 200) == B.ERR_INVALID                # beyond the table
    assert code(q, cache, 208, 4, 10, scores, 200) == B.ERR_UNSUPPORTED            # beyond max_ctx
    assert code(q, cache, N, 4, 10, scores, 184) == B.ERR_INVALID
    assert code(q, cache, N, 4, 10, scores, 198) == B.ERR_ALIGN
    one = B.PagedCache(pool.k, pool.v, pool.table[:1])
    assert code(q, one, N, 4, 10, scores, 200) == B.ERR_INVALID                    # fewer sequences than the batch
    idx = torch.zeros(2, 4, 5, dtype=torch.int32, device="cuda")
    layer = sk.new_layer(4, 10, 10)
    layer.Kc.fill_(7.0)
    code = lambda *a: pytest.raises(B.SagekvError, B.sagekv_paged_compact, sk.ctx, *a, layer.state).value.code
    assert code(idx, None, N, 4, 10, 10, layer.Kc, layer.Vc) == B.ERR_INVALID
    assert code(None, cache, N, 4, 10, 10, layer.Kc, layer.Vc) == B.ERR_INVALID
    assert code(idx, cache, N, 4, 10, 11, layer.Kc, layer.Vc) == B.ERR_INVALID     # k % G
    assert code(idx, cache, N, 4, 10, -2, layer.Kc, layer.Vc) == B.ERR_INVALID
    assert code(idx, one, N, 4, 10, 10, layer.Kc, layer.Vc) == B.ERR_INVALID
    assert code(idx, cache, 209, 4, 10, 10, layer.Kc, layer.Vc) == B.ERR_INVALID
    assert code(idx, cache, 208, 4, 10, 10, layer.Kc, layer.Vc) == B.ERR_UNSUPPORTED
    assert code(idx, cache, N, 4, 10, 100, layer.Kc, layer.Vc) == B.ERR_UNSUPPORTED    # L above max_len
    assert code(idx, cache, N, 4, 10, 10, layer.Kc[..., :120].reshape(-1)[4:516].view(1, 1, 4, 128), layer.Vc) == B.ERR_ALIGN
    B.sagekv_set_group_mode(sk.ctx, 1)
    assert code(idx, cache, N, 4, 10, 10, layer.Kc, layer.Vc) == B.ERR_UNSUPPORTED
    B.sagekv_set_group_mode(sk.ctx, 0)
    for bad in (idx.long(), idx[:, :, :4], idx[:1].contiguous()):
        with pytest.raises(ValueError):
            sk.paged_compact(bad, cache, N, 4, 10, 10)
    with pytest.raises(ValueError):
        sk.paged_score(q[:1], cache, N, 4, 10, scores)
    torch.cuda.synchronize()
    assert torch.all(layer.Kc == 7) and torch.all(scores == 7) and sk.status() == 0
    sk.close()


# ---- together ------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("Hq, Hkv", [(8, 2), (14, 2)])
def test_a_prompt_its_reduction_and_tokens_after_it(Hq, Hkv, dtype):
    """A prompt enters the pages; its last token scores them, the best tokens are kept, the reduced cache is decoded from; beside it
    full attention over the pages goes on.  The reduced path gives what the calls without pages give on the same rows."""
    N, S, R, k_q, steps, n = 2500, 4, 60, 90, 4, 2
    G, E = Hq // Hkv, N - 1 - S - R
    B, sk = context(Hq, Hkv, n, max_ctx=N + steps, max_len=S + G * k_q + R + 1)
    pool = O.Pool(Hkv, 64, n, -(-(N + steps) // 64), dtype, "cuda")
    lens = torch.tensor([N] * n, dtype=torch.int32, device="cuda")
    cache = B.PagedCache(pool.k, pool.v, pool.table, lens, pool.k_scale, pool.v_scale)
    plan, freq, amp = plan_of(B, TURNS[0], 500000.0)
    seq = torch.arange(n, device="cuda", dtype=torch.int32).repeat_interleave(N)
    pos = torch.arange(N, device="cuda", dtype=torch.int32).repeat(n)
    q = sk.paged_append(cache, random(n * N, Hkv, 128, seed=1), random(n * N, Hkv, 128, seed=2), pos, seq, plan, random(n * N, Hq, 128, seed=3, spread=3.0))
    q_last = q.view(n, N, Hq, 128)[:, -1].contiguous()
    scores = sk.paged_score(q_last, cache, N, S, R)
    idx = torch.empty(n, Hq, k_q, dtype=torch.int32, device="cuda")
    B.sagekv_select_topk(sk.ctx, scores, scores.stride(0), E, k_q, idx)
    layer = sk.paged_compact(idx, cache, N, S, R, G * k_q)
    K, V = (contiguous(pool, w, n, N).to(BF16).contiguous() for w in "kv")     # (8-bit: code * scale rounded to bf16, as the reduced cache holds it)
    plain = sk.select_compact(scores, K, V, S, R, G * k_q)
    assert torch.equal(plain.indices(), idx + S)
    if dtype == BF16:
        assert torch.equal(layer.Kc, plain.Kc) and torch.equal(layer.Vc, plain.Vc)
    else:
        for a, b in ((layer.Kc, plain.Kc), (layer.Vc, plain.Vc)):               # 32-bit against 64-bit product: a step at ties
            assert torch.all((a.double() - b.double()).abs() <= 2.0 ** -7 * b.double().abs())
    out, lse = torch.empty(n, Hq, 128, dtype=BF16, device="cuda"), torch.empty(n, Hq, device="cuda")
    for step in range(steps):
        lens += 1
        k, v, q = random(n, Hkv, 128, seed=10 + step), random(n, Hkv, 128, seed=20 + step), random(n, Hq, 128, seed=30 + step)
        q = sk.paged_append(cache, k, v, lens - 1, plan=plan, q=q)
        k_turned = sk.rope(k, lens - 1, plan)
        assert torch.equal(sk.decode_attn(q, k_turned, v, layer), sk.decode_attn(q, k_turned, v, plain)) or dtype == E4M3
        sk.paged_attn(q, cache, out, lse)
        for s in range(n):
            t = torch.arange(N + step + 1, device="cuda")
            want = O.attention(q[s], pool.rows("k", s, t), pool.rows("v", s, t), 128 ** -0.5)
            O.assert_attention(out[s], lse[s], *want, len(t), 2.0 ** -8 if dtype == BF16 else 2.0 ** -11)
        if dtype == BF16:
            assert torch.equal(pool.rows("k", 0, lens[:1].long() - 1)[0], k_turned[0].double())
    assert sk.status() == 0
    sk.close()


def test_a_captured_step_is_replayed_token_by_token():
    """Append and attention captured once; positions and lengths are the device's, so each replay is the next token."""
    B, sk = context(8, 2, 3)
    pool = O.Pool(2, 16, 3, 8, BF16, "cuda").fill([30, 0, 77])
    lens = torch.tensor([30, 0, 77], dtype=torch.int32, device="cuda")
    cache = B.PagedCache(pool.k, pool.v, pool.table, lens)
    plan, freq, amp = plan_of(B, TURNS[0])
    k, v, q = (torch.zeros(3, h, 128, dtype=BF16, device="cuda") for h in (2, 2, 8))
    pos, turned, out = lens.clone(), torch.zeros_like(q), torch.zeros_like(q)

    def step():
        pos.copy_(lens)
        lens.add_(1)
        sk.paged_append(cache, k, v, pos, None, plan, q, turned)
        sk.paged_attn(turned, cache, out)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    lens -= 1
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(5):
        k.copy_(random(3, 2, 128, seed=i)), v.copy_(random(3, 2, 128, seed=50 + i)), q.copy_(random(3, 8, 128, seed=90 + i))
        graph.replay()
        for s, n in enumerate([31 + i, 1 + i, 78 + i]):
            t = torch.arange(n, device="cuda")
            want, _, sizes, mean = O.attention(turned[s], pool.rows("k", s, t), pool.rows("v", s, t), 128 ** -0.5)
            O.assert_attention(out[s], None, want, None, sizes, mean, n, 2.0 ** -8)
            assert torch.equal(pool.rows("v", s, t[-1:])[0], v[s].double())
        assert_rotated(turned, q, pos, freq, False, amp)
    assert lens.tolist() == [35, 5, 82] and sk.status() == 0
    sk.close()
