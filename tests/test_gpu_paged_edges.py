"""Layouts, sizes and orders of calls that the interface of the paged cache allows and that lie at its edges."""

import pytest
import torch

import paged_oracle as O
from test_gpu_paged_attn import WEIGHTS
from test_gpu_paged_cache import TURNS, assert_rotated, assert_stored, context, contiguous, plan_of, random

pytestmark = pytest.mark.gpu
BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn


def padded(pool, pad, gap):
    """The pool's pages again, each row `pad` elements longer and each head `gap` rows longer, 16 bytes behind an allocation's start."""
    lead = 16 if pool.dtype == E4M3 else 8
    for which in "kv":
        old = pool.raw(which)
        n, H, page, d = old.shape
        flat = torch.full((lead + n * H * (page + gap) * (d + pad),), 0x7f if pool.dtype == E4M3 else 0x7fc0, dtype=old.dtype, device="cuda")
        new = flat[lead:].view(n, H, page + gap, d + pad)[:, :, :page, :d]
        new.copy_(old)
        setattr(pool, which, new.view(pool.dtype))
    return pool


@pytest.mark.parametrize("dtype, pads", [(BF16, (8, 24, 0)), (E4M3, (16, 48, 0))])
@pytest.mark.parametrize("gap", [0, 1])
def test_padded_rows_and_heads(gap, dtype, pads):
    """Strides that are multiples of 16 bytes and of nothing more, and a base that is so."""
    for pad in pads:
        N, S, R, Hq, Hkv = 300, 4, 10, 8, 2
        E = N - 1 - S - R
        B, sk = context(Hq, Hkv, 2, max_ctx=N, max_len=100)
        pool = padded(O.Pool(Hkv, 16, 2, 19, dtype, "cuda").fill([N, N]), pad, gap)
        assert pool.k.stride(2) == 128 + pad and pool.k.data_ptr() % 32 == 16
        cache = pool.cache(B, [N, N])
        plan, freq, amp = plan_of(B, TURNS[0])
        k, v, pos = random(2, Hkv, 128), random(2, Hkv, 128, seed=1), torch.tensor([N - 1, 33], dtype=torch.int32, device="cuda")
        sk.paged_append(cache, k, v, pos, plan=plan)
        for s in range(2):
            t = pos[s: s + 1].long()
            assert_stored(pool, "k", s, t, O.rotate(k[s: s + 1], t, freq), 2.0 ** -21 * O.pair_size(k[s: s + 1], freq))
            assert_stored(pool, "v", s, t, v[s: s + 1].double(), torch.zeros_like(v[s: s + 1]).double())
        q = random(2, Hq, 128, seed=2)
        lse = torch.empty(2, Hq, device="cuda")
        out = sk.paged_attn(q, cache, None, lse)
        t = torch.arange(N, device="cuda")
        for s in range(2):
            want = O.attention(q[s], pool.rows("k", s, t), pool.rows("v", s, t), 128 ** -0.5)
            O.assert_attention(out[s], lse[s], *want, N, WEIGHTS[dtype])
        scores = sk.paged_score(q, cache, N, S, R)
        K, V = (contiguous(pool, w, 2, N) for w in "kv")
        qg = q.double().view(2, Hkv, Hq // Hkv, 128)
        want = torch.softmax(torch.einsum("bhgd,bhtd->bhgt", qg, K[:, :, S: S + E]) * 128 ** -0.5, -1).view(2 * Hq, E)
        sizes = (torch.einsum("bhgd,bhtd->bhgt", qg.abs(), K.abs()).amax(-1) * 128 ** -0.5).view(2 * Hq, 1)
        tol = 2 * (2.0 ** -21 * sizes + 2.0 ** -22) + 2.0 ** -24 * (E / 2048 + 64)   # as in test_gpu_paged_cache.py
        assert torch.all((scores[:, :E].double() - want).abs() <= tol * want + 1e-38)
        idx = torch.rand(2 * Hq, E, device="cuda").topk(9, dim=1).indices.view(2, Hq, 9).to(torch.int32)
        layer = sk.paged_compact(idx, cache, N, S, R, 9 * Hq // Hkv)
        for b in range(2):
            for h in range(Hkv):
                rows = torch.cat([t[:S], idx[b, 4 * h: 4 * h + 4].reshape(-1).long() + S, t[S + E:]])
                for got, all_rows in ((layer.Kc, K), (layer.Vc, V)):
                    want = all_rows[b, h, rows]
                    assert torch.all((got[b, h, : len(rows)].double() - want).abs() <= (0 if dtype == BF16 else 2.0 ** -8 + 2.0 ** -23) * want.abs())
        assert sk.status() == 0
        sk.close()


def test_a_region_without_tokens_writes_no_score():
    B, sk = context(8, 2, 1, max_ctx=15, max_len=15)
    pool = O.Pool(2, 16, 1, 1, BF16, "cuda").fill([15])
    scores = torch.full((8, 4), 7.0, device="cuda")
    sk.paged_score(random(1, 8, 128), pool.cache(B), 15, 4, 10, scores)
    layer = sk.paged_compact(None, pool.cache(B), 15, 4, 10, 0)
    assert torch.all(scores == 7) and torch.equal(layer.Kc[0].transpose(0, 1).double(), pool.rows("k", 0, torch.arange(15, device="cuda")))
    assert sk.status() == 0
    sk.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_scores_of_a_batch_whose_rows_leave_a_head_few_blocks(dtype):
    """More than 4096 rows: the scratch holds as many parts per row as the longest context has chunks, here three."""
    n, Hq, Hkv, N, S, R = 150, 32, 8, 700, 4, 10
    E = N - 1 - S - R
    B, sk = context(Hq, Hkv, n, max_ctx=N)
    pool = O.Pool(Hkv, 64, n, 11, dtype, "cuda").fill([N] * n)
    q = random(n, Hq, 128, spread=2.0)
    scores = sk.paged_score(q, pool.cache(B), N, S, R)
    for s in (0, 1, 74, 148, 149):
        K = pool.rows("k", s, torch.arange(S, S + E, device="cuda"))
        qg = q[s].double().view(Hkv, Hq // Hkv, 128)
        want = torch.softmax(torch.einsum("hgd,thd->hgt", qg, K) * 128 ** -0.5, -1).view(Hq, E)
        sizes = (torch.einsum("hgd,thd->hgt", qg.abs(), K.abs()).amax(-1) * 128 ** -0.5).view(Hq, 1)
        tol = 2 * (2.0 ** -21 * sizes + 2.0 ** -22) + 2.0 ** -24 * (E / 2048 + 64)
        assert torch.all((scores[s * Hq: (s + 1) * Hq, :E].double() - want).abs() <= tol * want + 1e-38)
    assert sk.status() == 0
    sk.close()


@pytest.mark.parametrize("mode", [0, 1, 2])
@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_decode_ahead_of_its_wait_behind_the_paged_calls(mode, dtype):
    """Compaction of two layers, the token's append with its queries, decode of both layers in every overlap mode: in mode 2 the rows of
    the reduced cache are asked for before decode's wait, and neither the append nor the other layer's decode writes them.  Eager, and
    captured and replayed: the same bits as one call after the other."""
    N, S, R, k_q, Hq, Hkv, n = 3001, 4, 60, 90, 8, 2, 2
    G, E = Hq // Hkv, N - 1 - S - R
    B, sk = context(Hq, Hkv, n, max_ctx=N, max_len=S + G * k_q + R + 1)
    pools = [O.Pool(Hkv, 64, n, 48, dtype, "cuda", seed=i).fill([N] * n) for i in range(2)]
    caches = [p.cache(B, [N] * n) for p in pools]
    idx = [torch.rand(n * Hq, E, device="cuda").topk(k_q, dim=1).indices.sort(dim=1).values.view(n, Hq, k_q).to(torch.int32) for _ in range(2)]
    layers = [sk.new_layer(S, R, G * k_q) for _ in range(2)]
    plan, freq, amp = plan_of(B, TURNS[0])
    k, v, q = random(n, Hkv, 128, seed=5), random(n, Hkv, 128, seed=6), random(n, Hq, 128, seed=7)
    pos = torch.full((n,), N, dtype=torch.int32, device="cuda")
    turned, outs = [torch.empty_like(q) for _ in range(2)], [torch.empty_like(q) for _ in range(3)]

    def step(apart):
        gap = torch.cuda.synchronize if apart else lambda: None
        for i in range(2):
            sk.paged_compact(idx[i], caches[i], N, S, R, G * k_q, layers[i])
            gap()
        for i in range(2):
            sk.paged_append(caches[i], k, v, pos, plan=plan, q=q, q_out=turned[i])
            gap()
            sk.decode_attn(turned[i], k, v, layers[i], outs[i])
            gap()
        sk.paged_attn(turned[1], caches[1], outs[2])
        gap()

    sk.set_overlap(mode)                                            # (also which kernel decodes is a matter of the mode)
    step(True)
    want = [o.clone() for o in outs]
    assert all(bool(o.any()) and bool(torch.isfinite(o).all()) for o in want)

    def fresh():
        for layer in layers:
            layer.Kc.zero_(), layer.Vc.zero_()
        for o in outs + turned:
            o.zero_()
        torch.cuda.synchronize()

    def same():
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))

    for _ in range(10):
        fresh()
        step(False)
        same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(False)
    for _ in range(10):
        fresh()
        graph.replay()
        same()
    assert sk.status() == 0
    sk.close()


def test_absent_tokens_weigh_nothing_beside_the_lowest_logits():
    """Logits of -10^32: a token whose page is none still gets no weight, and those that are there share it."""
    N, S, R = 208, 0, 15
    E = N - 1 - S - R
    B, sk = context(1, 1, 1, max_ctx=N)
    pool = O.Pool(1, 16, 1, 13, BF16, "cuda").fill([N])
    pool.k.zero_()
    pool.k[..., 0] = -2.0 ** 50
    q = torch.zeros(1, 1, 128, dtype=BF16, device="cuda")
    q[..., 0] = 2.0 ** 60
    pool.table[0, 2] = -1
    p = sk.paged_score(q, pool.cache(B), N, S, R)[0, :E]
    with pytest.raises(B.SagekvError):
        sk.status()
    gone = torch.zeros(E, dtype=torch.bool, device="cuda")
    gone[32:48] = True
    assert not p[gone].any() and torch.allclose(p[~gone], torch.full_like(p[~gone], 1 / (E - 16)), rtol=1e-5)
    sk.close()
