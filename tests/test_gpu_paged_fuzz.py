"""Random shapes, layouts, lengths and settings of the paged cache's calls against 64 bits."""

import random

import pytest
import torch

import paged_oracle as O
from test_gpu_paged_attn import WEIGHTS
from test_gpu_paged_cache import TURNS, appended, contiguous

pytestmark = pytest.mark.gpu
BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn
ORDERS = [(0, 1, 2), (0, 2, 1), (1, 0, 2), (1, 2, 0), (2, 0, 1), (2, 1, 0)]


def shape(rng):
    Hkv = rng.choice([1, 1, 2, 3, 4, 8])
    return Hkv * rng.randint(1, 8), Hkv


def length(rng, most):
    kind = rng.random()
    return 0 if kind < 0.1 else rng.randint(1, 20) if kind < 0.3 else 16 * rng.randint(1, most // 16) if kind < 0.5 else rng.randint(1, most)


@pytest.mark.parametrize("seed", range(60))
def test_attention(seed):
    from paper_2503_08879_b200 import binding as B
    rng = random.Random(seed)
    Hq, Hkv = shape(rng)
    n = rng.choice([1, 1, 2, 3, 5, 17, 32, 33, 40, 150])
    most = rng.choice([20, 100, 700, 5000, 30000]) // (1 if n < 4 else 10 if n < 60 else 60) + 16
    lens = [length(rng, most) for _ in range(n)]
    dtype, page = rng.choice([BF16, E4M3]), rng.choice([16, 32, 48, 64, 112, 256])
    scale = rng.choice([0.0, 0.0, 0.02, 0.3])
    sk = B.SageKV(Hq, Hkv, 128, n + rng.randint(0, 3), max_ctx=64, max_len=16, softmax_scale=scale, device="cuda")
    pool = O.Pool(Hkv, page, n, max(1, -(-max(lens) // page)) + rng.randint(0, 2), dtype, "cuda", rng.choice(ORDERS), seed=seed,
                  scaled=rng.random() < 0.8).fill(lens, rng.choice([0.3, 1.0, 3.0]))
    wide = torch.randn(n, Hq + 3, 128, generator=pool.gen, device="cuda").to(BF16)
    q = wide[:, 1: Hq + 1] if rng.random() < 0.5 else wide[:, :Hq].contiguous()
    out, lse = torch.empty(n, Hq, 128, dtype=BF16, device="cuda"), torch.empty(n, Hq, device="cuda")
    sk.paged_attn(q, pool.cache(B, lens), out, lse)
    assert sk.status() == 0
    for s, m in enumerate(lens):
        t = torch.arange(m, device="cuda")
        want = O.attention(q[s], pool.rows("k", s, t), pool.rows("v", s, t), scale or 128 ** -0.5)
        # (a softmax scale is a 32-bit number: 2^-24 of a score more, below what is allowed for its sum)
        O.assert_attention(out[s], lse[s], *want, m, WEIGHTS[dtype])
    sk.close()


@pytest.mark.parametrize("seed", range(60))
def test_append(seed):
    rng = random.Random(1000 + seed)
    Hq, Hkv = shape(rng)
    n = rng.choice([1, 2, 3, 9])
    lens = [length(rng, rng.choice([30, 300, 2000]) // n + 16) for _ in range(n)]
    if not any(lens):
        lens[0] = 3
    appended(Hq, Hkv, lens, rng.choice([16, 32, 48, 80, 128]), rng.choice([BF16, E4M3]), rng.choice(TURNS + [None]), rng.choice(ORDERS),
             queries=rng.random() < 0.6, first=[rng.randint(0, 500) for _ in range(n)], padding=rng.randint(0, 9), fused=rng.random() < 0.5,
             batch=n + rng.randint(0, 2), scaled=rng.random() < 0.8)


@pytest.mark.parametrize("seed", range(40))
def test_score_and_compact(seed):
    from paper_2503_08879_b200 import binding as B
    rng = random.Random(2000 + seed)
    Hq, Hkv = shape(rng)
    G, n, N = Hq // Hkv, rng.choice([1, 1, 2, 3]), rng.choice([8, 40, 500, 3000, 20000])
    N = rng.randint(N // 2 + 2, N)
    S = rng.randint(0, N // 3)
    R = rng.randint(0, (N - 1 - S) // 2)
    E = N - 1 - S - R
    k_q = rng.randint(0, min(E + 2, 200))
    dtype, page = rng.choice([BF16, E4M3]), rng.choice([16, 32, 48, 64, 112, 256])
    sk = B.SageKV(Hq, Hkv, 128, n, max_ctx=N + rng.randint(0, 50), max_len=S + G * k_q + R + 1, device="cuda")
    pool = O.Pool(Hkv, page, n, -(-N // page) + rng.randint(0, 1), dtype, "cuda", rng.choice(ORDERS), seed=seed, scaled=rng.random() < 0.8).fill([N] * n)
    q = torch.randn(n, Hq, 128, generator=pool.gen, device="cuda").to(BF16)
    cache = pool.cache(B)
    K, V = (contiguous(pool, w, n, N) for w in "kv")
    idx, kept = None, min(k_q, E)
    if E > 0:
        scores = sk.paged_score(q, cache, N, S, R)
        qg = q.double().view(n, Hkv, G, 128)
        s = torch.einsum("bhgd,bhtd->bhgt", qg, K[:, :, S: S + E]) * 128 ** -0.5
        sizes = torch.einsum("bhgd,bhtd->bhgt", qg.abs(), K[:, :, S: S + E].abs()).amax(-1, keepdim=True) * 128 ** -0.5
        want = torch.softmax(s, -1).view(n * Hq, E)
        tol = (2 * (2.0 ** -21 * sizes + 2.0 ** -22)).view(n * Hq, 1) + 2.0 ** -24 * (E / 2048 + 64)   # as in test_gpu_paged_cache.py
        assert torch.all((scores[:, :E].double() - want).abs() <= tol * want + 1e-38)
        if kept:
            idx = torch.empty(n, Hq, kept, dtype=torch.int32, device="cuda")
            B.sagekv_select_topk(sk.ctx, scores, scores.stride(0), E, kept, idx)
    layer = sk.paged_compact(idx, cache, N, S, R, G * k_q)
    assert sk.status() == 0 and layer.state.k_q == kept
    L = layer.state.len
    for b in range(n):
        for h in range(Hkv):
            mine = idx[b, h * G: (h + 1) * G].reshape(-1).long() + S if kept else torch.zeros(0, dtype=torch.long, device="cuda")
            t = torch.cat([torch.arange(S, device="cuda"), mine, torch.arange(S + E, N, device="cuda")])
            for got, rows in ((layer.Kc, K), (layer.Vc, V)):
                want = rows[b, h, t]
                bound = (2.0 ** -8 + 2.0 ** -23) * want.abs() if dtype == E4M3 else torch.zeros_like(want)
                assert torch.all((got[b, h, :L].double() - want).abs() <= bound)
    sk.close()
