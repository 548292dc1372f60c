"""The paged calls one behind the other, out of an 8-bit cache, against the calls without pages on the very same rows: bit for bit."""

import pytest
import torch

import paged_oracle as O
from test_gpu_paged_cache import TURNS, context, plan_of, random

pytestmark = pytest.mark.gpu
BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn


def widened(pool, which, n, N):
    """[n, H, N, 128] in bf16: code * scale in 32 bits, rounded once, as sagekv_paged_compact stores a row."""
    t = torch.arange(N, device="cuda")
    codes = torch.stack([pool.rows(which, s, t, scaled=False) for s in range(n)]).float()
    scale = getattr(pool, which + "_scale")
    return (codes if scale is None else codes * scale[:, None]).to(BF16).transpose(1, 2).contiguous()


@pytest.mark.parametrize("scaled", [True, False])
@pytest.mark.parametrize("Hq, Hkv", [(8, 2), (14, 2), (5, 5)])
def test_decode_from_an_8_bit_prompt_is_that_from_its_widened_rows(Hq, Hkv, scaled):
    N, S, R, k_q, steps, n = 2500, 4, 60, 90, 4, 2
    G, E = Hq // Hkv, N - 1 - S - R
    B, sk = context(Hq, Hkv, n, max_ctx=N + steps, max_len=S + G * k_q + R + 1)
    pool = O.Pool(Hkv, 64, n, -(-(N + steps) // 64), E4M3, "cuda", scaled=scaled)
    cache = pool.cache(B)
    plan, freq, amp = plan_of(B, TURNS[0], 500000.0)
    seq = torch.arange(n, device="cuda", dtype=torch.int32).repeat_interleave(N)
    pos = torch.arange(N, device="cuda", dtype=torch.int32).repeat(n)
    q = sk.paged_append(cache, random(n * N, Hkv, 128, seed=1), random(n * N, Hkv, 128, seed=2), pos, seq, plan, random(n * N, Hq, 128, seed=3, spread=3.0))
    scores = sk.paged_score(q.view(n, N, Hq, 128)[:, -1].contiguous(), cache, N, S, R)
    idx = torch.empty(n, Hq, k_q, dtype=torch.int32, device="cuda")
    B.sagekv_select_topk(sk.ctx, scores, scores.stride(0), E, k_q, idx)
    layer = sk.paged_compact(idx, cache, N, S, R, G * k_q)
    plain = sk.select_compact(scores, widened(pool, "k", n, N), widened(pool, "v", n, N), S, R, G * k_q)
    assert torch.equal(plain.indices(), idx + S)
    assert torch.equal(layer.Kc, plain.Kc) and torch.equal(layer.Vc, plain.Vc)
    for step in range(steps):
        q, k, v = (random(n, h, 128, seed=10 * step + i) for i, h in enumerate((Hq, Hkv, Hkv)))
        lse, plain_lse = torch.empty(n, Hq, device="cuda"), torch.empty(n, Hq, device="cuda")
        out, want = sk.decode_attn(q, k, v, layer, None, lse), sk.decode_attn(q, k, v, plain, None, plain_lse)
        assert torch.equal(out, want) and torch.equal(lse, plain_lse) and torch.isfinite(out).all()
    assert sk.status() == 0
    sk.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_hints_change_no_list(dtype):
    """sagekv_select_topk passes over the rows in every hint mode, also of scores that have a histogram or a list behind them."""
    N, S, R, G, k_q = 20011, 4, 128, 4, 100
    E = N - 1 - S - R
    B, sk = context(8, 2, 1, max_ctx=N, max_len=S + G * k_q + R + 1)
    pool = O.Pool(2, 64, 1, -(-N // 64), dtype, "cuda").fill([N])
    q = random(1, 8, 128, spread=2.0)
    for hint in (0, 1, 2):
        sk.set_select_hint(hint, G * k_q)
        scores = sk.paged_score(q, pool.cache(B), N, S, R)
        idx = torch.empty(1, 8, k_q, dtype=torch.int32, device="cuda")
        B.sagekv_select_topk(sk.ctx, scores, scores.stride(0), E, k_q, idx)
        want = torch.sort(scores[:, :E], dim=1, descending=True, stable=True).indices[:, :k_q].sort(dim=1).values
        assert torch.equal(idx[0].long(), want)
        layer = sk.paged_compact(idx, pool.cache(B), N, S, R, G * k_q)
        assert layer.state.k_q == k_q
    assert sk.status() == 0
    sk.close()
