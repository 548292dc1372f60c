"""Long runs of tiles whose page id is none, one behind the other in every warp: they complete a copy barrier's phases without a
copy.  The tokens that are there give what they give alone, and the status word holds the bounds bit and no timeout."""

import math

import pytest
import torch

import paged_oracle as O
from test_gpu_paged_attn import WEIGHTS

pytestmark = pytest.mark.gpu
BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn


def sparse_pool(H, dtype, n_seqs, width, present):
    """`present[s]` are the pages of 16 tokens that sequence s has out of its table's `width`."""
    pool = O.Pool(H, 16, n_seqs, max(len(p) for p in present), dtype, "cuda")
    pool.fill([16 * len(p) for p in present])
    held, pool.table = pool.table, torch.full((n_seqs, width), -1, dtype=torch.int32, device="cuda")
    pool.table[:, 1::2] = pool.k.shape[0]                            # one kind of none beside the other
    for s, pages in enumerate(present):
        pool.table[s, pages] = held[s, : len(pages)]
    return pool


def tokens(pages):
    return (torch.tensor(pages, device="cuda")[:, None] * 16 + torch.arange(16, device="cuda")).flatten() if pages else torch.arange(0, device="cuda")


def only_bounds(B, sk):
    torch.cuda.synchronize()
    with pytest.raises(B.SagekvError) as e:
        sk.status()
    assert e.value.code == B.ERR_BOUNDS and e.value.bits == 2


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("Hq, Hkv", [(8, 2), (7, 1)])
def test_attention(Hq, Hkv, dtype):
    """2^18 tokens: dozens of tiles per warp, all but a few of them absent; one sequence without any page."""
    from paper_2503_08879_b200 import binding as B
    width = 1 << 14
    present = [[], [0, 1, 2, 700, 701, 5000, 9999, width - 1], list(range(width // 2, width // 2 + 40))]
    sk = B.SageKV(Hq, Hkv, 128, 3, max_ctx=64, max_len=16, device="cuda")
    pool = sparse_pool(Hkv, dtype, 3, width, present)
    q = torch.randn(3, Hq, 128, generator=pool.gen, device="cuda").to(BF16)
    lse = torch.empty(3, Hq, device="cuda")
    for _ in range(5):
        out = sk.paged_attn(q, pool.cache(B, [16 * width] * 3), None, lse)
        only_bounds(B, sk)
        for s, pages in enumerate(present):
            t = tokens(pages)
            want = O.attention(q[s], pool.rows("k", s, t), pool.rows("v", s, t), 128 ** -0.5)
            O.assert_attention(out[s], lse[s], *want, len(t), WEIGHTS[dtype])
    sk.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_score(dtype):
    from paper_2503_08879_b200 import binding as B
    Hq, Hkv, width, S, R = 8, 2, 1 << 14, 4, 10
    N = 16 * width
    E = N - 1 - S - R
    present = [list(range(100, 130)) + [3000, 3001, 3002, 12345]]
    sk = B.SageKV(Hq, Hkv, 128, 1, max_ctx=N, max_len=64, device="cuda")
    pool = sparse_pool(Hkv, dtype, 1, width, present)
    q = torch.randn(1, Hq, 128, generator=pool.gen, device="cuda").to(BF16)
    t = tokens(present[0])
    K = pool.rows("k", 0, t)
    qg = q[0].double().view(Hkv, Hq // Hkv, 128)
    want = torch.softmax(torch.einsum("hgd,thd->hgt", qg, K) / math.sqrt(128), -1).view(Hq, -1)
    sizes = (torch.einsum("hgd,thd->hgt", qg.abs(), K.abs()) / math.sqrt(128)).amax(-1).view(Hq, 1)
    tol = 2 * (2.0 ** -21 * sizes + 2.0 ** -22) + 2.0 ** -24 * (E / 2048 + 64)   # as in test_gpu_paged_cache.py
    for _ in range(5):
        p = sk.paged_score(q, pool.cache(B), N, S, R)[:, :E]
        only_bounds(B, sk)
        assert torch.all((p[:, t - S].double() - want).abs() <= tol * want + 1e-38)
        gone = torch.ones(E, dtype=torch.bool, device="cuda")
        gone[t - S] = False
        assert not p[:, gone].any()
    sk.close()
