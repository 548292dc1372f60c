"""Attention of one new token per sequence over a paged cache, against 64 bits."""

import math

import pytest
import torch

import paged_oracle as O

pytestmark = pytest.mark.gpu
BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn
WEIGHTS = {BF16: 2.0 ** -8, E4M3: 2.0 ** -11}                     # half a step of the type the weights are rounded to


def context(Hq, Hkv, batch, **kw):
    from paper_2503_08879_b200 import binding as B
    return B, B.SageKV(Hq, Hkv, 128, batch, max_ctx=1024, max_len=64, device="cuda", **kw)


def queries(pool, n, Hq, spread=1.0):
    return (torch.randn(n, Hq, 128, generator=pool.gen, device="cuda") * spread).to(BF16)


def check(pool, lens, q, out, lse, scale=128 ** -0.5):
    for s, n in enumerate(lens):
        t = torch.arange(n, device="cuda")
        want, want_lse, sizes, mean = O.attention(q[s], pool.rows("k", s, t), pool.rows("v", s, t), scale)
        O.assert_attention(out[s], None if lse is None else lse[s], want, want_lse, sizes, mean, n, WEIGHTS[pool.dtype])


def run(Hq, Hkv, lens, page=16, dtype=BF16, order=(0, 1, 2), batch=None, spread=1.0, want_lse=True, max_pages=None, **kw):
    n = len(lens)
    B, sk = context(Hq, Hkv, batch or n, **kw)
    pool = O.Pool(Hkv, page, n, max_pages or max(1, -(-max(lens) // page)), dtype, "cuda", order).fill(lens, spread)
    q = queries(pool, n, Hq, spread)
    out = torch.full((n + 2, Hq, 128), 7.0, dtype=BF16, device="cuda")
    lse = torch.full((n + 2, Hq), 7.0, device="cuda") if want_lse else None
    cache = pool.cache(B, lens)
    sk.paged_attn(q, cache, out, lse)
    torch.cuda.synchronize()
    assert sk.status() == 0
    check(pool, lens, q, out, lse, kw.get("softmax_scale") or 128 ** -0.5)
    assert torch.all(out[n:] == 7) and (lse is None or torch.all(lse[n:] == 7))      # rows behind the last sequence
    again = torch.zeros_like(out)
    sk.paged_attn(q, cache, again, lse)
    assert torch.equal(again[:n], out[:n])                        # the same bits, whoever arrives last
    sk.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("length", [0, 1, 2, 9, 15, 16, 17, 31, 33, 64, 65, 100, 300, 1000])
def test_one_sequence(length, dtype):
    run(32, 8, [length], dtype=dtype)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (2, 1), (3, 1), (8, 8), (10, 2), (6, 1), (28, 4), (16, 2), (5, 5)])
def test_head_counts(Hq, Hkv, dtype):
    run(Hq, Hkv, [77, 0, 513], dtype=dtype, page=32)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("page", [16, 32, 48, 80, 128, 1024])
@pytest.mark.parametrize("order", [(0, 1, 2), (0, 2, 1), (1, 0, 2), (2, 0, 1)])
def test_page_sizes_and_layouts(page, order, dtype):
    run(8, 2, [1000, 5, 161], page=page, order=order, dtype=dtype)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("lens", [[0, 0, 0], [0, 0, 40, 0, 0, 0, 700, 1, 0], [1] * 50, [3000] + [1] * 30, [16] * 7 + [4000, 0, 0],
                                  [5000, 17, 5000], list(range(70))])
def test_uneven_batches(lens, dtype):
    run(16, 4, lens, dtype=dtype)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("n", [127, 128, 129, 300, 777])
def test_many_sequences(n, dtype):
    """More sequences than a block has threads: each looks through several lengths."""
    run(4, 1, [(37 * s * s + 11 * s) % 90 if s % 5 else 0 for s in range(n)], dtype=dtype)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_a_long_sequence_of_one_head_is_shared_by_every_cta(dtype):
    run(4, 1, [70001], dtype=dtype, page=64)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("Hq, Hkv, lens", [(8, 1, [60000]), (7, 1, [9000]), (3, 1, [30000, 2, 25000]), (16, 2, [20000]), (5, 1, [40000, 40000, 1]), (1, 1, [28416]),
                                           (8, 1, [3500, 0, 3600])])
def test_pairs_of_very_many_parts(Hq, Hkv, lens, dtype):
    """Up to a part per CTA: more than 36 (eight heads) or 72 (four) are joined in groups first."""
    run(Hq, Hkv, lens, dtype=dtype, page=48)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_long_tables_and_a_batch_that_is_not_full(dtype):
    run(8, 2, [50, 2000], dtype=dtype, batch=9, max_pages=4000)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("spread, scale", [(0.001, 0.0), (6.0, 0.0), (1.0, 0.9), (3e4, 1e-9)])
def test_sharp_and_flat_weights(spread, scale, dtype):
    run(8, 2, [900, 33], dtype=dtype, spread=spread, softmax_scale=scale, want_lse=scale != 1e-9)


def test_a_table_without_columns_and_one_of_a_wider_table():
    B, sk = context(8, 2, 3)
    pool = O.Pool(2, 16, 3, 6, BF16, "cuda").fill([90, 20, 64])
    q = queries(pool, 3, 8)
    none = B.PagedCache(pool.k, pool.v, pool.table[:, :0], torch.zeros(3, dtype=torch.int32, device="cuda"))
    lse = torch.zeros(3, 8, device="cuda")
    assert not sk.paged_attn(q, none, None, lse).any() and torch.all(lse == -math.inf) and sk.status() == 0
    lens = [64, 20, 64]
    some = B.PagedCache(pool.k, pool.v, pool.table[:, :4], torch.tensor(lens, dtype=torch.int32, device="cuda"))
    out = sk.paged_attn(q, some, None, lse)
    check(pool, lens, q, out, lse)
    assert sk.status() == 0
    sk.close()


def test_without_lse_and_with_strided_queries():
    B, sk = context(8, 2, 3)
    lens = [100, 0, 35]
    pool = O.Pool(2, 16, 3, 7, BF16, "cuda").fill(lens)
    fused = queries(pool, 3, 12)
    q = fused[:, 2:10]
    out = sk.paged_attn(q, pool.cache(B, lens))
    check(pool, lens, q, out, None)
    sk.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_small_weights_are_not_lost(dtype):
    """One token far above 20000 others whose weights are 2^-26 of its own, together 2^-11.7: each is far below the steps of
    f16 around 1."""
    B, sk = context(1, 1, 1)
    n = 20001
    pool = O.Pool(1, 16, 1, -(-n // 16), dtype, "cuda", scaled=False).fill([n])
    q = torch.zeros(1, 1, 128, dtype=BF16, device="cuda")
    q[0, 0, 0] = 16.0
    t = torch.arange(n, device="cuda")
    raw = pool.raw("k")
    rows = torch.zeros(n, 1, 128, device="cuda")
    rows[7777, 0, 0] = 26 * math.log(2) * 128 ** 0.5 / 16           # (rounded by the type: about 2^-26)
    raw[pool.table[0, t // 16].long()[:, None], 0, (t % 16)[:, None]] = rows.to(dtype).view(raw.dtype)
    raw = pool.raw("v")
    rows = torch.full((n, 1, 128), 64.0, device="cuda")
    rows[7777] = 0.0
    raw[pool.table[0, t // 16].long()[:, None], 0, (t % 16)[:, None]] = rows.to(dtype).view(raw.dtype)
    lse = torch.empty(1, 1, device="cuda")
    out = sk.paged_attn(q, pool.cache(B, [n]), None, lse)
    check(pool, [n], q, out, lse)
    assert float(out.float().min()) > 0.01
    sk.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_queries_of_every_size(dtype):
    """Largest and smallest bf16 queries, zero ones, and queries whose elements differ by 2^40."""
    B, sk = context(8, 1, 1)
    pool = O.Pool(1, 16, 1, 10, dtype, "cuda").fill([150])
    q = queries(pool, 1, 8)
    q[0, 1] = 0
    q[0, 2] *= 2.0 ** -120
    q[0, 3] *= 2.0 ** 15
    q[0, 4, ::2] *= 2.0 ** -40
    q[0, 5, 1:] = 0
    q[0, 6] *= 2.0 ** -140
    q[0, 7] *= 2.0 ** -14
    lse = torch.empty(1, 8, device="cuda")
    out = sk.paged_attn(q, pool.cache(B, [150]), None, lse)
    check(pool, [150], q, out, lse)
    sk.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_values_that_are_not_finite_come_through(dtype):
    """NaN in a row that counts reaches the outputs that it should, and only those; behind the end nothing does (the
    pools hold NaN there in every test)."""
    B, sk = context(4, 2, 3)
    lens = [50, 40, 30]
    pool = O.Pool(2, 16, 3, 4, dtype, "cuda").fill(lens)
    nan = 0x7f if dtype == E4M3 else 0x7fc0
    q = queries(pool, 3, 4)
    pool.raw("v")[int(pool.table[0, 2]), 0, 5, 9] = nan             # sequence 0, token 37, head 0, column 9
    pool.raw("k")[int(pool.table[1, 0]), 1, 3, 0] = nan             # sequence 1, token 3, head 1
    out = sk.paged_attn(q, pool.cache(B, lens)).float()
    want = torch.zeros(3, 4, 128, dtype=torch.bool, device="cuda")
    want[0, 0:2, 9] = True
    want[1, 2:4] = True
    assert torch.equal(torch.isnan(out), want)
    assert sk.status() == 0
    sk.close()


def test_offsets_beyond_32_bits():
    """Pages more than 2^32 elements from the pool's start."""
    B, sk = context(4, 2, 2)
    page, H = 16, 2
    n_pages = (2 ** 32 + 2 ** 26) // (H * page * 128)
    pool = O.Pool(H, page, 2, 4, E4M3, "cuda")
    k = torch.empty(n_pages, H, page, 128, dtype=torch.uint8, device="cuda").view(E4M3)
    v = torch.empty(n_pages, H, page, 128, dtype=torch.uint8, device="cuda").view(E4M3)
    pool.k, pool.v = k, v
    pool.table = torch.tensor([[n_pages - 1, 0, n_pages - 9, 5], [n_pages - 2, 2 ** 32 // (H * page * 128), 3, 1]], dtype=torch.int32, device="cuda")
    lens = [64, 50]
    pool.fill(lens)
    q = queries(pool, 2, 4)
    lse = torch.empty(2, 4, device="cuda")
    out = sk.paged_attn(q, pool.cache(B, lens), None, lse)
    check(pool, lens, q, out, lse)
    sk.close()


def test_sequences_may_share_pages():
    B, sk = context(8, 2, 4)
    lens = [100, 100, 70, 33]
    pool = O.Pool(2, 16, 4, 7, BF16, "cuda")
    pool.table[1:] = pool.table[0]
    pool.fill([100, 0, 0, 0])
    q = queries(pool, 4, 8)
    out = sk.paged_attn(q, pool.cache(B, lens))
    check(pool, lens, q, out, None)
    sk.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_bad_pages_and_lengths_are_left_out_and_reported(dtype):
    """Every id and length here is checked by the kernel before it forms an address (tests/test_paged_host.py checks the
    address function on the host): tokens of pages that are none count as absent, lengths are cut to the table."""
    B, sk = context(4, 2, 5)
    lens = [64, 64, 64, 40, 20]
    pool = O.Pool(2, 16, 5, 4, dtype, "cuda").fill(lens)
    q = queries(pool, 5, 4)
    cache = pool.cache(B, lens)
    good = pool.table.clone()
    n_pages = pool.k.shape[0]
    pool.table[0, 1] = -1
    pool.table[1, 0] = n_pages
    pool.table[1, 3] = 2 ** 31 - 1
    pool.table[2] = -2 ** 31                                        # all of them
    lse = torch.empty(5, 4, device="cuda")
    out = sk.paged_attn(q, cache, None, lse)
    with pytest.raises(B.SagekvError) as e:
        sk.status()
    assert e.value.code == B.ERR_BOUNDS and e.value.bits == 2
    pool.table.copy_(good)
    present = [[0, 2, 3], [1, 2], [], [0, 1, 2], [0, 1]]
    for s, pages in enumerate(present):
        t = torch.cat([torch.arange(16 * p, min(16 * p + 16, lens[s]), device="cuda") for p in pages] + [torch.arange(0, device="cuda")])
        want = O.attention(q[s], pool.rows("k", s, t), pool.rows("v", s, t), 128 ** -0.5)
        O.assert_attention(out[s], lse[s], *want, len(t), WEIGHTS[dtype])
    pool.lens.copy_(torch.tensor([64, -5, 64, 40, -2 ** 31], dtype=torch.int32))
    out = sk.paged_attn(q, cache, None, lse)
    with pytest.raises(B.SagekvError):
        sk.status()
    check(pool, [64, 0, 64, 40, 0], q, out, lse)
    pool.fill([0, 0, 64, 0, 0])
    pool.lens.copy_(torch.tensor([64, 0, 2 ** 31 - 1, 40, 0], dtype=torch.int32))
    out = sk.paged_attn(q, cache, None, lse)
    with pytest.raises(B.SagekvError):
        sk.status()
    check(pool, [64, 0, 64, 40, 0], q, out, lse)
    sk.paged_attn(q[:4], cache_of(B, pool, [64, 0, 64, 40]), None, lse)
    assert sk.status() == 0
    sk.close()


def cache_of(B, pool, lens):
    pool.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    return B.PagedCache(pool.k, pool.v, pool.table[: len(lens)], pool.lens, pool.k_scale, pool.v_scale)


def test_captured_calls_read_the_lengths_and_tables_of_the_replay():
    """Two graphs of one context, replayed in turn, after lengths, tables and queries have changed."""
    B, sk = context(8, 2, 3)
    lens = [300, 5, 170]
    pool = O.Pool(2, 16, 3, 20, BF16, "cuda").fill([320, 320, 320])
    q, out, out2 = queries(pool, 3, 8), torch.zeros(3, 8, 128, dtype=BF16, device="cuda"), torch.zeros(3, 8, 128, dtype=BF16, device="cuda")
    cache = pool.cache(B, lens)
    sk.paged_attn(q, cache, out)
    torch.cuda.synchronize()
    graphs = []
    for o in (out, out2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            sk.paged_attn(q, cache, o)
    for k, new in enumerate([[0, 320, 1], [320, 320, 320], [17, 0, 0], [1, 2, 3]]):
        pool.lens.copy_(torch.tensor(new, dtype=torch.int32))
        pool.table.copy_(pool.table[:, torch.randperm(20, device="cuda")])
        q.copy_(queries(pool, 3, 8))
        graphs[k % 2].replay()
        graphs[1 - k % 2].replay()
        torch.cuda.synchronize()
        check(pool, new, q, out, None)
        assert torch.equal(out, out2)
    assert sk.status() == 0
    sk.close()


def test_on_another_stream_behind_the_work_that_makes_its_inputs():
    B, sk = context(8, 2, 2)
    lens = [2000, 900]
    pool = O.Pool(2, 16, 2, 125, BF16, "cuda").fill(lens)
    cache = pool.cache(B, lens)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        q = queries(pool, 2, 8)
        for _ in range(5):
            big = torch.randn(4096, 4096, device="cuda") @ torch.randn(4096, 4096, device="cuda")
            q.copy_((big[:2, :1024].reshape(2, 8, 128) * 0.01).to(BF16))
            out = sk.paged_attn(q, cache)
    side.synchronize()
    check(pool, lens, q, out, None)
    sk.close()


def test_two_contexts_at_once():
    """Contexts share nothing: calls of two of them may overlap on two streams."""
    lens = [1500, 300, 0, 900]
    B, a = context(8, 2, 4)
    _, b = context(8, 2, 4)
    pool = O.Pool(2, 16, 4, 100, BF16, "cuda").fill(lens)
    q, cache = queries(pool, 4, 8), pool.cache(B, lens)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = []
    for _ in range(20):
        for sk, s in ((a, s1), (b, s2)):
            with torch.cuda.stream(s):
                outs.append(sk.paged_attn(q, cache))
    torch.cuda.synchronize()
    check(pool, lens, q, outs[0], None)
    assert all(torch.equal(o, outs[0]) for o in outs)
    a.close(), b.close()


def test_refusals():
    B, sk = context(8, 2, 3)
    lens = [10, 20, 30]
    pool = O.Pool(2, 16, 3, 2, BF16, "cuda").fill(lens)
    q, out, cache = queries(pool, 3, 8), torch.full((3, 8, 128), 7.0, dtype=BF16, device="cuda"), pool.cache(B, lens)
    code = lambda *a: pytest.raises(B.SagekvError, B.sagekv_paged_attn, sk.ctx, *a).value.code
    assert code(None, cache, out) == B.ERR_INVALID
    assert code(q, None, out) == B.ERR_INVALID
    assert code(q, cache, None) == B.ERR_INVALID
    assert code(q, B.PagedCache(pool.k, pool.v, pool.table), out) == B.ERR_INVALID            # no lengths
    assert code(torch.empty(3, 4, 128, dtype=BF16, device="cuda"), cache, out) == B.ERR_INVALID   # sequences closer than H_q rows
    flat = torch.empty(3 * 1032 + 4, dtype=BF16, device="cuda")
    assert code(flat[4: 4 + 24 * 128].view(3, 8, 128), cache, out) == B.ERR_ALIGN
    assert code(torch.as_strided(flat, (3, 8, 128), (1028, 128, 1)), cache, out) == B.ERR_ALIGN
    wide = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    assert code(q, B.PagedCache(pool.k, pool.v, wide, torch.zeros(4, dtype=torch.int32, device="cuda")), out) == B.ERR_UNSUPPORTED
    small = torch.zeros(4, 2, 8, 128, dtype=BF16, device="cuda")
    assert code(q, B.PagedCache(small, small, pool.table, pool.lens), out) == B.ERR_UNSUPPORTED
    for bad in (dict(q=q[:2], cache=cache), dict(q=q, cache=cache, out=out[:2]), dict(q=q[:, :4], cache=cache),
                dict(q=q, cache=cache, out=out, lse=torch.empty(2, 8, device="cuda"))):
        with pytest.raises(ValueError):
            sk.paged_attn(**bad)
    torch.cuda.synchronize()
    assert torch.all(out == 7) and sk.status() == 0
    none = B.PagedCache(pool.k, pool.v, pool.table[:0], pool.lens[:0])
    assert B.sagekv_paged_attn(sk.ctx, q, none, out) is None                                  # no sequences: nothing to do
    sk.close()
