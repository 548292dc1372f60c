"""The operators of the paged cache, as cases that can be timed and compared.

The full cache of a layer as a server keeps it: pages of `page` tokens, found through a block table, in bf16 or in e4m3
with a scale per KV head.  Five operators, each one call of the package:

  rope      query or key rows rotated by their positions (SageKV.rope)
  append    keys and values of new tokens into their pages, keys rotated on the way, the queries of the same tokens
            rotated beside them (SageKV.paged_append)
  attn      one new token per sequence attends to its whole cache (SageKV.paged_attn)
  score     the last token's query scores the eviction region of a paged cache (SageKV.paged_score)
  compact   the reduced cache from the pages and the kept positions (SageKV.paged_compact)

A case is a dict of plain values: op, q_heads, kv_heads, and
  rope      tokens, heads, rotary (dimensions that turn), interleaved, scaling, fused (rows are a slice of a wider tensor)
  append    seqs, tokens (in all; a prompt's share is ragged), page, cache ("bf16", "e4m3"), rotary, interleaved, scaling, queries
  attn      seqs, length (the longest), ragged, page, cache
  score     seqs, n_ctx, budget, page, cache
  compact   seqs, n_ctx, budget, page, cache
Where `own` is false, `run` computes the same in elementary torch operations.
"""

import math

import torch

own = False

LLAMA = dict(q_heads=32, kv_heads=8)      # Llama-3.1-8B, Llama-3-8B
QWEN = dict(q_heads=28, kv_heads=4)       # Qwen2.5-7B: seven query heads per KV head
N_INIT, N_RECENT = 4, 128                 # sink and recent tokens of the reduced cache
THETA = 500000.0
DIM = 128
DEV = "cuda"


def _rope(name, tokens, heads, rotary=128, interleaved=False, scaling="none", fused=False):
    c = dict(op="rope", tokens=tokens, heads=heads, rotary=rotary, interleaved=interleaved, scaling=scaling, fused=fused)
    return dict(c, name=name) if name else c


def _append(name, shape, seqs, tokens, page=16, cache="bf16", rotary=128, interleaved=False, scaling="none", queries=True):
    c = dict(op="append", seqs=seqs, tokens=tokens, page=page, cache=cache, rotary=rotary, interleaved=interleaved,
             scaling=scaling, queries=queries, **shape)
    return dict(c, name=name) if name else c


def _attn(name, shape, seqs, length, ragged=False, page=16, cache="bf16"):
    c = dict(op="attn", seqs=seqs, length=length, ragged=ragged, page=page, cache=cache, **shape)
    return dict(c, name=name) if name else c


def _reduce(op, name, shape, seqs, n_ctx, budget, page=16, cache="bf16"):
    c = dict(op=op, seqs=seqs, n_ctx=n_ctx, budget=budget, page=page, cache=cache, **shape)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the query of one new token, a quarter of each head turning in neighbouring pairs: launch latency and host work
        _rope("rope-token", 1, 32, rotary=32, interleaved=True),
        # the queries of a long prompt out of a fused projection, frequencies scaled in bands for a longer context
        _rope("rope-prompt-20k", 20011, 28, scaling="bands", fused=True),
        # a decode step of a serving batch: one token per sequence, queries, keys and values in one call
        _append("append-step-b32", LLAMA, 32, 32),
        # the prompts of eight sequences of uneven lengths enter an 8-bit cache, layer by layer
        _append("append-prompt-64k-e4m3", LLAMA, 8, 65537, page=64, cache="e4m3", scaling="yarn", queries=False),
        # one short conversation: all latency
        _attn("attn-300", LLAMA, 1, 300),
        # the long document that the package is quoted on, its whole cache read for one token
        _attn("attn-128k", LLAMA, 1, 131072),
        # a serving batch of uneven lengths (empty places among them), seven query heads per KV head
        _attn("attn-b48-ragged", QWEN, 48, 16384, ragged=True, page=32),
        # a batch of long contexts in an 8-bit cache
        _attn("attn-b8-32k-e4m3", LLAMA, 8, 32768, ragged=True, page=64, cache="e4m3"),
        # the selection's scores over the long document
        _reduce("score", "score-128k", LLAMA, 1, 131072, 2048),
        # the same on two shorter prompts of odd length in an 8-bit cache
        _reduce("score", "score-9k-b2-e4m3", QWEN, 2, 9001, 1024, page=32, cache="e4m3"),
        # the reduced cache of the long document
        _reduce("compact", "compact-128k", LLAMA, 1, 131072, 2048),
        # the largest budget, a batch of four, out of an 8-bit cache
        _reduce("compact", "compact-33k-b4-e4m3", QWEN, 4, 33333, 8192, page=64, cache="e4m3"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    shape = rng.choice([LLAMA, LLAMA, QWEN, dict(q_heads=16, kv_heads=2), dict(q_heads=8, kv_heads=8)])
    op = rng.choice(["rope", "append", "append", "attn", "attn", "attn", "score", "compact"])
    page = rng.choice([16, 16, 32, 48, 64, 128])
    cache = rng.choice(["bf16", "bf16", "e4m3"])
    turn = dict(rotary=rng.choice([128, 128, 96, 64, 32, 16]), interleaved=rng.random() < 0.4,
                scaling=rng.choice(["none", "linear", "bands", "yarn"]))
    if op == "rope":
        return _rope(None, _log_int(rng, 1, 20000), rng.choice([1, 4, 7, 8, 28, 32]), fused=rng.random() < 0.5, **turn)
    if op == "append":
        seqs = _log_int(rng, 1, 64)
        tokens = seqs if rng.random() < 0.4 else _log_int(rng, seqs, 65537 * 8 // (2 * shape["kv_heads"]))
        return _append(None, shape, seqs, tokens, page, cache, queries=rng.random() < 0.5, **turn)
    if op == "attn":
        seqs = _log_int(rng, 1, 64)
        length = _log_int(rng, 1, max(1, min(131072, 131072 * 8 // (seqs * shape["kv_heads"]))))
        return _attn(None, shape, seqs, length, seqs > 1 and rng.random() < 0.7, page, cache)
    n_ctx = _log_int(rng, 1024, 131072)
    seqs = rng.randint(1, max(1, min(4, 131072 * 8 // (n_ctx * shape["kv_heads"]))))
    return _reduce(op, None, shape, seqs, n_ctx, _log_int(rng, 256, min(8192, n_ctx // 2)), page, cache)


# ---- inputs ---------------------------------------------------------------------------------------------------


def _scaling(kind):
    return {"none": None, "linear": dict(kind="linear", factor=4.0),
            "bands": dict(kind="bands", factor=8.0, low=1.0, high=4.0, original_ctx=8192),
            "yarn": dict(kind="yarn", factor=4.0, low=1.0, high=32.0, original_ctx=32768)}[kind]


def _frequencies(case):
    """(radians per position of every pair, in 64 bits; factor on sine and cosine)"""
    r, s = case["rotary"], _scaling(case["scaling"])
    i = torch.arange(r // 2, dtype=torch.float64, device=DEV)
    f = THETA ** (-2.0 * i / r)
    if s is None:
        return f, 1.0
    if s["kind"] == "linear":
        return f / s["factor"], 1.0
    if s["kind"] == "bands":      # short wavelengths as they are, long ones stretched, a blend between
        turns = s["original_ctx"] * f / (2 * math.pi)
        blend = ((turns - s["low"]) / (s["high"] - s["low"])).clamp(0, 1)
        return f / s["factor"] * (1 - blend) + f * blend, 1.0
    where = lambda turns: r * math.log(s["original_ctx"] / (turns * 2 * math.pi)) / (2 * math.log(THETA))
    lo, hi = max(math.floor(where(s["high"])), 0), min(math.ceil(where(s["low"])), r - 1)
    ramp = ((i - lo) / (hi - lo if hi != lo else 0.001)).clamp(0, 1)
    return f / s["factor"] * ramp + f * (1 - ramp), 0.1 * math.log(s["factor"]) + 1.0


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.bfloat16)


def _pages(case, gen, tokens_per_seq, n_seqs):
    """Pools, block table and scales of a cache with room for tokens_per_seq tokens in every sequence, pages in random order."""
    page, H = case["page"], case["kv_heads"]
    width = -(-tokens_per_seq // page)
    n_pages = n_seqs * width + 3
    order = torch.randperm(n_pages, generator=gen, device=DEV)
    st = dict(table=order[: n_seqs * width].view(n_seqs, width).to(torch.int32), k_scale=None, v_scale=None)
    for name in ("k", "v"):
        pool = _normal(gen, n_pages, H, page, DIM)
        if case["cache"] == "e4m3":
            st[name + "_scale"] = torch.rand(H, generator=gen, device=DEV) * 0.02 + 0.01
            pool = (pool.float() / st[name + "_scale"][None, :, None, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
        st[name + "_pages"] = pool
    return st


def _prepare_rope(case, gen):
    T, H = case["tokens"], case["heads"]
    x = _normal(gen, T, H + 2 if case["fused"] else H, DIM)[:, :H]
    pos = torch.randint(0, 131072, (1,), generator=gen, device=DEV) + torch.arange(T, device=DEV)
    st = dict(x=x, pos=pos.to(torch.int32), out=torch.empty(T, H, DIM, dtype=torch.bfloat16, device=DEV))
    if own:
        from paper_2503_08879_b200 import binding as B
        st["sk"] = B.SageKV(H, H, DIM, 1, max_ctx=1024, max_len=64, device=DEV)
    return st


def _prepare_append(case, gen):
    n, T, H, Hq = case["seqs"], case["tokens"], case["kv_heads"], case["q_heads"]
    step = T == n
    if step:                       # one token each, behind caches of uneven lengths
        lens, before = [1] * n, torch.randint(0, 2048, (n,), generator=gen, device=DEV)
    else:
        share = [1 + 5 * b % 7 for b in range(n)]
        lens = [1 + (T - n) * x // sum(share) for x in share]
        lens[-1] += T - sum(lens)
        before = torch.zeros(n, dtype=torch.int64, device=DEV)
    seq = torch.repeat_interleave(torch.arange(n, device=DEV), torch.tensor(lens, device=DEV))
    first = torch.cumsum(torch.tensor([0] + lens[:-1], device=DEV), 0)
    pos = torch.arange(T, device=DEV) - first[seq] + before[seq]
    st = _pages(case, gen, 2049 if step else max(lens), n)
    st |= dict(seq=seq.to(torch.int32), pos=pos.to(torch.int32), k=_normal(gen, T, H, DIM), v=_normal(gen, T, H, DIM),
               q=_normal(gen, T, Hq, DIM) if case["queries"] else None)
    st["q_out"] = torch.empty_like(st["q"]) if case["queries"] else None
    if own:
        from paper_2503_08879_b200 import binding as B
        st["sk"] = B.SageKV(Hq, H, DIM, n, max_ctx=1024, max_len=64, device=DEV)
        st["cache"] = B.PagedCache(st["k_pages"], st["v_pages"], st["table"], k_scale=st["k_scale"], v_scale=st["v_scale"])
        st["steps"] = step
    return st


def _prepare_attn(case, gen):
    n, L, H, Hq = case["seqs"], case["length"], case["kv_heads"], case["q_heads"]
    st = _pages(case, gen, L, n)
    lens = torch.full((n,), L, device=DEV)
    if case["ragged"]:             # the shortest are a quarter, and one place in sixteen is empty
        lens = torch.randint(max(1, L // 4), L + 1, (n,), generator=gen, device=DEV)
        lens[torch.rand(n, generator=gen, device=DEV) < 1 / 16] = 0
        lens[0] = L
    st |= dict(lens=lens.to(torch.int32), q=_normal(gen, n, Hq, DIM) * 2, out=torch.empty(n, Hq, DIM, dtype=torch.bfloat16, device=DEV),
               lse=torch.empty(n, Hq, device=DEV))
    if own:
        from paper_2503_08879_b200 import binding as B
        st["sk"] = B.SageKV(Hq, H, DIM, n, max_ctx=1024, max_len=64, device=DEV)
        st["cache"] = B.PagedCache(st["k_pages"], st["v_pages"], st["table"], st["lens"], k_scale=st["k_scale"], v_scale=st["v_scale"])
    return st


def _kept(case):
    """tokens kept per query head, recent tokens (what a budget leaves over goes to them), size of the eviction region"""
    G = case["q_heads"] // case["kv_heads"]
    k_q = (case["budget"] - N_INIT - N_RECENT) // G
    recent = case["budget"] - N_INIT - G * k_q
    return k_q, recent, case["n_ctx"] - 1 - N_INIT - recent


def _prepare_reduce(case, gen):
    n, N, H, Hq = case["seqs"], case["n_ctx"], case["kv_heads"], case["q_heads"]
    k_q, recent, E = _kept(case)
    st = _pages(case, gen, N, n)
    if case["op"] == "score":
        st |= dict(q=_normal(gen, n, Hq, DIM) * 2, scores=torch.empty(n * Hq, -(-E // 4) * 4, device=DEV))
    else:
        idx = torch.rand(n * Hq, E, generator=gen, device=DEV).topk(k_q, dim=1).indices.sort(dim=1).values
        st["idx"] = idx.view(n, Hq, k_q).to(torch.int32)
    if own:
        from paper_2503_08879_b200 import binding as B
        st["sk"] = B.SageKV(Hq, H, DIM, n, max_ctx=N, max_len=case["budget"] + 1, device=DEV)
        st["cache"] = B.PagedCache(st["k_pages"], st["v_pages"], st["table"], k_scale=st["k_scale"], v_scale=st["v_scale"])
        if case["op"] == "compact":
            st["layer"] = st["sk"].new_layer(N_INIT, recent, Hq // H * k_q)
    return st


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    st = dict(rope=_prepare_rope, append=_prepare_append, attn=_prepare_attn, score=_prepare_reduce,
              compact=_prepare_reduce)[case["op"]](case, gen)
    if "rotary" in case:
        st["freq"], st["amplitude"] = _frequencies(case)
        if own:
            from paper_2503_08879_b200 import binding as B
            st["plan"] = B.sagekv_rope_plan(case["rotary"], case["interleaved"], THETA, _scaling(case["scaling"]))
    return dict(st, case=case)


# ---- one pass: the package's calls ------------------------------------------------------------------------------


def _own(st):
    case, sk = st["case"], st["sk"]
    if case["op"] == "rope":
        return sk.rope(st["x"], st["pos"], st["plan"], st["out"])
    if case["op"] == "append":
        sk.paged_append(st["cache"], st["k"], st["v"], st["pos"], None if st["steps"] else st["seq"], st["plan"], st["q"], st["q_out"])
        return dict(k=st["k_pages"], v=st["v_pages"], q=st["q_out"])
    if case["op"] == "attn":
        return dict(out=sk.paged_attn(st["q"], st["cache"], st["out"], st["lse"]), lse=st["lse"])
    k_q, recent, E = _kept(case)
    if case["op"] == "score":
        return sk.paged_score(st["q"], st["cache"], case["n_ctx"], N_INIT, recent, st["scores"])[:, :E]
    layer = sk.paged_compact(st["idx"], st["cache"], case["n_ctx"], N_INIT, recent, case["q_heads"] // case["kv_heads"] * k_q, st["layer"])
    return dict(k=layer.Kc, v=layer.Vc, step=layer.step)


# ---- one pass: the plain forms ----------------------------------------------------------------------------------


def _turn(x, pos, st):
    """Rows x [tokens, heads, 128] (32 bits) rotated; angles in 64 bits, products in 32."""
    r = st["case"]["rotary"]
    angle = pos.to(torch.float64)[:, None] * st["freq"]
    cos, sin = (angle.cos() * st["amplitude"]).float()[:, None], (angle.sin() * st["amplitude"]).float()[:, None]
    y = x.clone()
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if st["case"]["interleaved"] else (x[..., : r // 2], x[..., r // 2: r])
    ya, yb = a * cos - b * sin, b * cos + a * sin
    if st["case"]["interleaved"]:
        y[..., 0:r:2], y[..., 1:r:2] = ya, yb
    else:
        y[..., : r // 2], y[..., r // 2: r] = ya, yb
    return y


def _store(pool, scale, table, seq, pos, rows):
    """rows [tokens, heads, 128] (32 bits) into their pages, rounded to the pool's type."""
    page = pool.shape[2]
    where = table[seq.long(), (pos // page).long()].long()
    if scale is not None:
        rows = (rows / scale[None, :, None]).clamp(-448, 448)
    raw = torch.uint8 if scale is not None else torch.int16
    heads = torch.arange(pool.shape[1], device=DEV)
    pool.view(raw)[where[:, None], heads[None], (pos % page).long()[:, None]] = rows.to(pool.dtype).view(raw)


def _rows(pool, scale, table):
    """The sequences' rows [seqs, heads, tokens, 128] in 32 bits."""
    n, width = table.shape
    raw = pool.view(torch.uint8)[table.long()].view(pool.dtype)
    x = raw.permute(0, 2, 1, 3, 4).reshape(n, pool.shape[1], width * pool.shape[2], DIM).float()
    return x if scale is None else x * scale[None, :, None, None]


def _plain(st):
    case = st["case"]
    if case["op"] == "rope":
        return _turn(st["x"].float(), st["pos"], st).to(torch.bfloat16)
    if case["op"] == "append":
        _store(st["k_pages"], st["k_scale"], st["table"], st["seq"], st["pos"], _turn(st["k"].float(), st["pos"], st))
        _store(st["v_pages"], st["v_scale"], st["table"], st["seq"], st["pos"], st["v"].float())
        q = _turn(st["q"].float(), st["pos"], st).to(torch.bfloat16) if case["queries"] else None
        return dict(k=st["k_pages"], v=st["v_pages"], q=q)
    n, H, Hq = case["seqs"], case["kv_heads"], case["q_heads"]
    K = _rows(st["k_pages"], st["k_scale"], st["table"])
    if case["op"] == "score":
        _, recent, E = _kept(case)
        s = torch.matmul(st["q"].float().view(n, H, Hq // H, DIM), K[:, :, N_INIT: N_INIT + E].transpose(2, 3)) / math.sqrt(DIM)
        p = (s - s.amax(dim=-1, keepdim=True)).exp()
        return (p / p.sum(dim=-1, keepdim=True)).view(n * Hq, E)
    V = _rows(st["v_pages"], st["v_scale"], st["table"])
    if case["op"] == "attn":
        s = torch.matmul(st["q"].float().view(n, H, Hq // H, DIM), K.transpose(2, 3)) / math.sqrt(DIM)
        there = torch.arange(K.shape[2], device=DEV) < st["lens"][:, None]
        s = s.masked_fill(~there[:, None, None], -math.inf)
        m = s.amax(dim=-1, keepdim=True).clamp(min=-1e30)
        p = (s - m).exp()
        total = p.sum(dim=-1, keepdim=True)
        out = torch.matmul(p, V) / total.clamp(min=1e-30)
        return dict(out=out.to(torch.bfloat16).view(n, Hq, DIM), lse=(m + total.log()).view(n, Hq))
    k_q, recent, E = _kept(case)
    sink, tail = torch.arange(N_INIT, device=DEV), torch.arange(N_INIT + E, case["n_ctx"], device=DEV)
    kept = st["idx"].view(n, H, Hq // H * k_q).long() + N_INIT
    at = torch.cat([sink.expand(n, H, -1), kept, tail.expand(n, H, -1)], dim=2)[..., None].expand(-1, -1, -1, DIM)
    return dict(k=K.gather(2, at).to(torch.bfloat16), v=V.gather(2, at).to(torch.bfloat16),
                step=torch.zeros(1, dtype=torch.int32, device=DEV))


def run(state):
    return _own(state) if own else _plain(state)


# ---- from the definitions, in 64 bits -----------------------------------------------------------------------------


def _exact_turn(x, pos, st):
    """A pair of dimensions as a complex number, multiplied by the unit number of its angle."""
    r, x = st["case"]["rotary"], x.double()
    pair = x[..., :r].unflatten(-1, (r // 2, 2)) if st["case"]["interleaved"] else x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2)
    z = torch.view_as_complex(pair.contiguous())
    z = z * torch.polar(torch.full_like(st["freq"], st["amplitude"]), pos.double()[:, None] * st["freq"])[:, None]
    y = torch.view_as_real(z)
    y = y.flatten(-2) if st["case"]["interleaved"] else y.transpose(-1, -2).flatten(-2)
    return torch.cat([y, x[..., r:]], dim=-1)


def _exact_sequence(st, which, b, h, tokens):
    """The given tokens' rows of one sequence and head, one page entry each."""
    pool, scale, page = st[which + "_pages"], st[which + "_scale"], st["case"]["page"]
    ids = st["table"][b].long()[tokens // page]
    x = pool.view(torch.uint8).view(*pool.shape[:3], -1)[ids, h, tokens % page].view(pool.dtype).double()
    return x if scale is None else x * scale[h].double()


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_turn(st["x"], st["pos"], st)
    if case["op"] == "append":
        got = dict(q=_exact_turn(st["q"], st["pos"], st) if case["queries"] else None)
        slot = st["pos"].long() + st["seq"].long() * st["table"].shape[1] * case["page"]
        for which in ("k", "v"):
            pool, scale = st[which + "_pages"], st[which + "_scale"]
            new = _exact_turn(st["k"], st["pos"], st) if which == "k" else st["v"].double()
            if scale is not None:
                new = (new / scale.double()[:, None]).clamp(-448, 448)
            flat = pool.double().permute(0, 2, 1, 3)
            rows = flat.reshape(-1, case["kv_heads"], DIM)
            page_of = st["table"].reshape(-1).long()[slot // case["page"]]
            rows[page_of * case["page"] + slot % case["page"]] = new if scale is None else new.to(torch.float8_e4m3fn).double()
            got[which] = rows.view(flat.shape).permute(0, 2, 1, 3)
        return got
    n, H, Hq = case["seqs"], case["kv_heads"], case["q_heads"]
    G, dev = Hq // H, DEV
    if case["op"] == "compact":
        k_q, recent, E = _kept(case)
        got = dict(k=[], v=[])
        for b in range(n):
            for h in range(H):
                kept = st["idx"][b, h * G: (h + 1) * G].reshape(-1).long() + N_INIT
                tokens = torch.cat([torch.arange(N_INIT, device=dev), kept, torch.arange(N_INIT + E, case["n_ctx"], device=dev)])
                for which in ("k", "v"):
                    got[which].append(_exact_sequence(st, which, b, h, tokens))
        return dict(step=None, **{w: torch.stack(x).view(n, H, -1, DIM) for w, x in got.items()})
    outs, lses, probs = [], [], []
    for b in range(n):
        for h in range(H):
            if case["op"] == "score":
                _, recent, E = _kept(case)
                tokens = torch.arange(N_INIT, N_INIT + E, device=dev)
            else:
                tokens = torch.arange(int(st["lens"][b]), device=dev)
            q = st["q"][b, h * G: (h + 1) * G].double()
            s = q @ _exact_sequence(st, "k", b, h, tokens).t() * DIM ** -0.5
            lse = torch.logsumexp(s, dim=1)
            p = torch.exp(s - lse[:, None])
            if case["op"] == "score":
                probs.append(p)
            else:
                outs.append(p @ _exact_sequence(st, "v", b, h, tokens))
                lses.append(lse)
    if case["op"] == "score":
        return torch.cat(probs)
    return dict(out=torch.cat(outs).view(n, Hq, DIM), lse=torch.cat(lses).view(n, Hq))


# ---- what a pass cannot do without ----------------------------------------------------------------------------------


def _expected(case):
    """tokens in all of the sequences of an attn case, in the mean"""
    n, L = case["seqs"], case["length"]
    return n * L if not case["ragged"] else L + (n - 1) * 15 / 16 * (max(1, L // 4) + L) / 2


def work(case):
    if case["op"] == "rope":
        rows = case["tokens"] * case["heads"]
        return dict(bytes=rows * DIM * 4 + case["tokens"] * 4, flops=rows * case["rotary"] * 3)
    size = 1 if case["cache"] == "e4m3" else 2
    H, Hq, n = case["kv_heads"], case["q_heads"], case["seqs"]
    if case["op"] == "append":
        T = case["tokens"]
        queries = Hq if case["queries"] else 0
        return dict(bytes=T * DIM * (2 * H * (2 + size) + 4 * queries) + 8 * T, flops=T * (H + queries) * case["rotary"] * 3)
    if case["op"] == "attn":
        tokens = _expected(case)
        return dict(bytes=tokens * H * DIM * 2 * size + n * Hq * (DIM * 4 + 4) + tokens / case["page"] * 4, flops=tokens * Hq * DIM * 4)
    k_q, recent, E = _kept(case)
    if case["op"] == "score":
        return dict(bytes=n * (H * E * DIM * size + Hq * E * 4 + Hq * DIM * 2), flops=n * Hq * E * DIM * 2)
    rows = n * H * (case["budget"] + 1)
    return dict(bytes=rows * DIM * 2 * (size + 2) + n * Hq * k_q * 4, flops=rows * DIM * 2)
