"""The paged cache's operators from their definitions, in 64 bits (torch on whatever device the inputs are), and inputs
for their tests.  Nothing here calls the library."""

import math

import torch

E4M3_MOST = 448.0


def frequencies(r, theta=10000.0):
    return theta ** (-2.0 * torch.arange(r // 2, dtype=torch.float64) / r)


def rotate(x, pos, freq, interleaved=False, amplitude=1.0):
    """Rows [tokens, heads, 128] rotated, one pair after the other."""
    r, y = 2 * len(freq), x.double().clone()
    angle = pos.double()[:, None] * freq.to(x.device)
    for i in range(r // 2):
        u, w = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
        c, s = (amplitude * angle[:, i].cos())[:, None], (amplitude * angle[:, i].sin())[:, None]
        a, b = x[..., u].double(), x[..., w].double()
        y[..., u], y[..., w] = a * c - b * s, b * c + a * s
    return y


def pair_size(x, freq, interleaved=False, amplitude=1.0):
    """|x_u| + |x_w| of every element's pair (|x| of those that stay): what a rounding in the rotation is relative to."""
    r, a = 2 * len(freq), x.double().abs()
    y = a.clone()
    u, w = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    y[..., u] = y[..., w] = (a[..., u] + a[..., w]) * amplitude
    return y


class Pool:
    """Pages in random order, every slot that no token has holding NaN; `order` is the order of the first three dimensions in memory."""

    def __init__(self, H, page, n_seqs, max_pages, dtype, dev, order=(0, 1, 2), spare=3, seed=0, scaled=True):
        g = torch.Generator(device=dev).manual_seed(seed)
        self.gen, self.H, self.page, self.dtype = g, H, page, dtype
        n_pages = n_seqs * max_pages + spare
        shape = [n_pages, H, page]
        raw = torch.uint8 if dtype == torch.float8_e4m3fn else torch.int16
        back = [order.index(i) for i in range(3)]

        def empty():
            nan = 0x7f if raw == torch.uint8 else 0x7fc0
            flat = torch.full([shape[i] for i in order] + [128], nan, dtype=raw, device=dev)
            return flat.permute(*back, 3).view(dtype)

        self.k, self.v = empty(), empty()
        self.table = torch.randperm(n_pages, generator=g, device=dev)[: n_seqs * max_pages].view(n_seqs, max_pages).to(torch.int32)
        self.k_scale = self.v_scale = None
        if dtype == torch.float8_e4m3fn and scaled:
            self.k_scale = torch.rand(H, generator=g, device=dev) * 0.02 + 0.005
            self.v_scale = torch.rand(H, generator=g, device=dev) * 0.02 + 0.005

    def raw(self, which):
        t = getattr(self, which)
        return t.view(torch.uint8 if self.dtype == torch.float8_e4m3fn else torch.int16)

    def fill(self, lens, spread=1.0):
        """Random rows for the first lens[s] tokens of every sequence."""
        for s, n in enumerate(lens):
            for which in "kv":
                if n:
                    x = torch.randn(n, self.H, 128, generator=self.gen, device=self.k.device) * spread
                    scale = getattr(self, which + "_scale")
                    if scale is not None:
                        x = (x / scale[:, None]).clamp(-E4M3_MOST, E4M3_MOST)
                    t = torch.arange(n, device=self.k.device)
                    pages = self.table[s, t // self.page].long()
                    self.raw(which)[pages[:, None], torch.arange(self.H, device=self.k.device)[None], (t % self.page)[:, None]] = \
                        x.to(self.dtype).view(self.raw(which).dtype)
        return self

    def rows(self, which, s, tokens, scaled=True):
        """[tokens, H, 128] in 64 bits."""
        raw = self.raw(which)
        x = raw[self.table[s, tokens // self.page].long()[:, None], torch.arange(self.H, device=raw.device)[None], (tokens % self.page)[:, None]]
        x = x.view(self.dtype).double()
        scale = getattr(self, which + "_scale")
        return x * scale.double()[:, None] if scale is not None and scaled else x

    def cache(self, B, lens=None):
        self.lens = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=self.k.device)
        return B.PagedCache(self.k, self.v, self.table, self.lens, self.k_scale, self.v_scale)


def attention(q, K, V, scale):
    """One sequence: q [H_q, 128], K and V [tokens, H_kv, 128] in 64 bits.  Returns out, lse, and what errors are relative to: the
    largest sum of absolute products behind a score (scaled), and sum of weights times |V| per output."""
    Hq, (n, H) = q.shape[0], K.shape[:2]
    if n == 0:
        z = torch.zeros(Hq, 128, dtype=torch.float64, device=q.device)
        return z, torch.full((Hq,), -math.inf, dtype=torch.float64, device=q.device), z[:, 0], z
    G = Hq // H
    qg = q.double().view(H, G, 128)
    s = torch.einsum("hgd,thd->hgt", qg, K) * scale
    sizes = (torch.einsum("hgd,thd->hgt", qg.abs(), K.abs()) * scale).amax(-1)
    w = torch.softmax(s, -1)
    out = torch.einsum("hgt,thd->hgd", w, V)
    return (out.reshape(Hq, 128), torch.logsumexp(s, -1).reshape(Hq), sizes.reshape(Hq),
            torch.einsum("hgt,thd->hgd", w, V.abs()).reshape(Hq, 128))


def assert_attention(got, lse, want, want_lse, sizes, mean_abs, n, weight_rounding):
    """A score's 128 products are summed in 32 bits by the tensor core in eight steps: off by at most 2^-21 of the sum of absolute
    products (2^-24 a step, and as much again for what its adder cuts off, generously), the weights' exponential by 2^-22: relative
    error d = 2 (2^-21 size + 2^-22) of a weight against the sum of all.  Then each weight is rounded (weight_rounding), and the result
    (half a step of bf16, 2^-8).  The sums of n / 8 terms per lane, 2^-24 each."""
    d = 2 * (2.0 ** -21 * sizes + 2.0 ** -22) + 2.0 ** -24 * (n / 8 + 64)
    tol = 2.0 ** -8 * want.abs() + (weight_rounding + d[:, None]) * (1 + 2.0 ** -8) * mean_abs + 1e-38
    err = (got.double() - want).abs()
    assert torch.all(err <= tol), float((err - tol).max())
    if lse is not None:
        finite = torch.isfinite(want_lse)
        assert torch.equal(torch.isfinite(lse), finite) and torch.all(lse[~finite] == -math.inf)
        err = (lse.double() - want_lse).abs()[finite]
        assert torch.all(err <= (d + 2.0 ** -22 * want_lse.abs())[finite]), float(err.max())
