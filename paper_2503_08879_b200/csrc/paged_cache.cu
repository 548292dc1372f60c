// What fills a paged cache and what reduces it:
//   rope      rows of queries or keys rotated by their positions;
//   append    keys and values of new tokens into their pages, the keys rotated on the way, the tokens' queries beside;
//   compact   Step 3 on pages: the reduced cache from the kept positions.
// Every row is read once and written once, 16 bytes per access (8 where a row is stored in 8 bits).  Many rows are bound by HBM, those
// that enter an 8-bit cache nearly as much by the issue rate; few rows by latency.
#include "paged.cuh"

namespace sagekv {

// ---- rotary positions ------------------------------------------------------------------------------------------------
// Eight lanes hold a row of 128 dimensions, each two 16-byte pieces such that the lane has both members of its eight
// pairs: with the halves paired, pieces p and p + r/16 (r the dimensions that turn), with neighbours paired, pieces
// 2p and 2p + 1; either way lane p needs the angles of pairs 8p .. 8p + 7.  The lanes beyond r/16 carry the rest
// of the row.  A warp works on rows of ONE token, four at a time, so its four groups of eight lanes need the same sines and
// cosines: each takes two of the eight and they are exchanged by shuffles.
//
// The angle.  position * f passes 10^5 radians, of which 32 bits keep no fraction worth having.  The host gives
// f / (2 pi) as a 64-bit fraction of a revolution, so the integer product with the position, modulo 2^64, is the
// fraction of a revolution exactly (within position * 2^-65), for positions up to 2^31 of either sign; its upper 32 bits are
// taken, and since the quadrant is two of them, no reduction of the argument is needed for sine and cosine.

__device__ __forceinline__ int first_piece(const RopeArgs &r, int p) {
  const int turning = r.rotary_dim >> 4;
  if (p >= turning) return 2 * p;                              // the rest: pieces r/8 + 2(p - r/16), + 1
  return r.interleaved ? 2 * p : p;
}
__device__ __forceinline__ int second_piece(const RopeArgs &r, int p) {
  const int turning = r.rotary_dim >> 4;
  if (p >= turning || r.interleaved) return 2 * p + 1;
  return p + turning;
}

// two 32-bit numbers side by side, as the packed instructions take them
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float lo, float hi) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 unpack2(f32x2 x) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

struct Angles {
  f32x2 cs[4], sn[4], ns[4];   // cosines, sines and negated sines of a lane's eight pairs
};

// Sines and cosines of two angles, given in 2^-31 half revolutions.  The upper two bits (rounded) are the quadrant, the rest is at
// most an eighth of a revolution either way: there the Taylor series to the ninth and tenth power leave out less than 2e-9, and
// the rest's rounding to 24 bits moves the angle by less than 3e-8.
__device__ __forceinline__ void sines(int half0, int half1, float (&sn)[2], float (&cs)[2]) {
  const int q[2] = {(int)((uint32_t)half0 + 0x20000000u) >> 30, (int)((uint32_t)half1 + 0x20000000u) >> 30};
  const f32x2 pi = pack2(3.14159265f * 0x1p-31f, 3.14159265f * 0x1p-31f);
  const f32x2 x = mul2(pack2((float)(int)((uint32_t)half0 - ((uint32_t)q[0] << 30)), (float)(int)((uint32_t)half1 - ((uint32_t)q[1] << 30))), pi);
  const f32x2 z = mul2(x, x);
  auto both = [](float v) { return pack2(v, v); };
  f32x2 s = fma2(z, both(1.f / 362880.f), both(-1.f / 5040.f)), c = fma2(z, both(-1.f / 3628800.f), both(1.f / 40320.f));
  s = fma2(z, s, both(1.f / 120.f));
  c = fma2(z, c, both(-1.f / 720.f));
  s = fma2(z, s, both(-1.f / 6.f));
  c = fma2(z, c, both(1.f / 24.f));
  s = fma2(mul2(z, s), x, x);
  c = fma2(z, c, both(-0.5f));
  c = fma2(z, c, both(1.f));
  const float2 s2 = unpack2(s), c2 = unpack2(c);
  const float ss[2] = {s2.x, s2.y}, cc[2] = {c2.x, c2.y};
#pragma unroll
  for (int e = 0; e < 2; ++e) {                                // a quadrant on: (cos, sin) becomes (-sin, cos)
    const float a = q[e] & 1 ? cc[e] : ss[e], b = q[e] & 1 ? ss[e] : cc[e];
    sn[e] = __uint_as_float(__float_as_uint(a) ^ ((uint32_t)(q[e] & 2) << 30));
    cs[e] = __uint_as_float(__float_as_uint(b) ^ ((uint32_t)((q[e] + 1) & 2) << 30));
  }
}

// lane: p = lane & 7, group = lane >> 3; all lanes take part
__device__ __forceinline__ void angles_of(const uint64_t *turns, float amplitude, int position, int lane, Angles &a) {
  const int p = lane & 7, group = lane >> 3;
  float cs[2], sn[2];
  int half[2];                                                 // in 2^-31 half revolutions, signed
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const uint64_t revolutions = turns[8 * p + 2 * group + e] * (uint64_t)(int64_t)position;
    half[e] = (int)(uint32_t)((revolutions + 0x80000000ull) >> 32);
  }
  sines(half[0], half[1], sn, cs);
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    sn[e] *= amplitude;
    cs[e] *= amplitude;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float c[2], s[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      c[i] = __shfl_sync(0xffffffffu, cs[i], e * 8 + p);
      s[i] = __shfl_sync(0xffffffffu, sn[i], e * 8 + p);
    }
    a.cs[e] = pack2(c[0], c[1]);
    a.sn[e] = pack2(s[0], s[1]);
    a.ns[e] = pack2(-s[0], -s[1]);
  }
}

__device__ __forceinline__ f32x2 widen(uint32_t w) { return pack2(bf16_low(w), bf16_high(w)); }

// the sixteen values of a lane's two pieces (eight twos), rotated
__device__ __forceinline__ void rotate(const RopeArgs &r, const Angles &a, const uint4 &first, const uint4 &second, f32x2 (&y)[8]) {
  const uint32_t w[8] = {first.x, first.y, first.z, first.w, second.x, second.y, second.z, second.w};
  if (r.interleaved) {                                         // a word holds a pair
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float2 c2 = unpack2(a.cs[e >> 1]), s2 = unpack2(a.sn[e >> 1]);
      const float c = e & 1 ? c2.y : c2.x, s = e & 1 ? s2.y : s2.x, lo = bf16_low(w[e]), hi = bf16_high(w[e]);
      y[e] = pack2(lo * c - hi * s, hi * c + lo * s);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x2 lo = widen(w[e]), hi = widen(w[4 + e]);
      y[e] = fma2(hi, a.ns[e], mul2(lo, a.cs[e]));
      y[4 + e] = fma2(lo, a.sn[e], mul2(hi, a.cs[e]));
    }
  }
}

__device__ __forceinline__ uint4 pack8_bf16(const f32x2 *y) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = unpack2(y[i]);
    w[i] = pack_bf16x2(v.x, v.y);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// The reciprocal of a scale in two parts: one a little below it (by 2^-22, more than the approximation is off), and what that leaves,
// which is therefore positive (an infinite value times both is infinite, and no NaN): a product with both has one
// rounding, as a division would.
struct Reciprocal {
  f32x2 high, low;
  __device__ __forceinline__ explicit Reciprocal(float scale) {
    float h;
    asm("rcp.approx.f32 %0, %1;" : "=f"(h) : "f"(scale));
    h *= 1.f - 0x1p-22f;
    const float l = fmaf(-h, scale, 1.f) * h;
    high = pack2(h, h);
    low = pack2(l, l);
  }
};
__device__ __forceinline__ uint2 pack8_e4m3(const f32x2 *y, const Reciprocal &inv) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = unpack2(fma2(y[i], inv.high, mul2(y[i], inv.low)));
    w[i] = pack_e4m3x2(v.x, v.y);
  }
  return make_uint2(__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410));
}

constexpr int kTurnWarps = 4;
constexpr int kTurnQuads = 2;       // groups of four rows whose loads are in flight at once
constexpr int kTurnCtasPerSm = 7;
constexpr int kTurnWaves = 4;       // waves of blocks that are left to even out
enum { kTurnOnly = 0, kTurnAppend = 1, kTurnAppendE4m3 = 2 };

// A warp takes rows of one kind (queries, keys or values; all of a token's, or some groups of four of them: blockIdx.y says which) of
// one token after another.  The rows are on their way while position and page are looked up.
// Bound by HBM where there are many tokens of bf16 (in a graph 65536 x 8 KV heads 85.4 us, floor 81.8; 20011 x 28 heads rotated alone 46.5 of 43.7),
// close to the issue rate into an 8-bit cache (73.1 us of 61.4: conversions and the angles against half the bytes), by latency where
// there are few (one token 2 us).  What it took (us, 65536 tokens x 8 KV heads, bf16 / 8-bit): a warp for all rows of a token
// 122.7 / 124.7 (1080 instructions a token); loads and angles shared out leaner, a kind per warp 100.7 / 98.6; frequencies
// through shared memory 90.3 / 84.1; sines from the quadrant, packed instructions 88.3 / 80.4; from token to token in 72 registers
// 85.3 / 73.0 (in 64, with spills: 90.4 / 83.4).  Rows through a ring of asynchronous copies instead: 106 / 119.
template <int kMode>
__global__ void __launch_bounds__(kTurnWarps * 32, kTurnCtasPerSm)
turn_rows_kernel(const __grid_constant__ PagedAppendParams p, const int per_warp, const int q_parts, const int kv_parts) {
  const int lane = threadIdx.x & 31, piece = lane & 7, group = lane >> 3;
  const int part = blockIdx.y;
  const int kind = kMode == kTurnOnly || part < q_parts ? 0 : part < q_parts + kv_parts ? 1 : 2;   // a query, a key, a value
  const int first = (part - (kind == 0 ? 0 : kind == 1 ? q_parts : q_parts + kv_parts)) * per_warp * 4 + group;   // my first head
  const int heads = kind == 0 ? p.H_q : p.H_kv, end = min(heads, first - group + per_warp * 4);
  const int pa = first_piece(p.rope, piece) * 8, pab = second_piece(p.rope, piece) * 8 - pa;
  const bool as_is = kind == 2 || piece >= (p.rope.rotary_dim >> 4);   // none of this lane's pairs turns
  // the frequencies through shared memory: lanes that ask the constant bank for 32 different words are served one by one
  // (65536 tokens x 8 KV heads into an 8-bit cache 98.6 -> 84.1 us)
  __shared__ uint64_t turns[kHeadDim / 2];
  if (kind != 2 && threadIdx.x < kHeadDim / 2) turns[threadIdx.x] = p.rope.turns[threadIdx.x];
  __syncthreads();
  wait_for_predecessor();
  const int64_t from_step = 4 * (kind == 0 ? p.q_head : p.kv_head), from_token = kind == 0 ? p.q_token : p.kv_token;
  const uint16_t *from = (kind == 0 ? p.q + first * p.q_head : (kind == 1 ? p.k : p.v) + first * p.kv_head) + pa;
  const int64_t stride = (int64_t)gridDim.x * kTurnWarps;
  int64_t t = (int64_t)blockIdx.x * kTurnWarps + (threadIdx.x >> 5);
  auto sequence_of = [&](int64_t token) { return kMode != kTurnOnly && kind != 0 && p.seqs != nullptr ? p.seqs[token] : (int)token; };
  int next_position = t < p.n_tokens ? p.positions[t] : -1, next_seq = t < p.n_tokens ? sequence_of(t) : -1;
  for (; t < p.n_tokens; t += stride) {
    const uint16_t *x = from + t * from_token;
    auto in_row = [&](int h) {                                 // checked build: a token's row, and this lane's pieces inside it
      return SAGEKV_OK_INDEX(p.c.status, t < p.n_tokens && h < heads && pa >= 0 && pa + 8 <= kHeadDim && pa + pab >= 0 && pa + pab + 8 <= kHeadDim);
    };
    uint4 xa[kTurnQuads], xb[kTurnQuads];
    auto load = [&](int h) {
#pragma unroll
      for (int u = 0; u < kTurnQuads; ++u)
        if (h + 4 * u < end && in_row(h + 4 * u)) {
          xa[u] = ld_v4(x);
          xb[u] = ld_v4(x + pab);
          x += from_step;
        }
    };
    load(first);
    const int position = next_position, seq = next_seq;
    if (t + stride < p.n_tokens) {
      next_position = p.positions[t + stride];
      next_seq = sequence_of(t + stride);
    }
    if (kMode != kTurnOnly && position < 0) continue;          // a place without a token
    int64_t row = -1;                                          // where any of position, sequence and page id is out of range: none
    if (kMode != kTurnOnly && kind != 0 && seq >= 0 && seq < p.c.n_seqs && position < p.c.max_pages * p.c.page_size) {
      const int entry = page_of(position, p.c.page_size, p.c.page_magic);
      const int slot = position - entry * p.c.page_size;
      if (SAGEKV_OK_ENTRY(p.c, seq, entry) && SAGEKV_OK_INDEX(p.c.status, slot >= 0 && slot < p.c.page_size))
        row = paged_row(p.c.table[seq * p.c.table_stride + entry], p.c.n_pages, slot, first, p.c.page_stride, p.c.head_stride, p.c.token_stride);
    }
    Angles a;
    if (kind != 2 && p.rope.rotary_dim > 0) angles_of(turns, p.rope.amplitude, position, lane, a);
    if (kMode != kTurnOnly && kind != 0 && row < 0) {
      if (lane == 0) atomicOr(p.c.status, kStatusBounds);
      continue;
    }
    if (kMode == kTurnAppendE4m3 && kind != 0) {
      uint8_t *o = (kind == 1 ? p.c.k : p.c.v) + row + pa;
      const float *scales = kind == 1 ? p.c.k_scale : p.c.v_scale;
      for (int h = first; h < end; h += 4 * kTurnQuads) {
        if (h > first) load(h);
#pragma unroll
        for (int u = 0; u < kTurnQuads; ++u) {
          if (h + 4 * u >= end || !in_row(h + 4 * u)) continue;
          f32x2 y[8];
          if (!as_is) {
            rotate(p.rope, a, xa[u], xb[u], y);
          } else {
            const uint32_t w[8] = {xa[u].x, xa[u].y, xa[u].z, xa[u].w, xb[u].x, xb[u].y, xb[u].z, xb[u].w};
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = widen(w[i]);
          }
          const Reciprocal inv(scales != nullptr ? scales[h + 4 * u] : 1.f);
          *reinterpret_cast<uint2 *>(o) = pack8_e4m3(y, inv);
          *reinterpret_cast<uint2 *>(o + pab) = pack8_e4m3(y + 4, inv);
          o += 4 * p.c.head_stride;
        }
      }
    } else {
      uint16_t *o = kMode == kTurnOnly || kind == 0 ? p.q_out + t * p.q_out_token + first * p.q_out_head + pa
                                                    : reinterpret_cast<uint16_t *>(kind == 1 ? p.c.k : p.c.v) + row + pa;
      const int64_t o_step = 4 * (kMode == kTurnOnly || kind == 0 ? p.q_out_head : p.c.head_stride);
      for (int h = first; h < end; h += 4 * kTurnQuads) {
        if (h > first) load(h);
#pragma unroll
        for (int u = 0; u < kTurnQuads; ++u) {
          if (h + 4 * u >= end || !in_row(h + 4 * u)) continue;
          if (as_is) {
            st_v4(o, xa[u]);
            st_v4(o + pab, xb[u]);
          } else {
            f32x2 y[8];
            rotate(p.rope, a, xa[u], xb[u], y);
            st_v4(o, pack8_bf16(y));
            st_v4(o + pab, pack8_bf16(y + 4));
          }
          o += o_step;
        }
      }
    }
  }
}

// One group of four rows per warp where there are few (latency), up to all of a token's of a kind where those fill the device: they
// share the angles.
template <int kMode>
static cudaError_t launch_turn(const PagedAppendParams &p, int n_sm, cudaStream_t stream) {
  if (p.n_tokens <= 0) return cudaSuccess;
  const int q_quads = kMode == kTurnOnly || p.q != nullptr ? (p.H_q + 3) / 4 : 0, kv_quads = kMode == kTurnOnly ? 0 : (p.H_kv + 3) / 4;
  const int64_t warps = (int64_t)n_sm * kTurnWarps * kTurnCtasPerSm;   // that run at once
  const int64_t share = p.n_tokens * (q_quads + 2 * kv_quads) / warps;
  const int per_warp = (int)(share < 1 ? 1 : share > kTurnMostQuads ? kTurnMostQuads : share);
  // (at most 65535 parts: a launch of fewer than kTurnMostQuads a warp has fewer groups than that, and the API bounds the heads of the others)
  const int q_parts = (q_quads + per_warp - 1) / per_warp, kv_parts = (kv_quads + per_warp - 1) / per_warp, parts = q_parts + 2 * kv_parts;
  const int64_t rounds = p.n_tokens * parts / (kTurnWaves * warps);    // tokens of a warp, if kTurnWaves waves of blocks are to remain
  const int64_t tokens = (p.n_tokens + (rounds > 1 ? rounds : 1) - 1) / (rounds > 1 ? rounds : 1);
  return launch_next(turn_rows_kernel<kMode>, dim3((unsigned)((tokens + kTurnWarps - 1) / kTurnWarps), (unsigned)parts), kTurnWarps * 32, 0,
                     stream, 0, p, per_warp, q_parts, kv_parts);
}

cudaError_t launch_rope(const PagedAppendParams &p, int n_sm, cudaStream_t stream) {
  if (p.H_q <= 0) return cudaSuccess;
  return launch_turn<kTurnOnly>(p, n_sm, stream);
}

cudaError_t launch_paged_append(const PagedAppendParams &p, int dtype, int n_sm, cudaStream_t stream) {
  return dtype == SAGEKV_CACHE_E4M3 ? launch_turn<kTurnAppendE4m3>(p, n_sm, stream) : launch_turn<kTurnAppend>(p, n_sm, stream);
}

// ---- compact ---------------------------------------------------------------------------------------------------------
// Rows as in sagekv_select_compact: sink, the G lists, recent tokens, last token.  A warp takes up to 32 rows of one KV head:
// each lane finds one row's place (list, then table: two loads one behind the other, for all rows at once), then the
// rows are moved kRows at a time, 16 bytes per lane, all loads ahead of the stores.  An 8-bit row is widened: code * scale,
// rounded to bf16.  Bound by that chain of loads where the rows are few, by their scatter where they are many.  (us, 8 heads x 2049 bf16
// rows / 16 x 8193 bf16 / 16 x 8193 8-bit in a graph, the first with its rows in L2; bytes at the copy rate 2.6 / 20.5 / 15.4: eight rows at once in blocks of eight warps, loads past L1
// 5.25 / 35.9 / 24.9, four in blocks of four 4.1 / 25.1 / 25.6, plain loads besides 3.5 / 24.0 / 25.5; 8-bit eight at once and 32 per
// warp 23.3, with stores of whole sectors 20.4, 16 per warp 19.1; bf16 now 3.4 / 23.7.  The first out of HBM, layer after layer: 5.8)
constexpr int kCompactWarps = 4;

template <bool kE4m3, int kRows>
__global__ void __launch_bounds__(kCompactWarps * 32) paged_compact_kernel(const PagedCompactParams p, const int rows_per_warp) {
  constexpr int kLanes = kE4m3 ? 8 : 16;                       // of a row of K or of V
  constexpr int kAtOnce = 32 / (2 * kLanes);                   // rows of K and V that a load instruction covers
  constexpr int kLoads = kRows / kAtOnce;
  const int lane = threadIdx.x & 31, piece = lane & (kLanes - 1);
  const bool is_v = (lane / kLanes) & 1;
  const int sub = lane / (2 * kLanes);                         // which of the rows of a load
  wait_for_predecessor();
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.d_step = 0;
  const int n_sel = p.G * p.k_q, L = p.S + n_sel + p.R + 1;
  const int bk = blockIdx.y, b = bk / p.H_kv, kvh = bk - b * p.H_kv;
  const int first = (int)(blockIdx.x * kCompactWarps + (threadIdx.x >> 5)) * rows_per_warp, n = min(rows_per_warp, L - first);
  if (n <= 0) return;
  int64_t src = -1;                                            // lane i: the place of row first + i, -1: there is none
  if (lane < n) {
    const int r = first + lane;
    int tok = r < p.S ? r : p.N - L + r;
    if (r >= p.S && r < p.S + n_sel) {                         // the lists of a KV head's query heads lie one behind the other, as its segments do
      const int off = SAGEKV_OK_INDEX(p.c.status, bk < p.B * p.H_kv) ? p.idx[(int64_t)bk * n_sel + (r - p.S)] : -1;
      tok = off >= 0 && off < p.E ? p.S + off : -1;
    }
    if (tok >= 0) {
      const int entry = page_of(tok, p.c.page_size, p.c.page_magic);
      const int slot = tok - entry * p.c.page_size;
      if (SAGEKV_OK_ENTRY(p.c, b, entry) && SAGEKV_OK_INDEX(p.c.status, slot >= 0 && slot < p.c.page_size && kvh < p.H_kv))
        src = paged_row(p.c.table[(int64_t)b * p.c.table_stride + entry], p.c.n_pages, slot, kvh, p.c.page_stride, p.c.head_stride, p.c.token_stride);
    }
    if (src < 0) atomicOr(p.c.status, kStatusBounds);          // a position or a page id out of range: the row is left as it was
  }
  const uint8_t *pages = is_v ? p.c.v : p.c.k;
  const float *scales = is_v ? p.c.v_scale : p.c.k_scale;
  const float scale = kE4m3 && scales != nullptr ? scales[kvh] : 1.f;
  uint16_t *dst = (is_v ? p.Vc : p.Kc) + (int64_t)b * p.cs.batch_stride + (int64_t)kvh * p.cs.head_stride + (int64_t)first * p.cs.token_stride +
                  piece * (128 / kLanes);
  for (int i0 = 0; i0 < n; i0 += kRows) {
    uint4 row[kLoads];
    bool there[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      row[u] = make_uint4(0u, 0u, 0u, 0u);
      const int i = i0 + u * kAtOnce + sub;
      const int64_t at = __shfl_sync(0xffffffffu, src, i & 31);
      there[u] = i < n && at >= 0 && SAGEKV_OK_INDEX(p.c.status, first + i < L && b < p.B);
      if (there[u]) row[u] = ld_v4(pages + at * (kE4m3 ? 1 : 2) + piece * 16);
    }
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      uint16_t *o = dst + (int64_t)(i0 + u * kAtOnce + sub) * p.cs.token_stride;
      if (kE4m3) {
        const uint32_t w[4] = {row[u].x, row[u].y, row[u].z, row[u].w};
        uint32_t y[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 x0 = float2_of_f16x2(f16x2_low(w[i])), x1 = float2_of_f16x2(f16x2_high(w[i]));
          y[2 * i] = pack_bf16x2(x0.x * scale, x0.y * scale);
          y[2 * i + 1] = pack_bf16x2(x1.x * scale, x1.y * scale);
        }
        // two neighbours swap halves, so that each store writes whole sectors: first the even lane's 32 bytes, then the odd lane's
        const bool odd = lane & 1;
        uint4 mine = odd ? make_uint4(y[4], y[5], y[6], y[7]) : make_uint4(y[0], y[1], y[2], y[3]);
        uint4 other = odd ? make_uint4(y[0], y[1], y[2], y[3]) : make_uint4(y[4], y[5], y[6], y[7]);
        other.x = __shfl_xor_sync(0xffffffffu, other.x, 1);
        other.y = __shfl_xor_sync(0xffffffffu, other.y, 1);
        other.z = __shfl_xor_sync(0xffffffffu, other.z, 1);
        other.w = __shfl_xor_sync(0xffffffffu, other.w, 1);
        if (!there[u]) continue;                               // (the same for both)
        st_v4(odd ? o - 8 : o, odd ? other : mine);
        st_v4(odd ? o + 8 : o + 16, odd ? mine : other);
      } else if (there[u]) {
        st_v4(o, row[u]);
      }
    }
  }
}

cudaError_t launch_paged_compact(const PagedCompactParams &p, int dtype, int n_sm, cudaStream_t stream) {
  const int64_t L = p.S + (int64_t)p.G * p.k_q + p.R + 1, heads = (int64_t)p.B * p.H_kv;
  // four rows per warp, of a long 8-bit launch up to sixteen, as long as that leaves every SM two dozen warps
  const bool e4m3 = dtype == SAGEKV_CACHE_E4M3;
  int rows = 4;
  while (e4m3 && rows < 16 && L * heads / (2 * rows) >= (int64_t)n_sm * 24) rows *= 2;
  const int64_t per_block = (int64_t)kCompactWarps * rows;
  const auto kernel = !e4m3 ? paged_compact_kernel<false, 4> : rows >= 8 ? paged_compact_kernel<true, 8> : paged_compact_kernel<true, 4>;
  return launch_next(kernel, dim3((unsigned)((L + per_block - 1) / per_block), (unsigned)heads), kCompactWarps * 32, 0, stream, 0, p, rows);
}

}  // namespace sagekv
