// What fills a paged cache and what reduces it:
//   rope      rows of queries or keys rotated by their positions;
//   append    keys and values of new tokens into their pages, the keys rotated on the way, the tokens' queries beside;
//   compact   Step 3 on pages: the reduced cache from the kept positions.
// All are bound by memory: every row is read once and written once, 16 bytes per access.
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
// fraction of a revolution exactly (within position * 2^-65), for positions up to 2^31 of either sign; its upper 32 bits go to
// sincospi in half revolutions.

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

struct Angles {
  float cs[8], sn[8];
};

// lane: p = lane & 7, group = lane >> 3; all lanes take part
__device__ __forceinline__ void angles_of(const RopeArgs &r, int position, int lane, Angles &a) {
  const int p = lane & 7, group = lane >> 3;
  float cs[2], sn[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const uint64_t revolutions = r.turns[8 * p + 2 * group + e] * (uint64_t)(int64_t)position;
    const int half = (int)(uint32_t)((revolutions + 0x80000000ull) >> 32);      // in 2^-31 half revolutions, signed
    sincospif((float)half * 0x1p-31f, &sn[e], &cs[e]);
    cs[e] *= r.amplitude;
    sn[e] *= r.amplitude;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    a.cs[e] = __shfl_sync(0xffffffffu, cs[e & 1], (e >> 1) * 8 + p);
    a.sn[e] = __shfl_sync(0xffffffffu, sn[e & 1], (e >> 1) * 8 + p);
  }
}

// the sixteen values of a lane's two pieces, rotated where the lane's pairs turn
__device__ __forceinline__ void rotate(const RopeArgs &r, const Angles &a, int p, uint4 first, uint4 second, float (&y)[16]) {
  const uint32_t w[8] = {first.x, first.y, first.z, first.w, second.x, second.y, second.z, second.w};
  float x[16];
#pragma unroll
  for (int i = 0; i < 8; ++i) { x[2 * i] = bf16_low(w[i]); x[2 * i + 1] = bf16_high(w[i]); }
  if (p < (r.rotary_dim >> 4)) {
    if (r.interleaved) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y[2 * e] = x[2 * e] * a.cs[e] - x[2 * e + 1] * a.sn[e];
        y[2 * e + 1] = x[2 * e + 1] * a.cs[e] + x[2 * e] * a.sn[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y[e] = x[e] * a.cs[e] - x[8 + e] * a.sn[e];
        y[8 + e] = x[8 + e] * a.cs[e] + x[e] * a.sn[e];
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = x[i];
  }
}

__device__ __forceinline__ uint4 pack8_bf16(const float *y) {
  return make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
}
__device__ __forceinline__ uint2 pack8_e4m3(const float *y, float inv_scale) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_e4m3x2(y[2 * i] * inv_scale, y[2 * i + 1] * inv_scale);
  return make_uint2(w[0] | (w[1] << 16), w[2] | (w[3] << 16));
}

constexpr int kRopeWarps = 8;
constexpr int kRopeQuads = 4;   // groups of four rows a warp loads before it stores any

// A warp takes `quads` groups of four heads of one token.
__global__ void __launch_bounds__(kRopeWarps * 32) rope_kernel(const __grid_constant__ RopeParams p, const int quads, const int warps_per_token) {
  const int lane = threadIdx.x & 31, piece = lane & 7, group = lane >> 3;
  const int64_t job = (int64_t)blockIdx.x * kRopeWarps + (threadIdx.x >> 5);
  wait_for_predecessor();
  const int64_t t = job / warps_per_token;
  if (t >= p.n_tokens) return;
  const int quad0 = (int)(job - t * warps_per_token) * quads, all_quads = (p.n_heads + 3) >> 2;
  const int pa = first_piece(p.rope, piece) * 8, pb = second_piece(p.rope, piece) * 8;
  const uint16_t *x = p.x + t * p.x_token;
  uint16_t *out = p.out + t * p.out_token;
  const int position = p.positions[t];
  Angles a;
  bool have = false;
  for (int q0 = quad0; q0 < min(quad0 + quads, all_quads); q0 += kRopeQuads) {
    uint4 xa[kRopeQuads], xb[kRopeQuads];
#pragma unroll
    for (int u = 0; u < kRopeQuads; ++u) {
      const int h = (q0 + u) * 4 + group;
      if (q0 + u < quad0 + quads && h < p.n_heads) {
        xa[u] = ld_v4(x + (int64_t)h * p.x_head + pa);
        xb[u] = ld_v4(x + (int64_t)h * p.x_head + pb);
      }
    }
    if (!have) { angles_of(p.rope, position, lane, a); have = true; }
#pragma unroll
    for (int u = 0; u < kRopeQuads; ++u) {
      const int h = (q0 + u) * 4 + group;
      if (q0 + u < quad0 + quads && h < p.n_heads) {
        float y[16];
        rotate(p.rope, a, piece, xa[u], xb[u], y);
        st_v4(out + (int64_t)h * p.out_head + pa, pack8_bf16(y));
        st_v4(out + (int64_t)h * p.out_head + pb, pack8_bf16(y + 8));
      }
    }
  }
}

// groups of four rows per warp: one where there are few (latency), up to all of a token's where the device is full
static int quads_per_warp(int64_t tokens, int quads, int n_sm) {
  int64_t n = tokens * quads / ((int64_t)n_sm * 32);
  return (int)(n < 1 ? 1 : n > quads ? quads : n);
}

cudaError_t launch_rope(const RopeParams &p, int n_sm, cudaStream_t stream) {
  if (p.n_tokens <= 0 || p.n_heads <= 0) return cudaSuccess;
  const int all = (p.n_heads + 3) / 4, quads = quads_per_warp(p.n_tokens, all, n_sm), warps = (all + quads - 1) / quads;
  const int64_t blocks = (p.n_tokens * warps + kRopeWarps - 1) / kRopeWarps;
  if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  return launch_next(rope_kernel, dim3((unsigned)blocks), kRopeWarps * 32, 0, stream, 0, p, quads, warps);
}

// ---- append ----------------------------------------------------------------------------------------------------------
// As rope, over the groups of four rows of a token's queries, keys and values in this order.
template <bool kE4m3>
__global__ void __launch_bounds__(kRopeWarps * 32) paged_append_kernel(const __grid_constant__ PagedAppendParams p, const int quads,
                                                                       const int warps_per_token) {
  const int lane = threadIdx.x & 31, piece = lane & 7, group = lane >> 3;
  const int64_t job = (int64_t)blockIdx.x * kRopeWarps + (threadIdx.x >> 5);
  wait_for_predecessor();
  const int64_t t = job / warps_per_token;
  if (t >= p.n_tokens) return;
  const int q_quads = p.q != nullptr ? (p.H_q + 3) >> 2 : 0, kv_quads = (p.H_kv + 3) >> 2, all_quads = q_quads + 2 * kv_quads;
  const int quad0 = (int)(job - t * warps_per_token) * quads;
  const int pa = first_piece(p.rope, piece) * 8, pb = second_piece(p.rope, piece) * 8;
  const int position = p.positions[t];
  const int64_t seq = p.seqs != nullptr ? (int64_t)p.seqs[t] : t;
  uint4 xa[kRopeQuads], xb[kRopeQuads];
  int head[kRopeQuads], kind[kRopeQuads];                      // kind 0: a query, 1: a key, 2: a value; head -1: nothing
  float scale[kRopeQuads];
  auto load = [&](int q0) {
#pragma unroll
    for (int u = 0; u < kRopeQuads; ++u) {
      const int quad = q0 + u;
      kind[u] = quad < q_quads ? 0 : quad < q_quads + kv_quads ? 1 : 2;
      head[u] = (quad - (kind[u] == 0 ? 0 : q_quads + (kind[u] - 1) * kv_quads)) * 4 + group;
      if (quad >= min(quad0 + quads, all_quads) || head[u] >= (kind[u] == 0 ? p.H_q : p.H_kv)) head[u] = -1;
      scale[u] = 1.f;
      if (head[u] >= 0) {
        const uint16_t *x = kind[u] == 0 ? p.q + t * p.q_token + (int64_t)head[u] * p.q_head
                                         : (kind[u] == 1 ? p.k : p.v) + t * p.kv_token + (int64_t)head[u] * p.kv_head;
        xa[u] = ld_v4(x + pa);
        xb[u] = ld_v4(x + pb);
        if (kE4m3 && kind[u] != 0) {
          const float *scales = kind[u] == 1 ? p.c.k_scale : p.c.v_scale;
          if (scales != nullptr) scale[u] = scales[head[u]];
        }
      }
    }
  };
  load(quad0);                                                 // on their way while the page is looked up
  if (position < 0) return;                                    // a place without a token
  // the token's page: where any of position, sequence and page id is out of range its rows have no place
  int page = -1, slot = 0;
  bool in_table = seq >= 0 && seq < p.c.n_seqs && position < p.c.max_pages * p.c.page_size;
  if (in_table) {
    const int entry = page_of(position, p.c.page_size, p.c.page_magic);
    slot = position - entry * p.c.page_size;
    page = p.c.table[seq * p.c.table_stride + entry];
  }
  Angles a;
  if (p.rope.rotary_dim > 0 && quad0 < q_quads + kv_quads) angles_of(p.rope, position, lane, a);
  const int64_t row = paged_row(page, p.c.n_pages, slot, 0, p.c.page_stride, 0, p.c.token_stride);
  if (row < 0 && lane == 0) atomicOr(p.c.status, kStatusBounds);
  for (int q0 = quad0; q0 < min(quad0 + quads, all_quads); q0 += kRopeQuads) {
    if (q0 > quad0) load(q0);
#pragma unroll
    for (int u = 0; u < kRopeQuads; ++u) {
      if (head[u] < 0 || (kind[u] != 0 && row < 0)) continue;
      float y[16];
      const bool as_is = kind[u] == 2 || p.rope.rotary_dim == 0;
      if (!as_is) rotate(p.rope, a, piece, xa[u], xb[u], y);
      if (kind[u] == 0) {
        uint16_t *o = p.q_out + t * p.q_out_token + (int64_t)head[u] * p.q_out_head;
        st_v4(o + pa, as_is ? xa[u] : pack8_bf16(y));
        st_v4(o + pb, as_is ? xb[u] : pack8_bf16(y + 8));
        continue;
      }
      uint8_t *pages = kind[u] == 1 ? p.c.k : p.c.v;
      const int64_t at = row + (int64_t)head[u] * p.c.head_stride;
      if (kE4m3) {
        if (as_is) {
          const uint32_t w[8] = {xa[u].x, xa[u].y, xa[u].z, xa[u].w, xb[u].x, xb[u].y, xb[u].z, xb[u].w};
#pragma unroll
          for (int i = 0; i < 8; ++i) { y[2 * i] = bf16_low(w[i]); y[2 * i + 1] = bf16_high(w[i]); }
        }
        const float inv = 1.f / scale[u];
        *reinterpret_cast<uint2 *>(pages + at + pa) = pack8_e4m3(y, inv);
        *reinterpret_cast<uint2 *>(pages + at + pb) = pack8_e4m3(y + 8, inv);
      } else {
        uint16_t *o = reinterpret_cast<uint16_t *>(pages) + at;
        st_v4(o + pa, as_is ? xa[u] : pack8_bf16(y));
        st_v4(o + pb, as_is ? xb[u] : pack8_bf16(y + 8));
      }
    }
  }
}

cudaError_t launch_paged_append(const PagedAppendParams &p, int dtype, int n_sm, cudaStream_t stream) {
  if (p.n_tokens <= 0) return cudaSuccess;
  const int all = (p.q != nullptr ? (p.H_q + 3) / 4 : 0) + 2 * ((p.H_kv + 3) / 4);
  const int quads = quads_per_warp(p.n_tokens, all, n_sm), warps = (all + quads - 1) / quads;
  const int64_t blocks = (p.n_tokens * warps + kRopeWarps - 1) / kRopeWarps;
  if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  return launch_next(dtype == SAGEKV_CACHE_E4M3 ? paged_append_kernel<true> : paged_append_kernel<false>, dim3((unsigned)blocks),
                     kRopeWarps * 32, 0, stream, 0, p, quads, warps);
}

// ---- compact ---------------------------------------------------------------------------------------------------------
// Rows as in sagekv_select_compact: sink, the G lists, recent tokens, last token.  A warp takes up to 32 rows of one KV head:
// each lane finds one row's place (list, then table: two loads one behind the other, for all rows at once), then the
// rows are moved kCompactRows at a time, 16 bytes per lane, all loads ahead of the stores.  An 8-bit row is widened: code * scale,
// rounded to bf16.
constexpr int kCompactWarps = 8;
constexpr int kCompactRows = 8;

template <bool kE4m3>
__global__ void __launch_bounds__(kCompactWarps * 32) paged_compact_kernel(const PagedCompactParams p, const int rows_per_warp) {
  constexpr int kLanes = kE4m3 ? 8 : 16;                       // of a row of K or of V
  constexpr int kAtOnce = 32 / (2 * kLanes);                   // rows of K and V that a load instruction covers
  constexpr int kLoads = kCompactRows / kAtOnce;
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
      const int off = p.idx[(int64_t)bk * n_sel + (r - p.S)];
      tok = off >= 0 && off < p.E ? p.S + off : -1;
    }
    if (tok >= 0) {
      const int entry = page_of(tok, p.c.page_size, p.c.page_magic);
      src = paged_row(p.c.table[(int64_t)b * p.c.table_stride + entry], p.c.n_pages, tok - entry * p.c.page_size, kvh, p.c.page_stride,
                      p.c.head_stride, p.c.token_stride);
    }
    if (src < 0) atomicOr(p.c.status, kStatusBounds);          // a position or a page id out of range: the row is left as it was
  }
  const uint8_t *pages = is_v ? p.c.v : p.c.k;
  const float *scales = is_v ? p.c.v_scale : p.c.k_scale;
  const float scale = kE4m3 && scales != nullptr ? scales[kvh] : 1.f;
  uint16_t *dst = (is_v ? p.Vc : p.Kc) + (int64_t)b * p.cs.batch_stride + (int64_t)kvh * p.cs.head_stride + (int64_t)first * p.cs.token_stride +
                  piece * (128 / kLanes);
  for (int i0 = 0; i0 < n; i0 += kCompactRows) {
    uint4 row[kLoads];
    bool there[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int i = i0 + u * kAtOnce + sub;
      const int64_t at = __shfl_sync(0xffffffffu, src, i & 31);
      there[u] = i < n && at >= 0;
      if (there[u]) row[u] = ld_stream_v4(pages + at * (kE4m3 ? 1 : 2) + piece * 16);
    }
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      if (!there[u]) continue;
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
        st_v4(o, make_uint4(y[0], y[1], y[2], y[3]));
        st_v4(o + 8, make_uint4(y[4], y[5], y[6], y[7]));
      } else {
        st_v4(o, row[u]);
      }
    }
  }
}

cudaError_t launch_paged_compact(const PagedCompactParams &p, int dtype, int n_sm, cudaStream_t stream) {
  const int64_t L = p.S + (int64_t)p.G * p.k_q + p.R + 1, heads = (int64_t)p.B * p.H_kv;
  // as many rows per warp as leave every SM a dozen warps
  int rows = kCompactRows;
  while (rows < 32 && L * heads / (2 * rows) >= (int64_t)n_sm * 12) rows *= 2;
  const int64_t per_block = (int64_t)kCompactWarps * rows;
  return launch_next(dtype == SAGEKV_CACHE_E4M3 ? paged_compact_kernel<true> : paged_compact_kernel<false>,
                     dim3((unsigned)((L + per_block - 1) / per_block), (unsigned)heads), kCompactWarps * 32, 0, stream, 0, p, rows);
}

}  // namespace sagekv
