// What fills a paged cache and what reduces it:
//   rope      rows of queries or keys rotated by their positions;
//   append    keys and values of new tokens into their pages, the keys rotated on the way, the tokens' queries beside;
//   score     Step 2 of the method (first half) on pages: sagekv_score with a table between a token and its row;
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
  if (position < 0) return;                                    // a place without a token
  // the token's page: where any of position, sequence and page id is out of range its rows have no place
  const int64_t seq = p.seqs != nullptr ? (int64_t)p.seqs[t] : t;
  int64_t row = -1;
  if (seq >= 0 && seq < p.c.n_seqs && position < p.c.max_pages * p.c.page_size) {
    const int entry = page_of(position, p.c.page_size, p.c.page_magic);
    row = paged_row(p.c.table[seq * p.c.table_stride + entry], p.c.n_pages, position - entry * p.c.page_size, 0, p.c.page_stride, 0,
                    p.c.token_stride);
  }
  if (row < 0 && lane == 0) atomicOr(p.c.status, kStatusBounds);
  Angles a;
  bool have = false;
  for (int q0 = quad0; q0 < min(quad0 + quads, all_quads); q0 += kRopeQuads) {
    uint4 xa[kRopeQuads], xb[kRopeQuads];
    int head[kRopeQuads], kind[kRopeQuads];                    // kind 0: a query, 1: a key, 2: a value; head -1: nothing
#pragma unroll
    for (int u = 0; u < kRopeQuads; ++u) {
      const int quad = q0 + u;
      kind[u] = quad < q_quads ? 0 : quad < q_quads + kv_quads ? 1 : 2;
      head[u] = (quad - (kind[u] == 0 ? 0 : q_quads + (kind[u] - 1) * kv_quads)) * 4 + group;
      if (quad >= min(quad0 + quads, all_quads) || head[u] >= (kind[u] == 0 ? p.H_q : p.H_kv)) head[u] = -1;
      if (head[u] >= 0) {
        const uint16_t *x = kind[u] == 0 ? p.q + t * p.q_token + (int64_t)head[u] * p.q_head
                                         : (kind[u] == 1 ? p.k : p.v) + t * p.kv_token + (int64_t)head[u] * p.kv_head;
        xa[u] = ld_v4(x + pa);
        xb[u] = ld_v4(x + pb);
      }
    }
    if (!have && p.rope.rotary_dim > 0 && q0 < q_quads + kv_quads) { angles_of(p.rope, position, lane, a); have = true; }
#pragma unroll
    for (int u = 0; u < kRopeQuads; ++u) {
      if (head[u] < 0 || (kind[u] != 0 && row < 0)) continue;
      float y[16];
      const bool as_is = kind[u] == 2 || p.rope.rotary_dim == 0;
      if (as_is && kind[u] == 0) {
        uint16_t *o = p.q_out + t * p.q_out_token + (int64_t)head[u] * p.q_out_head;
        st_v4(o + pa, xa[u]);
        st_v4(o + pb, xb[u]);
        continue;
      }
      if (!as_is) {
        rotate(p.rope, a, piece, xa[u], xb[u], y);
        if (kind[u] == 0) {
          uint16_t *o = p.q_out + t * p.q_out_token + (int64_t)head[u] * p.q_out_head;
          st_v4(o + pa, pack8_bf16(y));
          st_v4(o + pb, pack8_bf16(y + 8));
          continue;
        }
      }
      uint8_t *pages = kind[u] == 1 ? p.c.k : p.c.v;
      const int64_t at = row + (int64_t)head[u] * p.c.head_stride;
      if (kE4m3) {
        const float *scale = kind[u] == 1 ? p.c.k_scale : p.c.v_scale;
        const float inv = scale != nullptr ? 1.f / scale[head[u]] : 1.f;
        if (as_is) {
          const uint32_t w[8] = {xa[u].x, xa[u].y, xa[u].z, xa[u].w, xb[u].x, xb[u].y, xb[u].z, xb[u].w};
#pragma unroll
          for (int i = 0; i < 8; ++i) { y[2 * i] = bf16_low(w[i]); y[2 * i + 1] = bf16_high(w[i]); }
        }
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

// ---- score -----------------------------------------------------------------------------------------------------------
// The first pass of the score step (see score.cu: a warp's tiles go from global memory straight into matrix fragments,
// all loads in flight), with every lane looking up the pages of its own two rows per tile.  An 8-bit row is half as
// long, so a warp takes twice as many tiles: the bytes in flight are what the memory's latency needs.  Writes the scaled logits and
// a (max, sum) pair per CTA and head; the second pass is the score step's own.
template <bool kE4m3>
__global__ void __launch_bounds__(kScoreWarps * 32, 2) paged_score_kernel(const ScoreParams p, const PagedView c) {
  constexpr int kTiles = kE4m3 ? 2 * kScoreTiles : kScoreTiles;
  constexpr int kPieces = kE4m3 ? 2 : 4;                       // 16-byte pieces of a row that a lane holds
  const int chunk = blockIdx.x, kvh = blockIdx.y, b = blockIdx.z;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, cc = lane & 3;
  wait_for_predecessor();
  if (chunk == 0 && p.sketch_off >= 0) {                       // the rows' histograms are filled by atomic adds in the second pass
    for (int i = threadIdx.x; i < p.G * (kSketchBins + 4); i += kScoreWarps * 32) {
      const int h = i / (kSketchBins + 4);
      reinterpret_cast<uint32_t *>(p.scores + ((int64_t)b * p.H_q + kvh * p.G + h) * p.row_stride + p.sketch_off)[i - h * (kSketchBins + 4)] = 0u;
    }
  }

  const int tok_base = (chunk * kScoreWarps + warp) * 16 * kTiles;
  const int last = p.E - 1;
  const int32_t *table = c.table + (int64_t)b * c.table_stride;
  const uint8_t *head = c.k + (int64_t)kvh * c.head_stride * (kE4m3 ? 1 : 2);
  int ids[kTiles][2];
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int e = 0; e < 2; ++e) ids[t][e] = table[page_of(p.S + min(tok_base + t * 16 + g + 8 * e, last), c.page_size, c.page_magic)];
  uint4 k[kTiles][2][kPieces];
  uint32_t absent = 0u;                                        // bit 2t + e: no such page
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int tok = p.S + min(tok_base + t * 16 + g + 8 * e, last);
      const int64_t row = paged_row(ids[t][e], c.n_pages, tok - page_of(tok, c.page_size, c.page_magic) * c.page_size, 0, c.page_stride, 0, c.token_stride);
      if (row < 0) absent |= 1u << (2 * t + e);
      const uint8_t *src = head + row * (kE4m3 ? 1 : 2) + cc * 16;
#pragma unroll
      for (int j = 0; j < kPieces; ++j) k[t][e][j] = row >= 0 ? ld_stream_v4(src + j * 64) : make_uint4(0u, 0u, 0u, 0u);
    }
  if (absent != 0u) atomicOr(c.status, kStatusBounds);

  // B fragments: query head (kvh*G + g) for n = g, zero padding for n >= G; the dims as the pieces hold them
  uint32_t qf[8][2];
  const int h0 = 2 * cc, h1 = 2 * cc + 1;
  float mult0 = p.scale_log2, mult1 = p.scale_log2;
  {
    const uint16_t *qrow = p.q + ((int64_t)b * p.H_q + kvh * p.G + min(g, p.G - 1)) * kHeadDim;
    float largest = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      // bf16: piece j of a row holds dims 32j + 8cc .. + 7; 8-bit: piece j / 2 holds 64(j / 2) + 16cc .. + 15, eight of them here
      uint4 v = make_uint4(0u, 0u, 0u, 0u);
      if (g < p.G) v = ld_v4(qrow + (kE4m3 ? (j >> 1) * 64 + cc * 16 + (j & 1) * 8 : j * 32 + cc * 8));
      qf[2 * j][0] = v.x; qf[2 * j][1] = v.y; qf[2 * j + 1][0] = v.z; qf[2 * j + 1][1] = v.w;
    }
    if (kE4m3) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) largest = fmaxf(largest, fmaxf(fabsf(bf16_low(qf[j][e])), fabsf(bf16_high(qf[j][e]))));
      largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, 1));
      largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, 2));
      const int ex = query_exponent(largest);
      const float up = power_of_two(ex);
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) qf[j][e] = pack_f16x2(bf16_low(qf[j][e]) * up, bf16_high(qf[j][e]) * up);
      const float base = c.k_scale != nullptr ? p.scale_log2 * c.k_scale[kvh] : p.scale_log2;
      mult0 = base * power_of_two(-__shfl_sync(0xffffffffu, ex, h0 * 4));
      mult1 = base * power_of_two(-__shfl_sync(0xffffffffu, ex, h1 * 4));
    }
  }

  // running softmax statistics of heads 2cc and 2cc+1 over the rows this lane sees
  float m0 = -INFINITY, l0 = 0.f, m1 = -INFINITY, l1 = 0.f;
  float *row0 = p.scores + ((int64_t)b * p.H_q + kvh * p.G + h0) * p.row_stride;
  float *row1 = row0 + p.row_stride;
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    float a0 = 0.f, a1 = 0.f, a2 = 0.f, a3 = 0.f;
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const uint32_t wa[4] = {k[t][0][j].x, k[t][0][j].y, k[t][0][j].z, k[t][0][j].w};
      const uint32_t wb[4] = {k[t][1][j].x, k[t][1][j].y, k[t][1][j].z, k[t][1][j].w};
      if (kE4m3) {
#pragma unroll
        for (int w = 0; w < 4; ++w)
          mma_f16_16816(a0, a1, a2, a3, f16x2_low(wa[w]), f16x2_low(wb[w]), f16x2_high(wa[w]), f16x2_high(wb[w]), qf[4 * j + w][0], qf[4 * j + w][1]);
      } else {
#pragma unroll
        for (int w = 0; w < 2; ++w)
          mma_bf16_16816(a0, a1, a2, a3, wa[2 * w], wb[2 * w], wa[2 * w + 1], wb[2 * w + 1], qf[2 * j + w][0], qf[2 * j + w][1]);
      }
    }
    const int r0 = tok_base + t * 16 + g, r1 = r0 + 8;
    const bool ok0 = !((absent >> (2 * t)) & 1u), ok1 = !((absent >> (2 * t + 1)) & 1u);   // a row that is not there gets no weight
    const float s00 = ok0 ? a0 * mult0 : -INFINITY, s01 = ok0 ? a1 * mult1 : -INFINITY;   // (r0,h0) (r0,h1)
    const float s10 = ok1 ? a2 * mult0 : -INFINITY, s11 = ok1 ? a3 * mult1 : -INFINITY;   // (r1,h0) (r1,h1)
    const bool v0 = r0 < p.E && SAGEKV_OK_INDEX(p.status, r0 >= 0 && (int64_t)r0 < p.row_stride);
    const bool v1 = r1 < p.E && SAGEKV_OK_INDEX(p.status, r1 >= 0 && (int64_t)r1 < p.row_stride);
    if (h0 < p.G) {
      if (v0) row0[r0] = s00;
      if (v1) row0[r1] = s10;
      const float x0 = v0 ? s00 : -INFINITY, x1 = v1 ? s10 : -INFINITY;
      const float M = fmaxf(m0, fmaxf(x0, x1));
      if (M != -INFINITY) l0 = l0 * fast_exp2(m0 - M) + fast_exp2(x0 - M) + fast_exp2(x1 - M);
      m0 = M;
    }
    if (h1 < p.G) {
      if (v0) row1[r0] = s01;
      if (v1) row1[r1] = s11;
      const float x0 = v0 ? s01 : -INFINITY, x1 = v1 ? s11 : -INFINITY;
      const float M = fmaxf(m1, fmaxf(x0, x1));
      if (M != -INFINITY) l1 = l1 * fast_exp2(m1 - M) + fast_exp2(x0 - M) + fast_exp2(x1 - M);
      m1 = M;
    }
  }
  // over the 8 row groups of the warp (lanes with equal cc), then over the warps
#pragma unroll
  for (int off = 4; off < 32; off <<= 1) {
    merge_ml(m0, l0, __shfl_xor_sync(0xffffffffu, m0, off), __shfl_xor_sync(0xffffffffu, l0, off));
    merge_ml(m1, l1, __shfl_xor_sync(0xffffffffu, m1, off), __shfl_xor_sync(0xffffffffu, l1, off));
  }
  __shared__ float2 sm[kScoreWarps][kMaxGroup];
  if (g == 0) {
    sm[warp][h0] = make_float2(m0, l0);
    sm[warp][h1] = make_float2(m1, l1);
  }
  __syncthreads();
  if (threadIdx.x < p.G) {
    const int h = threadIdx.x;
    float m = sm[0][h].x, l = sm[0][h].y;
#pragma unroll
    for (int w = 1; w < kScoreWarps; ++w) merge_ml(m, l, sm[w][h].x, sm[w][h].y);
    if (SAGEKV_OK_INDEX(p.status, chunk < p.n_chunks && kvh * p.G + h < p.H_q))
      p.partials[((int64_t)b * p.H_q + kvh * p.G + h) * p.n_chunks + chunk] = make_float2(m, l);
  }
}

cudaError_t launch_paged_score(ScoreParams p, const PagedView &c, int dtype, int n_sm, cudaStream_t stream) {
  if (p.E <= 0) return cudaSuccess;
  const bool e4m3 = dtype == SAGEKV_CACHE_E4M3;
  const int per_cta = kScoreChunk * (e4m3 ? 2 : 1);
  p.n_chunks = (p.E + per_cta - 1) / per_cta;
  p.sketch_off = score_sketch_offset(p);
  const cudaError_t e = launch_next(e4m3 ? paged_score_kernel<true> : paged_score_kernel<false>,
                                    dim3((unsigned)p.n_chunks, (unsigned)p.H_kv, (unsigned)p.B), kScoreWarps * 32, 0, stream, 0, p, c);
  return e != cudaSuccess ? e : launch_score_normalise(p, n_sm, stream);
}

// ---- compact ---------------------------------------------------------------------------------------------------------
// Rows as in sagekv_select_compact: sink, the G lists, recent tokens, last token.  A warp takes kCompactRows rows, K by its
// lower half and V by its upper one; their chain of three loads (list, table, row) runs for all of them together.  An
// 8-bit row is widened: code * scale, rounded to bf16.
constexpr int kCompactWarps = 8;
constexpr int kCompactRows = 4;

template <bool kE4m3>
__global__ void __launch_bounds__(kCompactWarps * 32) paged_compact_kernel(const PagedCompactParams p) {
  const int lane = threadIdx.x & 31, piece = lane & 15;
  const bool is_v = lane >= 16;
  wait_for_predecessor();
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.d_step = 0;
  const int n_sel = p.G * p.k_q, L = p.S + n_sel + p.R + 1;
  const int64_t n_rows = (int64_t)p.B * p.H_kv * L;
  const uint8_t *pages = is_v ? p.c.v : p.c.k;
  uint16_t *dst = is_v ? p.Vc : p.Kc;
  const float *scales = is_v ? p.c.v_scale : p.c.k_scale;
  const int64_t first = ((int64_t)blockIdx.x * kCompactWarps + (threadIdx.x >> 5)) * kCompactRows;
  int tok[kCompactRows], b[kCompactRows], kvh[kCompactRows], r[kCompactRows], page[kCompactRows];
#pragma unroll
  for (int u = 0; u < kCompactRows; ++u) {
    tok[u] = -1;
    if (first + u >= n_rows) continue;
    const int bk = (int)((first + u) / L);
    r[u] = (int)(first + u - (int64_t)bk * L);
    b[u] = bk / p.H_kv;
    kvh[u] = bk - b[u] * p.H_kv;
    if (r[u] < p.S) tok[u] = r[u];
    else if (r[u] >= p.S + n_sel) tok[u] = p.N - L + r[u];
    else {
      // the lists of a KV head's query heads lie one behind the other, as its segments do
      const int off = p.idx[(int64_t)bk * n_sel + (r[u] - p.S)];
      tok[u] = off >= 0 && off < p.E ? p.S + off : -2;
    }
  }
#pragma unroll
  for (int u = 0; u < kCompactRows; ++u)
    page[u] = tok[u] >= 0 ? p.c.table[(int64_t)b[u] * p.c.table_stride + page_of(tok[u], p.c.page_size, p.c.page_magic)] : -1;
  uint4 row[kCompactRows];
#pragma unroll
  for (int u = 0; u < kCompactRows; ++u) {
    if (tok[u] == -1) continue;
    const int64_t src = tok[u] < 0 ? -1 : paged_row(page[u], p.c.n_pages, tok[u] - page_of(tok[u], p.c.page_size, p.c.page_magic) * p.c.page_size,
                                                   kvh[u], p.c.page_stride, p.c.head_stride, p.c.token_stride);
    if (src < 0) {                                             // a position or a page id out of range: the row is left as it was
      tok[u] = -1;
      if (lane == 0) atomicOr(p.c.status, kStatusBounds);
    } else if (kE4m3) {
      const uint2 v = *reinterpret_cast<const uint2 *>(pages + src + piece * 8);
      row[u].x = v.x; row[u].y = v.y;
    } else {
      row[u] = ld_stream_v4(reinterpret_cast<const uint16_t *>(pages) + src + piece * 8);
    }
  }
#pragma unroll
  for (int u = 0; u < kCompactRows; ++u) {
    if (tok[u] == -1) continue;
    if (kE4m3) {
      const float scale = scales != nullptr ? scales[kvh[u]] : 1.f;
      const uint32_t w[4] = {f16x2_low(row[u].x), f16x2_high(row[u].x), f16x2_low(row[u].y), f16x2_high(row[u].y)};
      uint32_t y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 x = float2_of_f16x2(w[i]);
        y[i] = pack_bf16x2(x.x * scale, x.y * scale);
      }
      row[u] = make_uint4(y[0], y[1], y[2], y[3]);
    }
    st_v4(dst + (int64_t)b[u] * p.cs.batch_stride + (int64_t)kvh[u] * p.cs.head_stride + (int64_t)r[u] * p.cs.token_stride + piece * 8, row[u]);
  }
}

cudaError_t launch_paged_compact(const PagedCompactParams &p, int dtype, int n_sm, cudaStream_t stream) {
  (void)n_sm;
  const int64_t n_rows = (int64_t)p.B * p.H_kv * (p.S + (int64_t)p.G * p.k_q + p.R + 1);
  const int64_t per_block = kCompactWarps * kCompactRows, blocks = (n_rows + per_block - 1) / per_block;
  if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  return launch_next(dtype == SAGEKV_CACHE_E4M3 ? paged_compact_kernel<true> : paged_compact_kernel<false>, dim3((unsigned)blocks),
                     kCompactWarps * 32, 0, stream, 0, p);
}

}  // namespace sagekv
