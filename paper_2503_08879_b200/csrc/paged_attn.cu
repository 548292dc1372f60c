// Attention of one new token per sequence over its whole paged cache.
//
//   out[s, h] = sum_t w_t V[t] / sum_t w_t,   w_t = exp(scale <q[s, h], K[t]>),   t < seq_lens[s],
// K and V of KV head h / G.  The rows are read once, so the floor is HBM: sum of the lengths * H_kv * 2 rows.
//
// Split.  The lengths are known on the device only (a captured launch serves later lengths), and a batch may be one
// long sequence or many uneven ones.  So the 16-token tiles of all (sequence, KV head) pairs form one list, cut into
// equal ranges, one per CTA; every CTA finds its range from the lengths by a block-wide scan.  A range may
// hold the end of one pair, several whole pairs and the start of another.  Whole pairs are finished where they
// are; of a pair that several CTAs share each leaves (maximum, sum, 128 columns) per head in scratch, and the one
// that arrives last (a ticket per pair, no waiting) joins the parts in the order of the tokens: the result does not
// depend on which arrives last.
//
// In a CTA the tiles are dealt to four warps in turn, and each works for itself: its tiles come through a private ring
// (K and V of a tile, tensor copies counted on an mbarrier of the stage), it keeps a running maximum, the
// sums and the whole 128-column result in registers and refills a stage as soon as it has read it.  The page id of
// the next tile is loaded while the present one is worked on.  Products as in the streamed decode over the reduced
// cache: S = K Q^T with tokens as rows (M = 16) and the heads as columns (N = 8), O^T += V^T P.  An 8-bit cache is
// staged as it is and widened to f16 (exact) between shared memory and the tensor cores.
//
// A tile's rows behind the sequence's end hold anything: their scores are replaced, not added to, and their V rows are
// cleared in the fragments, since zero times NaN is NaN.
#include "paged.cuh"
#include "tiles.cuh"

namespace sagekv {

constexpr int kPaWarps = 4;
constexpr int kPaThreads = kPaWarps * 32;
constexpr int kPaRingBytes = 3 * 2 * kSlotBytes;    // per warp: three stages of bf16 tiles, or six of 8-bit ones
constexpr int kPaHeadStride = kHeadDim + 4;         // floats between the heads of a warp's result: the 32 lanes of a store fall into 32 banks
constexpr int kPaMinTiles = 4;                      // a CTA's least share of the list: a tile per warp
constexpr int kPaMaxStages = 6;
constexpr int kPaMaxParts = kPaWarps * kPaHeadStride;   // most CTAs that may share a pair: their factors lie in sh.o, kMaxGroup floats each

struct PaShared {
  unsigned char ring[kPaWarps][kPaRingBytes];           // boxes with the 128-byte swizzle: 1024-byte boundaries
  float o[kPaWarps][kMaxGroup * kPaHeadStride];         // results of the warps
  float2 ml[kPaWarps][kMaxGroup];                       // (max, sum) of a warp's tiles
  unsigned long long bar[kPaWarps][kPaMaxStages];
  int start[4];                                         // where my range begins: sequence, tiles of the list before it, all tiles; arrival order
};
static_assert(2 * (sizeof(PaShared) + 1024) <= 228 * 1024, "two CTAs per SM");

__device__ __forceinline__ void tensor_copy_page(uint32_t dst, const CUtensorMap *map, int x, int slot, int head, int page, uint32_t bar,
                                                 uint64_t policy) {
  tensor_copy_4d(dst, map, x, slot, head, page, bar, policy);
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// byte offset of 16-byte piece `piece` (0..7) of row `row` in a staged tile of 128-byte rows
__device__ __forceinline__ uint32_t tile8_offset(int row, int piece) { return (uint32_t)(row * 128 + ((piece ^ (row & 7)) << 4)); }

// tokens of a sequence: what the caller gave, cut to what the table can hold
__device__ __forceinline__ int tokens_of(const PagedView &c, int seq) {
  const int len = seq < c.n_seqs ? c.seq_lens[seq] : 0;
  const int most = c.max_pages * c.page_size;
  return len < 0 ? 0 : min(len, most);
}

// A place in the list of tiles: tile `tile` of head `head` of sequence `seq`, which has `len` tokens.
struct PaCursor {
  int seq, head, tile, len;
  __device__ __forceinline__ int tiles() const { return (len + 15) >> 4; }
  // moves a tile index that has run past the pair's end on to the pair that holds it
  __device__ __forceinline__ void settle(const PagedView &c, int H_kv) {
    while (tile >= tiles() && seq < c.n_seqs) {
      tile -= tiles();
      if (len == 0 || ++head == H_kv) {
        head = 0;
        len = tokens_of(c, ++seq);
      }
    }
  }
};

template <bool kE4m3>
__global__ void __launch_bounds__(kPaThreads, kPagedCtasPerSm)
paged_attn_kernel(const PagedAttnParams p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  constexpr int kRowBytes = kE4m3 ? 128 : 256;
  constexpr int kTileBytes = 16 * kRowBytes;
  constexpr int kStageBytes = 2 * kTileBytes;                // K and V of one tile
  constexpr int kStages = kPaRingBytes / kStageBytes;
  static_assert(kStages <= kPaMaxStages, "barriers");
  // 8-bit caches: the weights go to the second product in f16, up to 2^14, so that the small ones (down to 2^-38 of the
  // largest) are not lost; bf16 has the range without that
  constexpr float kWeightShift = kE4m3 ? 14.f : 0.f;
  extern __shared__ __align__(1024) unsigned char pa_smem[];
  PaShared &sh = *reinterpret_cast<PaShared *>(pa_smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = lane >> 2, c = lane & 3, h0 = 2 * c, h1 = 2 * c + 1;

  const uint32_t ring = smem_u32(&sh.ring[warp][0]), bars = smem_u32(&sh.bar[warp][0]);
  if (lane == 0) {
#pragma unroll
    for (int s = 0; s < kStages; ++s) mbar_init(bars + 8u * s, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
  }
  wait_for_predecessor();

  // ---- my range of the list ----
  const int per_thread = (p.c.n_seqs + kPaThreads - 1) / kPaThreads;
  const int s0 = min(tid * per_thread, p.c.n_seqs), s1 = min(s0 + per_thread, p.c.n_seqs);
  int mine = 0;
  for (int s = s0; s < s1; ++s) {
    const int len = p.c.seq_lens[s];
    if (len < 0 || len > p.c.max_pages * p.c.page_size) atomicOr(p.c.status, kStatusBounds);
    mine += (tokens_of(p.c, s) + 15) >> 4;
  }
  int incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  int *warp_total = reinterpret_cast<int *>(sh.o[0]);
  if (lane == 31) warp_total[warp] = incl;
  __syncthreads();
  int total = 0, before = incl - mine;
#pragma unroll
  for (int w = 0; w < kPaWarps; ++w) {
    if (w < warp) before += warp_total[w];
    total += warp_total[w];
  }
  const int n_ctas = (int)gridDim.x;
  const int all = total * p.H_kv;                            // fits: the host has checked the most the tables can hold
  int per_cta = max((int)(((int64_t)all + n_ctas - 1) / n_ctas), kPaMinTiles);
  if (per_cta < 64) per_cta = (per_cta + kPaWarps - 1) & ~(kPaWarps - 1);   // the same for the busiest warp, fewer parts to join
  const int lo = (int)min((int64_t)blockIdx.x * per_cta, (int64_t)all), n = min(per_cta, all - lo);
  if (mine > 0 && lo >= before * p.H_kv && lo < (before + mine) * p.H_kv) {   // the range begins in one of this thread's sequences
    int at = before, s = s0;
    for (int len; at + (len = (tokens_of(p.c, s) + 15) >> 4) <= lo / p.H_kv; ++s) at += len;
    sh.start[0] = s;
    sh.start[1] = at * p.H_kv;
  }
  __syncthreads();

  if (n > 0) {
    // ---- requests: one tile ahead the page id, kStages tiles ahead the rows ----
    PaCursor next;                                           // my next tile to request
    next.seq = sh.start[0];
    next.len = tokens_of(p.c, next.seq);
    const int into = lo - sh.start[1], first_head = into / next.tiles(), first_tile = into - first_head * next.tiles();
    next.head = first_head;
    next.tile = first_tile + warp;
    int rx = warp;                                           // its index in my range
    const int tiles_per_page = p.c.page_size >> 4;
    uint64_t stream_policy;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(stream_policy));
    int next_page = -1, next_slot = 0;
    auto look_up = [&] {
      next_page = -1;
      if (rx >= n) return;
      next.settle(p.c, p.H_kv);
      if (next.seq >= p.c.n_seqs) return;
      const int entry = next.tile / tiles_per_page;
      next_slot = (next.tile - entry * tiles_per_page) << 4;
      next_page = p.c.table[(int64_t)next.seq * p.c.table_stride + entry];
    };
    uint32_t absent = 0u;                                    // stages whose page id is none: nothing is on its way
    auto request = [&](int s) {
      if (rx >= n) return;
      const uint32_t bar = bars + 8u * s;
      if (next_page >= 0 && next_page < p.c.n_pages) {
        absent &= ~(1u << s);
        if (lane == 0) mbar_expect_tx(bar, kStageBytes);
        __syncwarp();
        constexpr int kBoxes = kE4m3 ? 2 : 4;                // 16 rows of 128 bytes each
        if (lane < kBoxes)
          tensor_copy_page(ring + (uint32_t)(s * kStageBytes + lane * kHalfBytes), lane < kBoxes / 2 ? &map_k : &map_v,
                           kE4m3 ? 0 : (lane & 1) * 64, next_slot, next.head, next_page, bar, stream_policy);
      } else {
        absent |= 1u << s;
        if (lane == 0) {
          mbar_arrive(bar);
          atomicOr(p.c.status, kStatusBounds);
        }
      }
      rx += kPaWarps;
      next.tile += kPaWarps;
      look_up();
    };
    look_up();
#pragma unroll
    for (int s = 0; s < kStages; ++s) request(s);

    // fragment addresses within a stage
    const int mi = lane >> 3, l8 = lane & 7;
    uint32_t k_off[8], v_off[8];
#pragma unroll
    for (int j = 0; j < (kE4m3 ? 4 : 8); ++j) {
      if (kE4m3) {
        k_off[j] = v_off[j] = tile8_offset((mi & 1) * 8 + l8, 2 * j + (mi >> 1));
        v_off[j] += kTileBytes;
      } else {
        k_off[j] = tile_offset((mi & 1) * 8 + l8, 2 * j + (mi >> 1));
        v_off[j] = kTileBytes + tile_offset((mi >> 1) * 8 + l8, 2 * j + (mi & 1));
      }
    }
    const bool in0 = h0 < p.G, in1 = h1 < p.G;

    bool timed_out = false;
    int stage = 0;
    uint32_t phase = 0;
    int x = warp;                                            // my next tile, as an index into my range
    PaCursor at;                                             // the pair being worked on
    at.seq = sh.start[0];
    at.len = tokens_of(p.c, at.seq);
    at.head = first_head;
    int pair_x0 = -first_tile;                               // index (may be negative) of the pair's tile 0 in the range
    while (pair_x0 < n && at.seq < p.c.n_seqs) {
      const int pair_tiles = at.tiles(), x_end = min(n, pair_x0 + pair_tiles);
      // B fragments of Q^T: lane (g, c) holds of head g, bf16: dims 16j + 2c, +1 and 16j + 8 + 2c, +1; 8-bit: 16j + 4c .. + 3
      uint32_t qb[8][2];
      float mult0 = p.scale_log2, mult1 = p.scale_log2;      // what brings a score of heads 2c, 2c + 1 to log2 units
      {
        const uint16_t *q_row = p.q + (int64_t)at.seq * p.q_stride + (at.head * p.G + min(g, p.G - 1)) * kHeadDim;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          qb[j][0] = qb[j][1] = 0u;
          if (g < p.G) {
            if (kE4m3) {
              const uint2 v = *reinterpret_cast<const uint2 *>(q_row + 16 * j + 4 * c);
              qb[j][0] = v.x; qb[j][1] = v.y;
            } else {
              qb[j][0] = *reinterpret_cast<const uint32_t *>(q_row + 16 * j + 2 * c);
              qb[j][1] = *reinterpret_cast<const uint32_t *>(q_row + 16 * j + 8 + 2 * c);
            }
          }
        }
        if (kE4m3) {
          float largest = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) largest = fmaxf(largest, fmaxf(fabsf(bf16_low(qb[j][e])), fabsf(bf16_high(qb[j][e]))));
          largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, 1));
          largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, 2));
          const int e = query_exponent(largest);
          const float up = power_of_two(e);
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i) qb[j][i] = pack_f16x2(bf16_low(qb[j][i]) * up, bf16_high(qb[j][i]) * up);
          const float base = p.c.k_scale != nullptr ? p.scale_log2 * p.c.k_scale[at.head] : p.scale_log2;
          mult0 = base * power_of_two(-__shfl_sync(0xffffffffu, e, h0 * 4));
          mult1 = base * power_of_two(-__shfl_sync(0xffffffffu, e, h1 * 4));
        }
      }

      float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;   // the maxima are kept kWeightShift below the scores'
      float acc[8][4];
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;

      for (; x < x_end; x += kPaWarps) {
        const uint32_t tb = ring + (uint32_t)(stage * kStageBytes);
        if (!mbar_wait(bars + 8u * stage, phase)) timed_out = true;
        if (!((absent >> stage) & 1u)) {
          // ---- S = K Q^T, four accumulator chains: lane (g, c) gets tokens g, g + 8 of heads 2c, 2c + 1 ----
          float ch[4][4];
#pragma unroll
          for (int j = 0; j < 4; ++j) ch[j][0] = ch[j][1] = ch[j][2] = ch[j][3] = 0.f;
          uint32_t fa[4];
          uint32_t va[8][4];
          if (kE4m3) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              ldmatrix_x4(tb + k_off[j], fa[0], fa[1], fa[2], fa[3]);
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                float(&d)[4] = ch[(2 * j + e) & 3];
                mma_f16_16816(d[0], d[1], d[2], d[3], f16x2_low(fa[2 * e]), f16x2_low(fa[2 * e + 1]), f16x2_high(fa[2 * e]),
                              f16x2_high(fa[2 * e + 1]), qb[2 * j + e][0], qb[2 * j + e][1]);
              }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              // tokens 2c, 2c + 1 (and + 8) of dims 2g, 2g + 1 of two pieces, regrouped by dim
              ldmatrix_x4_trans(tb + v_off[j], fa[0], fa[1], fa[2], fa[3]);
#pragma unroll
              for (int e = 0; e < 4; ++e) fa[e] = __byte_perm(fa[e], 0u, 0x3120);
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                va[2 * j + e][0] = f16x2_low(fa[2 * e]);
                va[2 * j + e][1] = f16x2_high(fa[2 * e]);
                va[2 * j + e][2] = f16x2_low(fa[2 * e + 1]);
                va[2 * j + e][3] = f16x2_high(fa[2 * e + 1]);
              }
            }
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              ldmatrix_x4(tb + k_off[j], fa[0], fa[1], fa[2], fa[3]);
              float(&d)[4] = ch[j & 3];
              mma_bf16_16816(d[0], d[1], d[2], d[3], fa[0], fa[1], fa[2], fa[3], qb[j][0], qb[j][1]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) ldmatrix_x4_trans(tb + v_off[j], va[j][0], va[j][1], va[j][2], va[j][3]);
          }
          // ---- softmax weights ----
          float sv[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) sv[e] = ((ch[0][e] + ch[1][e]) + (ch[2][e] + ch[3][e])) * (e & 1 ? mult1 : mult0);
          const int left = at.len - ((x - pair_x0) << 4);    // tokens of the sequence from this tile's first on
          if (left < 16) {
            if (g >= left) sv[0] = sv[1] = -INFINITY;
            if (g + 8 >= left) sv[2] = sv[3] = -INFINITY;
            const uint32_t keep_lo = (2 * c < left ? 0xffffu : 0u) | (2 * c + 1 < left ? 0xffff0000u : 0u);
            const uint32_t keep_hi = (2 * c + 8 < left ? 0xffffu : 0u) | (2 * c + 9 < left ? 0xffff0000u : 0u);
#pragma unroll
            for (int j = 0; j < 8; ++j) { va[j][0] &= keep_lo; va[j][1] &= keep_lo; va[j][2] &= keep_hi; va[j][3] &= keep_hi; }
          }
          if (!in0) sv[0] = sv[2] = -INFINITY;
          if (!in1) sv[1] = sv[3] = -INFINITY;
          float t0 = fmaxf(sv[0], sv[2]) - kWeightShift, t1 = fmaxf(sv[1], sv[3]) - kWeightShift;
          if (__any_sync(0xffffffffu, t0 > m0 || t1 > m1)) {   // a new maximum: seldom after the first tiles
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) {
              t0 = fmaxf(t0, __shfl_xor_sync(0xffffffffu, t0, o));
              t1 = fmaxf(t1, __shfl_xor_sync(0xffffffffu, t1, o));
            }
            t0 = fmaxf(t0, m0); t1 = fmaxf(t1, m1);
            const float f0 = t0 == m0 ? 1.f : fast_exp2(m0 - t0), f1 = t1 == m1 ? 1.f : fast_exp2(m1 - t1);
            m0 = t0; m1 = t1;
            l0 *= f0; l1 *= f1;
#pragma unroll
            for (int j = 0; j < 8; ++j) { acc[j][0] *= f0; acc[j][1] *= f1; acc[j][2] *= f0; acc[j][3] *= f1; }
          }
          const float r0 = m0 == -INFINITY ? 0.f : m0, r1 = m1 == -INFINITY ? 0.f : m1;
          const float w0 = fast_exp2(sv[0] - r0), w1 = fast_exp2(sv[1] - r1), w2 = fast_exp2(sv[2] - r0), w3 = fast_exp2(sv[3] - r1);
          l0 += w0 + w2;                                     // (in 32 bits: the log-sum-exp is read from them)
          l1 += w1 + w3;
          const uint32_t pa = kE4m3 ? pack_f16x2(w0, w1) : pack_bf16x2(w0, w1), pb = kE4m3 ? pack_f16x2(w2, w3) : pack_bf16x2(w2, w3);
          const uint32_t b0 = movmatrix(pa), b1 = movmatrix(pb);   // head g, tokens 2c, 2c + 1 and 2c + 8, 2c + 9
          // ---- O^T += V^T P: lane (g, c) holds two dims (see the stores below) of heads 2c and 2c + 1 ----
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            if (kE4m3) mma_f16_16816(acc[j][0], acc[j][1], acc[j][2], acc[j][3], va[j][0], va[j][1], va[j][2], va[j][3], b0, b1);
            else mma_bf16_16816(acc[j][0], acc[j][1], acc[j][2], acc[j][3], va[j][0], va[j][1], va[j][2], va[j][3], b0, b1);
          }
          __syncwarp();                                      // every lane has its fragments: the stage may be refilled
        }
        request(stage);
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
      }

      // ---- the pair (or my part of it) is done: merge the four warps ----
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        l0 += __shfl_xor_sync(0xffffffffu, l0, o);
        l1 += __shfl_xor_sync(0xffffffffu, l1, o);
      }
      __syncthreads();                                       // the previous pair's results have been read
      if (g == 0) { sh.ml[warp][h0] = make_float2(m0, l0); sh.ml[warp][h1] = make_float2(m1, l1); }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        constexpr int kStep = kE4m3 ? 1 : 8;                 // dims 16j + 2g, + 1 (8-bit) or 16j + g, + 8
        float *o0 = sh.o[warp] + h0 * kPaHeadStride + 16 * j + (kE4m3 ? 2 * g : g), *o1 = o0 + kPaHeadStride;
        o0[0] = acc[j][0]; o1[0] = acc[j][1]; o0[kStep] = acc[j][2]; o1[kStep] = acc[j][3];
      }
      __syncthreads();
      const int pair_first = lo + pair_x0;                   // the pair's first tile in the list
      const int cta_first = pair_first / per_cta, cta_last = (pair_first + pair_tiles - 1) / per_cta;
      const bool whole = cta_first == cta_last;
      const int64_t row0 = (int64_t)at.seq * p.H_q + at.head * p.G;   // the pair's first row of out and lse
      const float v_scale = kE4m3 && p.c.v_scale != nullptr ? p.c.v_scale[at.head] : 1.f;
      auto finish = [&](int h, int col, float4 o, float M, float l) {
        const float inv = l == 0.f ? 0.f : v_scale / l;
        *reinterpret_cast<uint2 *>(p.out + (row0 + h) * kHeadDim + col) = make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
        if (p.lse != nullptr && col == 0) p.lse[row0 + h] = l == 0.f ? -INFINITY : (M + log2f(l)) * kLn2;
      };
      // of a shared pair: slot 0 of a CTA whose range begins inside the pair, slot 1 of the one where the pair begins
      float *part = p.partials + ((int64_t)blockIdx.x * 2 + (cta_first == (int)blockIdx.x ? 1 : 0)) * kPartialStride;
      for (int item = tid; item < p.G * (kHeadDim / 4); item += kPaThreads) {
        const int h = item >> 5, col = (item & 31) * 4;
        float M = -INFINITY, l = 0.f;
#pragma unroll
        for (int w = 0; w < kPaWarps; ++w) M = fmaxf(M, sh.ml[w][h].x);
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kPaWarps; ++w) {
          const float2 ml = sh.ml[w][h];
          const float f = ml.x == M ? 1.f : fast_exp2(ml.x - M);   // (equal also where both are infinite)
          const float4 v = *reinterpret_cast<const float4 *>(sh.o[w] + h * kPaHeadStride + col);
          l += ml.y * f;
          o.x += v.x * f; o.y += v.y * f; o.z += v.z * f; o.w += v.w * f;
        }
        if (whole) {
          finish(h, col, o, M, l);
        } else {
          *reinterpret_cast<float4 *>(part + h * kHeadDim + col) = o;
          if (col == 0) *reinterpret_cast<float2 *>(part + kMaxGroup * kHeadDim + 2 * h) = make_float2(M, l);
        }
      }
      if (!whole) {
        __threadfence();
        __syncthreads();
        const int parts = cta_last - cta_first + 1;
        int32_t *ticket = p.tickets + (int64_t)at.seq * p.H_kv + at.head;
        if (tid == 0) sh.start[3] = atomicAdd(ticket, 1);
        __syncthreads();
        if (sh.start[3] == parts - 1) {                      // every other part is in scratch
          __threadfence();
          if (tid == 0) *ticket = 0;
          const float *first = p.partials + ((int64_t)cta_first * 2 + 1) * kPartialStride;
          auto part_of = [&](int i) { return i == 0 ? first : first + ((int64_t)i * 2 - 1) * kPartialStride; };
          float *factor = sh.o[0];                           // [part][head]; every thread has read the warps' results
          float Ms[kMaxGroup / 4], ls[kMaxGroup / 4];        // of the heads h = warp, warp + 4: their lanes take the parts in turn
#pragma unroll
          for (int k = 0; k < kMaxGroup / 4; ++k) {
            const int h = warp + 4 * k;
            Ms[k] = -INFINITY; ls[k] = 0.f;
            if (h < p.G) {
              for (int i = lane; i < parts; i += 32) Ms[k] = fmaxf(Ms[k], __ldcg(part_of(i) + kMaxGroup * kHeadDim + 2 * h));
#pragma unroll
              for (int o = 1; o < 32; o <<= 1) Ms[k] = fmaxf(Ms[k], __shfl_xor_sync(0xffffffffu, Ms[k], o));
              for (int i = lane; i < parts; i += 32) {
                const float2 ml = __ldcg(reinterpret_cast<const float2 *>(part_of(i) + kMaxGroup * kHeadDim + 2 * h));
                const float f = ml.x == Ms[k] ? 1.f : fast_exp2(ml.x - Ms[k]);
                factor[i * kMaxGroup + h] = f;
                ls[k] += ml.y * f;
              }
#pragma unroll
              for (int o = 1; o < 32; o <<= 1) ls[k] += __shfl_xor_sync(0xffffffffu, ls[k], o);
              if (lane == 0) sh.ml[0][h] = make_float2(Ms[k], ls[k]);
            }
          }
          __syncthreads();
          for (int item = tid; item < p.G * (kHeadDim / 4); item += kPaThreads) {
            const int h = item >> 5, col = (item & 31) * 4;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
            for (int i = 0; i < parts; ++i) {
              const float4 v = __ldcg(reinterpret_cast<const float4 *>(part_of(i) + h * kHeadDim + col));
              const float f = factor[i * kMaxGroup + h];
              o.x += v.x * f; o.y += v.y * f; o.z += v.z * f; o.w += v.w * f;
            }
            finish(h, col, o, sh.ml[0][h].x, sh.ml[0][h].y);
          }
        }
      }
      // ---- the next pair with tokens ----
      pair_x0 += pair_tiles;
      if (++at.head == p.H_kv) {
        at.head = 0;
        do at.len = tokens_of(p.c, ++at.seq);
        while (at.len == 0 && at.seq < p.c.n_seqs);
      }
    }
    if (timed_out) atomicOr(p.c.status, kStatusWaitTimeout);
  }

  // ---- sequences without tokens ----
  for (int s = blockIdx.x; s < p.c.n_seqs; s += n_ctas) {
    if (tokens_of(p.c, s) > 0) continue;
    for (int i = tid; i < p.H_q * (kHeadDim / 8); i += kPaThreads) st_v4(p.out + (int64_t)s * p.H_q * kHeadDim + i * 8, make_uint4(0u, 0u, 0u, 0u));
    if (p.lse != nullptr)
      for (int i = tid; i < p.H_q; i += kPaThreads) p.lse[(int64_t)s * p.H_q + i] = -INFINITY;
  }
}

// [n_pages, H_kv, page_size, 128] through the cache's strides, boxes of 16 rows x 128 bytes with the 128-byte swizzle
static bool make_page_map(CUtensorMap *map, uint8_t *base, const PagedAttnParams &p, bool e4m3) {
  EncodeTiledFn enc = encode_tiled_fn();
  if (enc == nullptr) return false;
  const cuuint64_t size = e4m3 ? 1 : 2;
  const cuuint64_t dims[4] = {(cuuint64_t)kHeadDim, (cuuint64_t)p.c.page_size, (cuuint64_t)p.H_kv, (cuuint64_t)p.c.n_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)p.c.token_stride * size, (cuuint64_t)p.c.head_stride * size, (cuuint64_t)p.c.page_stride * size};
  const cuuint32_t box[4] = {e4m3 ? 128u : 64u, 16, 1, 1};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  return enc(map, e4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, base, dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t paged_attn_setup() {
  cudaError_t e = cudaFuncSetAttribute(paged_attn_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(PaShared));
  if (e == cudaSuccess) e = cudaFuncSetAttribute(paged_attn_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(PaShared));
  return e;
}

cudaError_t launch_paged_attn(const PagedAttnParams &p, int dtype, int n_sm, cudaStream_t stream) {
  if (p.c.n_seqs <= 0) return cudaSuccess;
  const bool e4m3 = dtype == SAGEKV_CACHE_E4M3;
  CUtensorMap map_k, map_v;
  if (!make_page_map(&map_k, p.c.k, p, e4m3) || !make_page_map(&map_v, p.c.v, p, e4m3)) return cudaErrorInvalidValue;
  const int64_t most = (int64_t)p.c.n_seqs * p.H_kv * p.c.max_pages * (p.c.page_size / 16);   // tiles, if every sequence filled its table
  int64_t ctas = (most + kPaMinTiles - 1) / kPaMinTiles;
  int most_ctas = paged_attn_max_ctas(n_sm);
  static_assert(kPaMaxParts >= 2 * 160, "a pair may be shared by every CTA");
  if (most_ctas > kPaMaxParts) most_ctas = kPaMaxParts;
  if (ctas > most_ctas) ctas = most_ctas;
  if (ctas < 1) ctas = 1;
  return launch_next(e4m3 ? paged_attn_kernel<true> : paged_attn_kernel<false>, dim3((unsigned)ctas), kPaThreads, sizeof(PaShared), stream, 0,
                     p, map_k, map_v);
}

}  // namespace sagekv
