// The paged cache inside the library: what a kernel needs to find a token's rows, the arguments of the kernels that
// work on pages (paged_attn.cu, paged_score.cu, paged_cache.cu), and conversions from the 8-bit type.
#pragma once

#include "common.cuh"

namespace sagekv {

// A paged cache as the kernels see it.  Page ids come from device memory, so no host check has seen them: every
// kernel compares each id with n_pages before it forms an address (in every build), leaves the access out where it
// does not fit, and sets kStatusBounds.
struct PagedView {
  uint8_t *k, *v;                                   // pages of K and of V
  int64_t page_stride, head_stride, token_stride;   // elements
  const int32_t *table;                             // [n_seqs, max_pages] page ids
  int64_t table_stride;
  const int32_t *seq_lens;                          // [n_seqs]
  const float *k_scale, *v_scale;                   // [H_kv] or null
  int32_t *status;
  int n_seqs, max_pages, n_pages, page_size;
  uint32_t page_magic;                              // floor(2^32 / page_size)
};

// position / page_size without a division (position < 2^31): the estimate is at most one too low
__host__ __device__ inline int page_of(int position, int page_size, uint32_t magic) {
  int q = (int)(((uint64_t)(uint32_t)position * magic) >> 32);
  if (position - q * page_size >= page_size) ++q;
  return q;
}
inline uint32_t page_magic(int page_size) { return (uint32_t)(((uint64_t)1 << 32) / (uint32_t)page_size); }

// element offset of a row, or -1 if the page id is none
__host__ __device__ inline int64_t paged_row(int page, int n_pages, int slot, int head, int64_t page_stride, int64_t head_stride,
                                             int64_t token_stride) {
  if (page < 0 || page >= n_pages) return -1;
  return (int64_t)page * page_stride + (int64_t)head * head_stride + (int64_t)slot * token_stride;
}

#if defined(__CUDACC__)
// checked build: is this an entry of a sequence's row of the table?
#define SAGEKV_OK_ENTRY(c, seq, entry) SAGEKV_OK_INDEX((c).status, (seq) >= 0 && (seq) < (c).n_seqs && (entry) >= 0 && (entry) < (c).max_pages)
// checked build: do these 16 rows lie in a page, and in one of its heads?
#define SAGEKV_OK_TILE(c, slot, head, H_kv) SAGEKV_OK_INDEX((c).status, (slot) >= 0 && (slot) + 16 <= (c).page_size && (head) >= 0 && (head) < (H_kv))
#endif

// ---- attention of one token per sequence over its pages -------------------------------------------------------
constexpr int kPagedCtasPerSm = 2;
constexpr int paged_attn_max_ctas(int n_sm) { return kPagedCtasPerSm * n_sm; }
__host__ __device__ constexpr int paged_part_floats(int G) { return G * kHeadDim + (2 * G + 3) / 4 * 4; }   // what a CTA leaves of a pair: O[G][128], (m, l)[G]

struct PagedAttnParams {
  PagedView c;
  const uint16_t *q;       // [n_seqs, H_q, 128], sequences q_stride apart
  int64_t q_stride;
  uint16_t *out;           // [n_seqs, H_q, 128]
  float *lse;              // [n_seqs, H_q] or null
  float *partials;         // [CTAs][2][paged_part_floats(G)]
  int32_t *tickets;        // [n_seqs * H_kv], zero between launches
  int32_t *group_tickets;  // [CTAs][2], zero between launches
  int G, H_q, H_kv;
  float scale_log2;
  int most_ctas, n_tickets;   // extents of the scratch (looked at in the checked build): CTAs with parts and group tickets, pair tickets
};
cudaError_t launch_paged_attn(const PagedAttnParams &p, int dtype, int n_sm, cudaStream_t stream);
cudaError_t paged_attn_setup();   // one-time function attributes, with the device current

// ---- rotary positions, append, score and compaction -------------------------------------------------------------
struct RopeArgs {
  uint64_t turns[kHeadDim / 2];   // revolutions per position, a 64-bit fraction
  int rotary_dim, interleaved;
  float amplitude;
};
struct PagedAppendParams {
  RopeArgs rope;                  // rotary_dim 0: nothing turns
  PagedView c;
  const uint16_t *k, *v, *q;      // q null: no queries
  uint16_t *q_out;
  int64_t kv_token, kv_head, q_token, q_head, q_out_token, q_out_head;
  const int32_t *positions, *seqs;   // seqs null: token t is sequence t's
  int64_t n_tokens;
  int H_q, H_kv;
};
constexpr int kTurnMostQuads = 8;                                  // groups of four rows of a token that a warp takes at most
constexpr int kRopeMostHeads = 65535 * kTurnMostQuads * 4;         // what a grid's second dimension covers
cudaError_t launch_rope(const PagedAppendParams &p, int n_sm, cudaStream_t stream);   // the queries alone (H_q of them; every position counts)
cudaError_t launch_paged_append(const PagedAppendParams &p, int dtype, int n_sm, cudaStream_t stream);

constexpr int kPagedScoreChunks = 64;   // CTAs that a KV head's tokens may be dealt to, however few (where the rows are not too many for it)
// p.K and p.ks are unused; p.n_chunks (at most max_chunks) is set here
cudaError_t launch_paged_score(ScoreParams p, const PagedView &c, int dtype, int max_chunks, int n_sm, cudaStream_t stream);
cudaError_t paged_score_setup();   // one-time function attributes, with the device current

struct PagedCompactParams {
  PagedView c;
  const int32_t *idx;      // [B, H_q, k_q] offsets into the eviction region
  uint16_t *Kc, *Vc;
  sagekv_strides cs;
  int32_t *d_step;
  int E, S, R, N, k_q, G, H_kv, B;
};
cudaError_t launch_paged_compact(const PagedCompactParams &p, int dtype, int n_sm, cudaStream_t stream);

#if defined(__CUDACC__)

// two e4m3 values (the low or the high half of a word) as f16: exact, NaN stays NaN
__device__ __forceinline__ uint32_t f16x2_of_e4m3x2(uint16_t x) {
  uint32_t y;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(y) : "h"(x));
  return y;
}
__device__ __forceinline__ uint32_t f16x2_low(uint32_t w) { return f16x2_of_e4m3x2((uint16_t)(w & 0xffffu)); }
__device__ __forceinline__ uint32_t f16x2_high(uint32_t w) { return f16x2_of_e4m3x2((uint16_t)(w >> 16)); }

__device__ __forceinline__ float2 float2_of_f16x2(uint32_t w) {
  float2 r;
  asm("{ .reg .f16 a, b; mov.b32 {a, b}, %2; cvt.f32.f16 %0, a; cvt.f32.f16 %1, b; }" : "=f"(r.x), "=f"(r.y) : "r"(w));
  return r;
}
// two fp32 -> packed f16x2 (lo in the low half), round to nearest even
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// two fp32 -> two e4m3 (lo in the low byte), round to nearest even, beyond +-448 the largest finite value
__device__ __forceinline__ uint32_t pack_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

// D(16x8, fp32) += A(16x16, f16, row) * B(16x8, f16, col)
__device__ __forceinline__ void mma_f16_16816(float &d0, float &d1, float &d2, float &d3, uint32_t a0, uint32_t a1, uint32_t a2,
                                              uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d0), "+f"(d1), "+f"(d2), "+f"(d3)
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// The query beside an 8-bit cache.  e4m3 values are exact in f16, and so is a bf16 query once a power of two has brought
// its largest element just below 2^14 (elements more than 2^27 times smaller than that one are rounded, to steps of at most
// 2^-37 of it): the products with the cache are those of the bf16 query.  Returns the exponent e of that power, for the largest
// magnitude of the query's elements; 0 where that is zero or not finite.
__device__ __forceinline__ int query_exponent(float largest) {
  const int biased = (int)((__float_as_uint(largest) >> 23) & 0xffu);
  if (largest == 0.f || biased == 0xff) return 0;
  return min(13 - (biased - 127), 100);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }   // -126 <= e <= 127

#endif  // __CUDACC__

}  // namespace sagekv
