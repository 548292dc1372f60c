// Step 2 of the method (first half) on pages: sagekv_score with a block table between a token and its row.
//
// As in the attention over pages, 16-token tiles of K come into shared memory by tensor copies and go from there into
// matrix fragments; here every sequence has the same length, so a KV head's tiles are simply dealt to `n_chunks` CTAs, and in
// a CTA to its warps in turn.  A warp's page ids are looked up 32 tiles at a time.  (Loading the rows straight into
// fragments, as the score step without pages does, puts the look-up in front of every CTA's loads: both passes on 131072
// tokens x 8 heads 59.6 us, this 48.1.)  Writes the scaled logits and a (max, sum) pair per CTA and head; the second pass is the
// score step's own, 7 us of those.  Bound by HBM, K being read once, and like the attention served best by few bytes in flight (us, bf16 / 8-bit
// cache: 18 warps per SM with 8 KB each 50.1 / 35.0, 24 with 8 KB 50.2 / 36.0, 24 with 4 KB 48.1 / 34.2).
#include "paged_tiles.cuh"

namespace sagekv {

constexpr int kPsWarps = 8;
constexpr int kPsThreads = kPsWarps * 32;
constexpr int kPsRingBytes = kSlotBytes;        // per warp: one stage of bf16 tiles, or two of 8-bit ones
constexpr int kPsCtasPerSm = 3;
constexpr int kPsMaxStages = 2;

struct PsShared {
  unsigned char ring[kPsWarps][kPsRingBytes];   // boxes with the 128-byte swizzle: 1024-byte boundaries
  float2 ml[kPsWarps][kMaxGroup];
  unsigned long long bar[kPsWarps][kPsMaxStages];
};

// The CTA (x, kv head, sequence) takes units [x * per_cta, ...) of the n_units units of kPsWarps tiles from the region's first on.
template <bool kE4m3>
__global__ void __launch_bounds__(kPsThreads, kPsCtasPerSm)
paged_score_kernel(const ScoreParams p, const PagedView c, const __grid_constant__ CUtensorMap map_k, const int n_units, const int per_cta) {
  constexpr int kTileBytes = 16 * (kE4m3 ? 128 : 256);
  constexpr int kStages = kPsRingBytes / kTileBytes;
  static_assert(kStages <= kPsMaxStages, "barriers");
  extern __shared__ __align__(1024) unsigned char ps_smem[];
  PsShared &sh = *reinterpret_cast<PsShared *>(ps_smem);
  const int chunk = blockIdx.x, kvh = blockIdx.y, b = blockIdx.z;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, cc = lane & 3;
  const uint32_t ring = smem_u32(&sh.ring[warp][0]), bars = smem_u32(&sh.bar[warp][0]);
  if (lane == 0) {
#pragma unroll
    for (int s = 0; s < kStages; ++s) mbar_init(bars + 8u * s, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
  }
  __syncwarp();
  wait_for_predecessor();

  const int first_tile = p.S >> 4, end_tile = (p.S + p.E + 15) >> 4;
  const int u_end = min(n_units, (chunk + 1) * per_cta);
  int next = chunk * per_cta;                                  // the unit of my next tile to request
  const int32_t *table = c.table + (int64_t)b * c.table_stride;
  int ids = -1, ids_unit = 0, next_page = -1, next_slot = 0;
  uint32_t absent = 0u;                                        // stages whose page id is none: nothing is on its way
  uint64_t stream_policy;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(stream_policy));
  auto tile_of = [&](int unit) { return first_tile + unit * kPsWarps + warp; };
  auto look_up = [&](bool anew) {
    if (next >= u_end || tile_of(next) >= end_tile) return;
    if (anew || next - ids_unit >= 32) {
      ids_unit = next;
      const int tile = tile_of(next + lane);
      const int entry = page_of(tile << 4, c.page_size, c.page_magic);
      ids = tile < end_tile && SAGEKV_OK_ENTRY(c, b, entry) ? table[entry] : -1;
    }
    const int first = tile_of(next) << 4;
    next_slot = first - page_of(first, c.page_size, c.page_magic) * c.page_size;
    next_page = __shfl_sync(0xffffffffu, ids, next - ids_unit);
  };
  auto request = [&](int s) {
    if (next >= u_end || tile_of(next) >= end_tile) return;
    const uint32_t bar = bars + 8u * s;
    if (next_page >= 0 && next_page < c.n_pages && SAGEKV_OK_TILE(c, next_slot, kvh, p.H_kv)) {
      absent &= ~(1u << s);
      if (lane == 0) mbar_expect_tx(bar, kTileBytes);
      __syncwarp();
      if (lane < (kE4m3 ? 1 : 2))
        tensor_copy_4d(ring + (uint32_t)(s * kTileBytes + lane * kHalfBytes), &map_k, lane * 64, next_slot, kvh, next_page, bar, stream_policy);
    } else {
      absent |= 1u << s;
      if (lane == 0) {
        mbar_arrive(bar);
        atomicOr(c.status, kStatusBounds);
      }
    }
    ++next;
    look_up(false);
  };
  look_up(true);
#pragma unroll
  for (int s = 0; s < kStages; ++s) request(s);

  if (chunk == 0 && p.sketch_off >= 0) {                       // the rows' histograms are filled by atomic adds in the second pass
    for (int i = threadIdx.x; i < p.G * (kSketchBins + 4); i += kPsThreads) {
      const int h = i / (kSketchBins + 4);
      if (!SAGEKV_OK_INDEX(p.status, p.sketch_off >= p.E && p.sketch_off + kSketchBins + 4 <= p.row_stride && kvh * p.G + h < p.H_q)) continue;
      reinterpret_cast<uint32_t *>(p.scores + ((int64_t)b * p.H_q + kvh * p.G + h) * p.row_stride + p.sketch_off)[i - h * (kSketchBins + 4)] = 0u;
    }
  }
  uint32_t k_off[8], qb[8][2];
  float mult0, mult1;
  k_fragment_offsets<kE4m3>(lane, k_off);
  load_queries<kE4m3>(p.q + ((int64_t)b * p.H_q + kvh * p.G) * kHeadDim, p.G, c.k_scale, kvh, p.scale_log2, lane, qb, mult0, mult1);

  // running softmax statistics of heads 2cc and 2cc + 1 over the tokens this lane sees
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  float *row0 = p.scores + ((int64_t)b * p.H_q + kvh * p.G + 2 * cc) * p.row_stride;
  bool timed_out = false;
  int stage = 0;
  uint32_t phase = 0;
  for (int unit = chunk * per_cta; unit < u_end && tile_of(unit) < end_tile; ++unit) {
    float sv[4];
    if (!mbar_wait(bars + 8u * stage, phase)) timed_out = true;
    if ((absent >> stage) & 1u) {                              // tokens that are not there get no weight; a row without any stays finite
      sv[0] = sv[1] = sv[2] = sv[3] = -3.40282347e38f;         // (the lowest number: no logit is below it)
    } else {
      score_tile<kE4m3>(ring + (uint32_t)(stage * kTileBytes), k_off, qb, mult0, mult1, sv);
    }
    // Every lane has its fragments, and has seen this phase of the barrier: the stage may be refilled.  (Where the next tile's page is
    // none, lane 0 completes the next phase at once: a lane that still polled for this one would then never see it.)
    __syncwarp();
    request(stage);
    if (++stage == kStages) { stage = 0; phase ^= 1u; }
    const int i0 = (tile_of(unit) << 4) + g - p.S, i1 = i0 + 8;   // places in the eviction region: the first and last tiles reach beyond
    const bool v0 = i0 >= 0 && i0 < p.E && SAGEKV_OK_INDEX(p.status, (int64_t)i0 < p.row_stride);
    const bool v1 = i1 >= 0 && i1 < p.E && SAGEKV_OK_INDEX(p.status, (int64_t)i1 < p.row_stride);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if (2 * cc + e >= p.G || !SAGEKV_OK_INDEX(p.status, kvh * p.G + 2 * cc + e < p.H_q && b < p.B)) continue;
      float *row = row0 + e * p.row_stride;
      if (v0) row[i0] = sv[e];
      if (v1) row[i1] = sv[2 + e];
      const float x0 = v0 ? sv[e] : -INFINITY, x1 = v1 ? sv[2 + e] : -INFINITY;
      const float M = fmaxf(m[e], fmaxf(x0, x1));
      if (M != -INFINITY) l[e] = l[e] * fast_exp2(m[e] - M) + fast_exp2(x0 - M) + fast_exp2(x1 - M);
      m[e] = M;
    }
  }
  if (timed_out) atomicOr(p.status, kStatusWaitTimeout);
  // over the 8 row groups of the warp (lanes with equal cc), then over the warps
#pragma unroll
  for (int off = 4; off < 32; off <<= 1)
#pragma unroll
    for (int e = 0; e < 2; ++e) merge_ml(m[e], l[e], __shfl_xor_sync(0xffffffffu, m[e], off), __shfl_xor_sync(0xffffffffu, l[e], off));
  if (g == 0) {
    sh.ml[warp][2 * cc] = make_float2(m[0], l[0]);
    sh.ml[warp][2 * cc + 1] = make_float2(m[1], l[1]);
  }
  __syncthreads();
  if (threadIdx.x < p.G) {
    const int h = threadIdx.x;
    float M = sh.ml[0][h].x, sum = sh.ml[0][h].y;
#pragma unroll
    for (int w = 1; w < kPsWarps; ++w) merge_ml(M, sum, sh.ml[w][h].x, sh.ml[w][h].y);
    if (SAGEKV_OK_INDEX(p.status, chunk < p.n_chunks && kvh * p.G + h < p.H_q))
      p.partials[((int64_t)b * p.H_q + kvh * p.G + h) * p.n_chunks + chunk] = make_float2(M, sum);
  }
}

cudaError_t paged_score_setup() {
  cudaError_t e = cudaFuncSetAttribute(paged_score_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(PsShared));
  if (e == cudaSuccess) e = cudaFuncSetAttribute(paged_score_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(PsShared));
  return e;
}

cudaError_t launch_paged_score(ScoreParams p, const PagedView &c, int dtype, int max_chunks, int n_sm, cudaStream_t stream) {
  if (p.E <= 0) return cudaSuccess;
  const bool e4m3 = dtype == SAGEKV_CACHE_E4M3;
  CUtensorMap map_k;
  if (!make_page_map(&map_k, c.k, c, p.H_kv, e4m3)) return cudaErrorInvalidValue;
  const int tiles = ((p.S + p.E + 15) >> 4) - (p.S >> 4), n_units = (tiles + kPsWarps - 1) / kPsWarps;
  // one wave of CTAs; with so many heads that fewer than four would share one, eight each: the waves then even out
  const int heads = p.B * p.H_kv, wave = kPsCtasPerSm * n_sm;
  int ctas = heads > wave / 4 ? 8 : wave / heads;
  if (ctas > n_units) ctas = n_units;                          // a CTA's least share: a tile per warp
  if (ctas > max_chunks) ctas = max_chunks;
  const int per_cta = (n_units + ctas - 1) / ctas;
  p.n_chunks = (n_units + per_cta - 1) / per_cta;
  p.sketch_off = score_sketch_offset(p);
  const cudaError_t e = launch_next(e4m3 ? paged_score_kernel<true> : paged_score_kernel<false>,
                                    dim3((unsigned)p.n_chunks, (unsigned)p.H_kv, (unsigned)p.B), kPsThreads, sizeof(PsShared), stream, 0, p, c,
                                    map_k, n_units, per_cta);
  return e != cudaSuccess ? e : launch_score_normalise(p, n_sm, stream);
}

}  // namespace sagekv
