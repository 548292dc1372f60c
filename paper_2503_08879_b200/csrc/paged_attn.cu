// Attention of one new token per sequence over its whole paged cache.
//
//   out[s, h] = sum_t w_t V[t] / sum_t w_t,   w_t = exp(scale <q[s, h], K[t]>),   t < seq_lens[s],
// K and V of KV head h / G.  The rows are read once: sum of the lengths * H_kv * 2 rows out of HBM.  ("Bytes" below is that at the rate of a
// copy, which a stream that only reads may pass by a few per cent.)
//
// Split.  The lengths are known on the device only (a captured launch serves later lengths), and a batch may be one
// long sequence or many uneven ones.  So all (sequence, KV head) pairs form one list of units of six 16-token tiles, a
// tile per warp, cut into equal ranges, one per CTA; every CTA finds its range from the lengths by a scan.  A range may
// hold the end of one pair, several whole pairs and the start of another; in front of each pair the list has two empty places, so that a
// CTA whose range changes pairs gets that much less to do (without them those CTAs were the last ones, 10 us behind the
// others at 131072 tokens x 8 heads).  Whole pairs are finished where they are; of a pair that several CTAs share each leaves
// (maximum, sum, 128 columns) per head in scratch, and the one that arrives last (a ticket per pair, no waiting) joins
// the parts, each warp always the same ones: the result does not depend on which arrives last.
//
// In a CTA each warp works for itself: its tiles come through a private ring (K and V of a tile, tensor copies counted on an
// mbarrier of the stage), it keeps a running maximum, the sums and the whole 128-column result in registers and refills a
// stage as soon as it has read it.  Page ids are looked up 32 tiles at a time.  Products as in the streamed decode over the
// reduced cache: S = K Q^T with tokens as rows (M = 16) and the heads as columns (N = 8), O^T += V^T P.  An 8-bit cache is
// staged as it is and widened to f16 (exact) between shared memory and the tensor cores.
//
// The weights are rounded to the 16 bits that the second product takes, bf16 or, beside an 8-bit cache, f16; the sum beneath the line is
// that of the unrounded ones.  At 131072 tokens that brings the result from 1.66e-3 of its norm (its own rounding to bf16) to 1.76e-3; two
// halves of a weight would double the second product.
//
// What bounds it.  Long caches: HBM.  Twelve warps per SM with 8 KB on the way each are enough; more bytes in flight only let some
// SMs have more of the bandwidth than others, and the launch waits for the others (us, 8 heads x 131072 tokens / x 8
// sequences of 32768 / 8-bit; bytes 81.8 / 163.5 / 40.9, 81.8): eight warps with 24 KB each 94.6 / 171 / 59.4, 101; with 16 KB
// 89.9 / 170 / 55.5, 99.6; twelve with 8 KB 82.8 / 161 / 46.5, 86; sixteen (128 registers) 93.6 / 168 / 53.6, 94.2.  Short ones: a chain of waits
// (us in a launch on 8 heads x 300 tokens, 5.9 in all): the previous launch's end seen 1.1, lengths 0.6, page ids and copies issued
// 0.9, rows there 0.4, a tile and the warps' merge 1.1, ticket 0.9, join 1.2.  Between them both (8 heads x 8192 tokens: 12.3, bytes 5.1).
//
// A tile's rows behind the sequence's end hold anything: their scores are replaced, not added to, and their V rows are
// cleared in the fragments, since zero times NaN is NaN.
#include "paged_tiles.cuh"
#include "trace.cuh"

namespace sagekv {

constexpr int kPaWarps = 6;
constexpr int kPaThreads = kPaWarps * 32;
constexpr int kPaRingBytes = 2 * kSlotBytes;        // per warp: one stage of bf16 tiles, or two of 8-bit ones
constexpr int kPaHeadStride = kHeadDim + 4;         // floats between the heads of a warp's result: the 32 lanes of a store fall into 32 banks
constexpr int kPaPairCost = 2;                      // places of the list in front of a pair's units: what a change of pair costs a CTA, in units
constexpr int kPaWholeUnits = 2;                    // pairs that are this short in the mean are not cut where there are CTAs to spare
constexpr int kPaRounds = 3;                        // a pair's parts are joined in groups beyond so many rounds of one CTA's warps
constexpr int kPaMaxStages = 2;

struct PaShared {
  unsigned char ring[kPaWarps][kPaRingBytes];           // boxes with the 128-byte swizzle: 1024-byte boundaries
  float o[kPaWarps][kMaxGroup * kPaHeadStride];         // results of the warps
  float2 ml[kPaWarps][kMaxGroup];                       // (max, sum) of a warp's tiles
  unsigned long long bar[kPaWarps][kPaMaxStages];
  int start[2];                                         // where my range begins (many sequences): sequence, where its places begin
  int arrived;                                          // parts of a shared pair that had arrived before mine
};
static_assert(kPagedCtasPerSm * (sizeof(PaShared) + 1024) <= 228 * 1024, "they fit on an SM together");

// tokens of a sequence: what the caller gave, cut to what the table can hold
__device__ __forceinline__ int tokens_of(const PagedView &c, int seq) {
  const int len = seq < c.n_seqs ? c.seq_lens[seq] : 0;
  const int most = c.max_pages * c.page_size;
  return len < 0 ? 0 : min(len, most);
}

// The lengths of 32 sequences in a row, one per lane of a warp: what moves through the list in order reads memory once
// per 32 sequences.  All lanes call with the same sequence.
struct PaLengths {
  int base, mine;
  __device__ __forceinline__ void load(const PagedView &c, int seq, int lane) {
    base = seq;
    mine = tokens_of(c, seq + lane);
  }
  __device__ __forceinline__ int of(const PagedView &c, int seq, int lane) {
    if (seq - base >= 32) load(c, seq, lane);
    return __shfl_sync(0xffffffffu, mine, seq - base);
  }
};

// A place in the list of units: unit `unit` of head `head` of sequence `seq`, which has `len` tokens; `base` is the place of
// the pair's first unit in the list.
struct PaCursor {
  int seq, head, len, unit;
  uint32_t base;
  __device__ __forceinline__ int tiles() const { return (len + 15) >> 4; }
  __device__ __forceinline__ int units() const { return (len + 16 * kPaWarps - 1) / (16 * kPaWarps); }
  __device__ __forceinline__ void next_pair(const PagedView &c, int H_kv, PaLengths &lens, int lane) {
    base += (uint32_t)units() + kPaPairCost;
    unit = 0;
    if (++head < H_kv) return;
    head = 0;
    do len = lens.of(c, ++seq, lane);
    while (len == 0 && seq < c.n_seqs);
  }
};
// places in the list that the pairs of a sequence take, per head
__device__ __forceinline__ int places_of(int len) { return len > 0 ? (len + 16 * kPaWarps - 1) / (16 * kPaWarps) + kPaPairCost : 0; }

// Joins `count` results of a shared pair, those of its parts base, base + step, ...: each warp takes every kPaWarps-th, kParts of up to
// kHeads heads at a time with all their loads in flight; what it has goes where a warp's result of tiles does.  (Part 0 lies in
// slot 1 of its CTA, the others in slot 0 of theirs; part_0: slot 0 of part 0's CTA.)
// (us from the last ticket to the end, 4 / 10 / 22 / 32 / 37 parts of four heads: 1.2 / 1.4 / 1.7 / 2.5 / 2.2.  A thread per four columns of
// a head going through sixteen parts at a time: 1.2 at 2 parts, 1.7 at 8, 3.1 at 29, 3.7 at 37.  Six parts at a time instead of four
// cost registers and with them the loop over the tiles: 8-bit, 8 x 32768 tokens 86.6 -> 90.2)
template <int kParts, int kHeads>
__device__ __forceinline__ void join_parts(const PagedAttnParams &p, const float *part_0, int base, int step, int count, int G, int warp, int lane,
                                           float *o_to, float2 *ml_to) {
  static_assert(kParts * kHeads <= 32 && (kHeads & (kHeads - 1)) == 0, "a lane per part and head");
  const int u_mine = lane / kHeads, h_mine = lane & (kHeads - 1);   // the lane of part u and head h works out its weight
  float M = -INFINITY, l = 0.f;                              // of head h_mine
  float4 o[kHeads];
#pragma unroll
  for (int h = 0; h < kHeads; ++h) o[h] = make_float4(0.f, 0.f, 0.f, 0.f);
  const int part_floats = paged_part_floats(G);
  auto part_of = [&](int k) {
    const int i = base + k * step;
    return part_0 + (int64_t)(2 * i + (i == 0 ? 1 : 0)) * part_floats;
  };
  auto in_scratch = [&](int k) {
    return SAGEKV_OK_INDEX(p.c.status, part_of(k) >= p.partials && part_of(k) + part_floats <= p.partials + (int64_t)p.most_ctas * 2 * part_floats);
  };
  for (int i0 = warp; i0 < count; i0 += kPaWarps * kParts) {
    float2 ml = make_float2(-INFINITY, 0.f);
    const int i_mine = i0 + u_mine * kPaWarps;
    if (u_mine < kParts && i_mine < count && h_mine < G && in_scratch(i_mine))
      ml = __ldcg(reinterpret_cast<const float2 *>(part_of(i_mine) + G * kHeadDim + 2 * h_mine));
    float4 v[kParts][kHeads];
#pragma unroll
    for (int u = 0; u < kParts; ++u) {
      const float *from = part_of(i0 + u * kPaWarps) + lane * 4;
#pragma unroll
      for (int h = 0; h < kHeads; ++h) {
        v[u][h] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i0 + u * kPaWarps < count && h < G && in_scratch(i0 + u * kPaWarps)) v[u][h] = __ldcg(reinterpret_cast<const float4 *>(from + h * kHeadDim));
      }
    }
    float top = fmaxf(M, ml.x);
#pragma unroll
    for (int x = kHeads; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
    const float f = ml.x == top ? 1.f : fast_exp2(ml.x - top), back = M == top ? 1.f : fast_exp2(M - top);   // (equal also where both are infinite)
    float sum = ml.y * f;
#pragma unroll
    for (int x = kHeads; x < 32; x <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
    l = l * back + sum;
    M = top;
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
      const float bk = __shfl_sync(0xffffffffu, back, h);
      o[h].x *= bk; o[h].y *= bk; o[h].z *= bk; o[h].w *= bk;
#pragma unroll
      for (int u = 0; u < kParts; ++u) {
        const float fu = __shfl_sync(0xffffffffu, f, u * kHeads + h);
        o[h].x += v[u][h].x * fu; o[h].y += v[u][h].y * fu; o[h].z += v[u][h].z * fu; o[h].w += v[u][h].w * fu;
      }
    }
  }
#pragma unroll
  for (int h = 0; h < kHeads; ++h)
    if (h < G) *reinterpret_cast<float4 *>(o_to + h * kPaHeadStride + lane * 4) = o[h];
  if (lane < G) ml_to[lane] = make_float2(M, l);
}

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

  SAGEKV_TRACE_BEGIN
  SAGEKV_STAMP(0);
  const uint32_t ring = smem_u32(&sh.ring[warp][0]), bars = smem_u32(&sh.bar[warp][0]);
  if (lane == 0) {
#pragma unroll
    for (int s = 0; s < kStages; ++s) mbar_init(bars + 8u * s, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
  }
  __syncwarp();
  wait_for_predecessor();
  SAGEKV_STAMP(1);

  // ---- my range of the list: [lo, lo + n), which begins in sequence start_seq, whose places begin at start_before ----
  const int most_tokens = p.c.max_pages * p.c.page_size;
  const uint32_t n_ctas = gridDim.x;
  uint32_t total, per_cta, lo;
  auto cut = [&](uint32_t least) {                           // (all fits 31 bits: the host has checked the most the tables can hold)
    const uint32_t all = total * (uint32_t)p.H_kv;
    per_cta = max(all > 0u ? (all - 1u) / n_ctas + 1u : 0u, least);
    lo = min((uint32_t)blockIdx.x * per_cta, all);
    return (int)min(per_cta, all - lo);
  };
  int n, start_seq = 0, start_before = 0;
  PaLengths lens;
  if (p.c.n_seqs <= 32) {                                    // every warp by itself
    const int given = lane < p.c.n_seqs ? p.c.seq_lens[lane] : 0;
    if (given < 0 || given > most_tokens) atomicOr(p.c.status, kStatusBounds);
    lens.base = 0;
    lens.mine = min(max(given, 0), most_tokens);
    const int mine = places_of(lens.mine);
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    total = (uint32_t)__shfl_sync(0xffffffffu, incl, 31);
    // A second CTA per pair costs a ticket and the join, 2.1 us, and saves half of the steps of 1 us (8 heads x 100 tokens 4.9 / 5.9 us
    // whole / cut, x 300 tokens 6.9 / 5.9).
    constexpr uint32_t kWhole = kPaPairCost + kPaWholeUnits;
    n = cut(total <= kWhole * (uint32_t)__popc(__ballot_sync(0xffffffffu, mine > 0)) ? kWhole : 1u);
    if (n > 0) {
      start_seq = __ffs(__ballot_sync(0xffffffffu, lo < (uint32_t)incl * p.H_kv)) - 1;
      start_before = __shfl_sync(0xffffffffu, incl - mine, start_seq) * p.H_kv;
    }
  } else {                                                   // a block-wide scan, every thread over some sequences in a row
    const int per_thread = (p.c.n_seqs + kPaThreads - 1) / kPaThreads;
    const int s0 = min(tid * per_thread, p.c.n_seqs), s1 = min(s0 + per_thread, p.c.n_seqs);
    int mine = 0;
    for (int s = s0; s < s1; ++s) {
      const int given = p.c.seq_lens[s];
      if (given < 0 || given > most_tokens) atomicOr(p.c.status, kStatusBounds);
      mine += places_of(min(max(given, 0), most_tokens));
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
    int before = incl - mine;
    total = 0u;
#pragma unroll
    for (int w = 0; w < kPaWarps; ++w) {
      if (w < warp) before += warp_total[w];
      total += (uint32_t)warp_total[w];
    }
    n = cut(1u);
    if (lo >= (uint32_t)before * p.H_kv && lo < (uint32_t)(before + mine) * p.H_kv) {   // the range begins in one of this thread's sequences
      int at = before, s = s0;
      for (int t; at + (t = places_of(tokens_of(p.c, s))) <= (int)(lo / p.H_kv); ++s) at += t;
      sh.start[0] = s;
      sh.start[1] = at * p.H_kv;
    }
    __syncthreads();
    if (n > 0) {
      start_seq = sh.start[0];
      start_before = sh.start[1];
    }
    lens.load(p.c, start_seq, lane);
  }

  SAGEKV_STAMP_AFTER(2, (float)n);

  // ---- requests ----
  const uint32_t hi = lo + (uint32_t)max(n, 0);
  PaCursor begin, next;                                      // where my range begins; my next tile to request
  PaLengths ahead = lens;
  bool more = false;                                         // there is one
  int ids = -1, ids_unit = 0;                                // page ids of the warp's tiles in 32 units of the pair, from ids_unit on
  int next_page = -1, next_slot = 0;
  uint32_t absent = 0u;                                      // stages whose page id is none: nothing is on its way
  uint64_t stream_policy;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(stream_policy));
  auto look_up = [&](bool moved) {                           // settles on the next tile, if there is one, and finds its page
    while (next.unit >= next.units() || next.unit * kPaWarps + warp >= next.tiles()) {   // (a pair's last unit may lack my tile)
      next.next_pair(p.c, p.H_kv, ahead, lane);
      moved = true;
      if (next.base >= hi) break;
    }
    more = next.base + (uint32_t)next.unit < hi && next.seq < p.c.n_seqs;
    if (!more) return;
    if (moved || next.unit - ids_unit >= 32) {
      ids_unit = next.unit;
      const int tile = (next.unit + lane) * kPaWarps + warp;
      const int entry = page_of(tile << 4, p.c.page_size, p.c.page_magic);
      ids = tile < next.tiles() && SAGEKV_OK_ENTRY(p.c, next.seq, entry) ? p.c.table[(int64_t)next.seq * p.c.table_stride + entry] : -1;
    }
    const int first = (next.unit * kPaWarps + warp) << 4;
    next_slot = first - page_of(first, p.c.page_size, p.c.page_magic) * p.c.page_size;
    next_page = __shfl_sync(0xffffffffu, ids, next.unit - ids_unit);
  };
  auto request = [&](int s) {
    if (!more) return;
    const uint32_t bar = bars + 8u * s;
    if (next_page >= 0 && next_page < p.c.n_pages && SAGEKV_OK_TILE(p.c, next_slot, next.head, p.H_kv)) {
      absent &= ~(1u << s);
      if (lane == 0) mbar_expect_tx(bar, kStageBytes);
      __syncwarp();
      constexpr int kBoxes = kE4m3 ? 2 : 4;                  // 16 rows of 128 bytes each
      if (lane < kBoxes)
        tensor_copy_4d(ring + (uint32_t)(s * kStageBytes + lane * kHalfBytes), lane < kBoxes / 2 ? &map_k : &map_v,
                         kE4m3 ? 0 : (lane & 1) * 64, next_slot, next.head, next_page, bar, stream_policy);
    } else {
      absent |= 1u << s;
      if (lane == 0) {
        mbar_arrive(bar);
        atomicOr(p.c.status, kStatusBounds);
      }
    }
    ++next.unit;
    look_up(false);
  };
  if (n > 0) {
    begin.seq = start_seq;
    begin.len = ahead.of(p.c, start_seq, lane);
    const uint32_t into = lo - (uint32_t)start_before, places = (uint32_t)places_of(begin.len);
    begin.head = (int)(into / places);
    begin.base = (uint32_t)start_before + (uint32_t)begin.head * places + kPaPairCost;
    begin.unit = max((int)(lo - begin.base), 0);             // (the range may begin in the places in front of the pair)
    next = begin;
    look_up(true);
#pragma unroll
    for (int s = 0; s < kStages; ++s) request(s);
  }
  SAGEKV_STAMP(3);

  // ---- sequences without tokens ----
  for (int s = blockIdx.x; s < p.c.n_seqs; s += n_ctas) {
    if ((p.c.n_seqs <= 32 ? __shfl_sync(0xffffffffu, lens.mine, s) : tokens_of(p.c, s)) > 0) continue;
    for (int i = tid; i < p.H_q * (kHeadDim / 8); i += kPaThreads) st_v4(p.out + (int64_t)s * p.H_q * kHeadDim + i * 8, make_uint4(0u, 0u, 0u, 0u));
    if (p.lse != nullptr)
      for (int i = tid; i < p.H_q; i += kPaThreads) p.lse[(int64_t)s * p.H_q + i] = -INFINITY;
  }

  if (n > 0) {
    // fragment addresses within a stage
    const int mi = lane >> 3, l8 = lane & 7;
    uint32_t k_off[8], v_off[8];
    k_fragment_offsets<kE4m3>(lane, k_off);
#pragma unroll
    for (int j = 0; j < (kE4m3 ? 4 : 8); ++j)
      v_off[j] = kTileBytes + (kE4m3 ? k_off[j] : tile_offset((mi >> 1) * 8 + l8, 2 * j + (mi & 1)));
    const bool in0 = h0 < p.G, in1 = h1 < p.G;

    bool timed_out = false;
    int stage = 0;
    uint32_t phase = 0;
    PaCursor at = begin;                                     // the pair being worked on
    while (at.base < hi && at.seq < p.c.n_seqs) {
      const int tiles = at.tiles(), unit_end = min(at.units(), (int)(hi - at.base));
      uint32_t qb[8][2];
      float mult0, mult1;
      // (in the checked build a pair that is none is worked on as pair 0, and its result left out)
      const bool a_pair = SAGEKV_OK_INDEX(p.c.status, at.seq < p.c.n_seqs && at.head < p.H_kv && at.seq * p.H_kv + at.head < p.n_tickets);
      const int q_seq = a_pair ? at.seq : 0, q_head = a_pair ? at.head : 0;
      load_queries<kE4m3>(p.q + (int64_t)q_seq * p.q_stride + q_head * p.G * kHeadDim, p.G, p.c.k_scale, q_head, p.scale_log2, lane, qb, mult0, mult1);

      float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;   // the maxima are kept kWeightShift below the scores'
      float acc[8][4];
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;

      for (int tile = at.unit * kPaWarps + warp; tile < min(tiles, unit_end * kPaWarps); tile += kPaWarps) {
        const uint32_t tb = ring + (uint32_t)(stage * kStageBytes);
        if (!mbar_wait(bars + 8u * stage, phase)) timed_out = true;
        if (at.base + at.unit <= lo + kPaPairCost && tile == at.unit * kPaWarps + warp) SAGEKV_STAMP(4);
        if (!((absent >> stage) & 1u)) {
          // ---- S = K Q^T; V's fragments on their way meanwhile ----
          float sv[4];
          score_tile<kE4m3>(tb, k_off, qb, mult0, mult1, sv);
          uint32_t fa[4], va[8][4];
          if (kE4m3) {
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
            for (int j = 0; j < 8; ++j) ldmatrix_x4_trans(tb + v_off[j], va[j][0], va[j][1], va[j][2], va[j][3]);
          }
          // ---- softmax weights ----
          const int left = at.len - (tile << 4);             // tokens of the sequence from this tile's first on
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
        }
        // Every lane has its fragments, and has seen this phase of the barrier: the stage may be refilled.  (Where the next tile's page is
        // none, lane 0 completes the next phase at once: a lane that still polled for this one would then never see it.)
        __syncwarp();
        request(stage);
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
      }

      SAGEKV_STAMP_AFTER(5, acc[0][0] + acc[7][3]);
      // ---- the pair (or my part of it) is done: merge the warps ----
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
      const int cta_first = (int)(at.base / per_cta), cta_last = (int)((at.base + (uint32_t)at.units() - 1u) / per_cta);
      const bool whole = cta_first == cta_last;
      const int64_t row0 = (int64_t)at.seq * p.H_q + at.head * p.G;   // the pair's first row of out and lse
      const float v_scale = kE4m3 && p.c.v_scale != nullptr ? p.c.v_scale[q_head] : 1.f;
      auto finish = [&](int h, int col, float4 o, float M, float l) {
        if (!SAGEKV_OK_INDEX(p.c.status, at.seq < p.c.n_seqs && (at.head + 1) * p.G <= p.H_q && h < p.G)) return;
        const float inv = l == 0.f ? 0.f : v_scale / l;
        *reinterpret_cast<uint2 *>(p.out + (row0 + h) * kHeadDim + col) = make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
        if (p.lse != nullptr && col == 0) p.lse[row0 + h] = l == 0.f ? -INFINITY : (M + log2f(l)) * kLn2;
      };
      const int part_floats = paged_part_floats(p.G);
      // the warps' results (of tiles, or of parts) as one
      auto merge_warps = [&](auto emit) {
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
          emit(h, col, o, M, l);
        }
      };
      if (whole) {
        merge_warps(finish);
      } else {
        auto leave = [&](float *part) {
          if (!SAGEKV_OK_INDEX(p.c.status, part >= p.partials && part + part_floats <= p.partials + (int64_t)p.most_ctas * 2 * part_floats)) return;
          merge_warps([&](int h, int col, float4 o, float M, float l) {
            *reinterpret_cast<float4 *>(part + h * kHeadDim + col) = o;
            if (col == 0) *reinterpret_cast<float2 *>(part + p.G * kHeadDim + 2 * h) = make_float2(M, l);
          });
        };
        // slot 0 of a CTA whose range begins inside the pair, slot 1 of the one where the pair begins
        leave(p.partials + ((int64_t)blockIdx.x * 2 + (cta_first == (int)blockIdx.x ? 1 : 0)) * part_floats);
        SAGEKV_STAMP(6);
        // The last CTA of the pair joins its parts; of very many (few pairs on the whole device) the last of each group of
        // neighbours first joins the group, its result taking the place of the group's first part (one head of eight queries x
        // 131072 tokens 34.1 -> 18.2 us, two x 32768 19.7 -> 14.5).
        const int parts = cta_last - cta_first + 1, group_size = (p.G <= 4 ? 4 : 2) * kPaWarps;
        float *const part_0 = p.partials + (int64_t)cta_first * 2 * part_floats;
        bool grouped = parts > kPaRounds * group_size;
        const int group = ((int)blockIdx.x - cta_first) / group_size;
        int base = grouped ? group * group_size : 0, step = 1, count = grouped ? min(group_size, parts - base) : parts;
        int32_t *const pair_ticket = p.tickets + (int64_t)at.seq * p.H_kv + at.head;
        int32_t *ticket = grouped ? p.group_tickets + 2 * (cta_first + base) + (base == 0 ? 1 : 0) : pair_ticket;
        for (;;) {
          __syncthreads();
          if (!SAGEKV_OK_INDEX(p.c.status, (ticket >= p.tickets && ticket < p.tickets + p.n_tickets) ||
                                               (ticket >= p.group_tickets && ticket < p.group_tickets + 2 * p.most_ctas)))
            break;
          if (tid == 0)                                      // (behind the barrier its release stands for the whole block, and so does its acquire)
            asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(sh.arrived) : "l"(ticket) : "memory");
          __syncthreads();
          SAGEKV_STAMP(7);
          if (sh.arrived != count - 1) break;                // else every other part is in scratch
          if (tid == 0) *ticket = 0;
          // (beside an 8-bit cache fewer at a time: the loop over the tiles needs the registers, 8 x 32768 tokens 88.7 -> 86.1 us)
          if (p.G <= 4) join_parts<kE4m3 ? 3 : 4, 4>(p, part_0, base, step, count, p.G, warp, lane, sh.o[warp], sh.ml[warp]);
          else join_parts<kE4m3 ? 1 : 2, 8>(p, part_0, base, step, count, p.G, warp, lane, sh.o[warp], sh.ml[warp]);
          __syncthreads();
          if (!grouped) {
            merge_warps(finish);
            break;
          }
          leave(part_0 + (int64_t)(2 * base + (base == 0 ? 1 : 0)) * part_floats);
          grouped = false;
          base = 0; step = group_size; count = (parts + group_size - 1) / group_size;
          ticket = pair_ticket;
        }
      }
      SAGEKV_STAMP(8);
      at.next_pair(p.c, p.H_kv, lens, lane);
    }
    if (timed_out) atomicOr(p.c.status, kStatusWaitTimeout);
  }
#if defined(SAGEKV_TRACE)
  for (int i = 4; i < 9; ++i)                                // (a CTA without tiles, or with whole pairs alone, has not been everywhere)
    if (trace_t[i] < trace_t[i - 1]) trace_t[i] = trace_t[i - 1];
#endif
  SAGEKV_STAMP(9);
  SAGEKV_TRACE_END(p.q);
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
  if (!make_page_map(&map_k, p.c.k, p.c, p.H_kv, e4m3) || !make_page_map(&map_v, p.c.v, p.c, p.H_kv, e4m3)) return cudaErrorInvalidValue;
  const int64_t most_units = ((int64_t)p.c.max_pages * p.c.page_size + 16 * kPaWarps - 1) / (16 * kPaWarps);   // of a sequence that fills its table
  int64_t ctas = p.c.n_seqs * p.H_kv * (most_units + kPaPairCost);
  if (ctas > paged_attn_max_ctas(n_sm)) ctas = paged_attn_max_ctas(n_sm);
  if (ctas < 1) ctas = 1;
  return launch_next(e4m3 ? paged_attn_kernel<true> : paged_attn_kernel<false>, dim3((unsigned)ctas), kPaThreads, sizeof(PaShared), stream, 0,
                     p, map_k, map_v);
}

}  // namespace sagekv

SAGEKV_TRACE_READER(sagekv_trace_read_paged)
