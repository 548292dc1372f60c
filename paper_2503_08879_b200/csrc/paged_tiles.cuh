// What the kernels that stream a paged cache share: 16-token tiles of K (and V) brought in by tensor copies, and the product of
// a staged K tile with a KV head's queries.
#pragma once

#include "paged.cuh"
#include "tiles.cuh"

namespace sagekv {

__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// byte offset of 16-byte piece `piece` (0..7) of row `row` in a staged tile of 128-byte rows
__device__ __forceinline__ uint32_t tile8_offset(int row, int piece) { return (uint32_t)(row * 128 + ((piece ^ (row & 7)) << 4)); }

// Addresses of a lane's matrix rows in a staged K tile, for the fragments of score_tile.
template <bool kE4m3>
__device__ __forceinline__ void k_fragment_offsets(int lane, uint32_t (&k_off)[8]) {
  const int mi = lane >> 3, l8 = lane & 7;
#pragma unroll
  for (int j = 0; j < (kE4m3 ? 4 : 8); ++j)
    k_off[j] = kE4m3 ? tile8_offset((mi & 1) * 8 + l8, 2 * j + (mi >> 1)) : tile_offset((mi & 1) * 8 + l8, 2 * j + (mi >> 1));
}

// The B fragments of a KV head's queries (head g of the lane (g, c), zeros for g >= G) as score_tile takes them: bf16 dims
// 16j + 2c, +1 and 16j + 8 + 2c, +1, or f16 dims 16j + 4c .. + 3 beside an 8-bit cache; and what brings a
// score of heads 2c and 2c + 1 to log2 units.  q: the first of the heads.
template <bool kE4m3>
__device__ __forceinline__ void load_queries(const uint16_t *q, int G, const float *k_scale, int kv_head, float scale_log2, int lane,
                                             uint32_t (&qb)[8][2], float &mult0, float &mult1) {
  const int g = lane >> 2, c = lane & 3;
  const uint16_t *q_row = q + min(g, G - 1) * kHeadDim;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    qb[j][0] = qb[j][1] = 0u;
    if (g < G) {
      if (kE4m3) {
        const uint2 v = *reinterpret_cast<const uint2 *>(q_row + 16 * j + 4 * c);
        qb[j][0] = v.x; qb[j][1] = v.y;
      } else {
        qb[j][0] = *reinterpret_cast<const uint32_t *>(q_row + 16 * j + 2 * c);
        qb[j][1] = *reinterpret_cast<const uint32_t *>(q_row + 16 * j + 8 + 2 * c);
      }
    }
  }
  mult0 = mult1 = scale_log2;
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
    const float base = k_scale != nullptr ? scale_log2 * k_scale[kv_head] : scale_log2;
    mult0 = base * power_of_two(-__shfl_sync(0xffffffffu, e, 8 * c));
    mult1 = base * power_of_two(-__shfl_sync(0xffffffffu, e, 8 * c + 4));
  }
}

// S = K Q^T of the tile staged at tb, 16 tokens x 8 heads in four accumulator chains: lane (g, c) gets tokens g (0, 1) and g + 8
// (2, 3) of heads 2c (0, 2) and 2c + 1 (1, 3), in log2 units.  An 8-bit tile is widened to f16 on the way: a lane's 32-bit word
// holds dims 4c .. + 3 of its row, whose halves fill the k slots that the query's halves do.
template <bool kE4m3>
__device__ __forceinline__ void score_tile(uint32_t tb, const uint32_t (&k_off)[8], const uint32_t (&qb)[8][2], float mult0, float mult1,
                                           float (&sv)[4]) {
  float ch[4][4];
#pragma unroll
  for (int j = 0; j < 4; ++j) ch[j][0] = ch[j][1] = ch[j][2] = ch[j][3] = 0.f;
  uint32_t fa[4];
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
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      ldmatrix_x4(tb + k_off[j], fa[0], fa[1], fa[2], fa[3]);
      float(&d)[4] = ch[j & 3];
      mma_bf16_16816(d[0], d[1], d[2], d[3], fa[0], fa[1], fa[2], fa[3], qb[j][0], qb[j][1]);
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) sv[e] = ((ch[0][e] + ch[1][e]) + (ch[2][e] + ch[3][e])) * (e & 1 ? mult1 : mult0);
}

// [n_pages, H_kv, page_size, 128] through the cache's strides, boxes of 16 rows x 128 bytes with the 128-byte swizzle
inline bool make_page_map(CUtensorMap *map, uint8_t *base, const PagedView &c, int H_kv, bool e4m3) {
  EncodeTiledFn enc = encode_tiled_fn();
  if (enc == nullptr) return false;
  const cuuint64_t size = e4m3 ? 1 : 2;
  const cuuint64_t dims[4] = {(cuuint64_t)kHeadDim, (cuuint64_t)c.page_size, (cuuint64_t)H_kv, (cuuint64_t)c.n_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)c.token_stride * size, (cuuint64_t)c.head_stride * size, (cuuint64_t)c.page_stride * size};
  const cuuint32_t box[4] = {e4m3 ? 128u : 64u, 16, 1, 1};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  return enc(map, e4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, base, dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace sagekv
