// The context behind the C interface, for the files that implement its entry points.
#pragma once

#include "common.cuh"
#include "paged.cuh"

struct sagekv_ctx {
  sagekv_shape shape;
  int G;
  int64_t max_ctx;
  int32_t max_len;
  int device;               // the device the context was created on; every call must find it current
  const sagekv::DeviceInfo *dev;    // that device's one-time set-up
  float scale;
  float2 *score_partials;   // [B*H_q, max_chunks]
  int max_chunks;           // ceil(max_ctx / kScoreChunk), or the CTAs per head that the scores of short paged sequences are spread over
  float *decode_partials;   // [B*H_kv, max_splits (clusters per head), kPartialStride]
  int max_splits;
  float *paged_partials;    // [grid of the paged attention][2][paged_part_floats(G)]: what a CTA leaves of heads that it shares (behind decode_partials)
  int32_t *paged_tickets;   // [B*H_kv] + [grid of the paged attention][2] arrival counters of its pairs and groups, zero between launches (behind tickets)
  int32_t *tickets;         // [B*H_kv + 1], zero between launches; the status word and the selection's ready word follow them
  int32_t *status;          // one int32: kStatus* bits raised by the kernels
  int last_cuda_error;
  int overlap;              // 0, 1 or 2: see sagekv_set_overlap
  int select_overlap;       // 0, 1 or 2: see sagekv_set_select_overlap
  bool select_ahead;        // the last select call releases its successor before it has waited for its own predecessor
  int decode_variant;       // 0, 1 or 2: see sagekv_set_decode_variant
  int hint;                 // 0, 1, 2: see sagekv_set_select_hint
  int32_t hint_k;
  int group_mode;           // 0: a selection per query head (the paper's), 1: one per KV head from pooled scores
};

namespace sagekv {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline int cuda_fail(sagekv_ctx *ctx, cudaError_t e) {
  if (ctx) ctx->last_cuda_error = (int)e;
  return SAGEKV_ERR_CUDA;
}

// false: another device is current than the one the context belongs to
inline bool on_own_device(const sagekv_ctx *ctx) {
  int cur = -1;
  return cudaGetDevice(&cur) == cudaSuccess && cur == ctx->device;
}

}  // namespace sagekv
