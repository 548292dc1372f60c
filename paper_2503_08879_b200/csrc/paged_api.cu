// The C interface of the paged cache (include/sagekv.h): rotary plans, argument checks on the host, then the launches.
#include <math.h>

#include "context.cuh"

using namespace sagekv;

namespace {

constexpr int kPlanMark = 0x524f5045;   // sagekv_rope_plan::reserved of a plan that one of the two calls has filled
constexpr double kTwoPi = 6.283185307179586476925286766559;

bool rotary_ok(int32_t r) { return r >= 16 && r <= kHeadDim && r % 16 == 0; }
bool plan_ok(const sagekv_rope_plan *p) { return p->reserved == kPlanMark && rotary_ok(p->rotary_dim); }

RopeArgs rope_args(const sagekv_rope_plan *plan) {
  RopeArgs r = {};
  if (plan == nullptr) return r;
  for (int i = 0; i < kHeadDim / 2; ++i) r.turns[i] = plan->turns[i];
  r.rotary_dim = plan->rotary_dim;
  r.interleaved = plan->interleaved != 0 ? 1 : 0;
  r.amplitude = plan->amplitude;
  return r;
}

bool rows_aligned(const sagekv_rows &r) { return r.token_stride % 8 == 0 && r.head_stride % 8 == 0; }
// a stride that is never stepped along may be anything
bool rows_apart(const sagekv_rows &r, int64_t tokens, int32_t heads) {
  return (tokens <= 1 || r.token_stride >= kHeadDim) && (heads <= 1 || r.head_stride >= kHeadDim);
}

PagedView view_of(const sagekv_ctx *ctx, const sagekv_paged_cache *c) {
  PagedView v;
  v.k = static_cast<uint8_t *>(c->k_pages);
  v.v = static_cast<uint8_t *>(c->v_pages);
  v.page_stride = c->page_stride;
  v.head_stride = c->head_stride;
  v.token_stride = c->token_stride;
  v.table = c->block_table;
  v.table_stride = c->table_stride;
  v.seq_lens = c->seq_lens;
  v.k_scale = c->k_scale;
  v.v_scale = c->v_scale;
  v.status = ctx->status;
  v.n_seqs = c->n_seqs;
  v.max_pages = c->max_pages;
  v.n_pages = c->n_pages;
  v.page_size = c->page_size;
  v.page_magic = page_magic(c->page_size);
  return v;
}

int done(sagekv_ctx *ctx, cudaError_t e) { return e == cudaSuccess ? SAGEKV_OK : cuda_fail(ctx, e); }

}  // namespace

extern "C" {

int sagekv_paged_check(const sagekv_shape *shape, const sagekv_paged_cache *c) {
  if (shape == nullptr || c == nullptr || c->k_pages == nullptr || c->v_pages == nullptr) return SAGEKV_ERR_INVALID;
  if (c->n_pages < 1 || c->page_size < 1 || c->max_pages < 0 || c->n_seqs < 0 ||
      (c->dtype != SAGEKV_CACHE_BF16 && c->dtype != SAGEKV_CACHE_E4M3) || c->table_stride < c->max_pages ||
      (c->block_table == nullptr && c->max_pages > 0 && c->n_seqs > 0) || c->token_stride < kHeadDim || c->head_stride < kHeadDim ||
      c->page_stride < kHeadDim || (c->dtype == SAGEKV_CACHE_BF16 && (c->k_scale != nullptr || c->v_scale != nullptr)))
    return SAGEKV_ERR_INVALID;
  const int64_t size = c->dtype == SAGEKV_CACHE_E4M3 ? 1 : 2, step = 16 / size;
  const int64_t most_bytes = ((int64_t)1 << 40) / size;
  if (c->page_size % 16 != 0 || c->n_seqs > shape->batch || (int64_t)c->max_pages * c->page_size > (int64_t)1 << 30 ||
      c->page_stride >= most_bytes || c->head_stride >= most_bytes || c->token_stride >= most_bytes)
    return SAGEKV_ERR_UNSUPPORTED;
  // (the first two factors together are below 2^31: a sequence's tiles fit 2^26, its heads 65535)
  const int64_t tiles = (int64_t)c->max_pages * (c->page_size / 16) * shape->n_kv_heads;
  if (c->n_seqs > 0 && tiles > 0x7fffffff / c->n_seqs) return SAGEKV_ERR_UNSUPPORTED;
  if (!aligned16(c->k_pages) || !aligned16(c->v_pages) || c->page_stride % step != 0 || c->head_stride % step != 0 || c->token_stride % step != 0)
    return SAGEKV_ERR_ALIGN;
  return SAGEKV_OK;
}

int64_t sagekv_paged_offset(const sagekv_paged_cache *c, int32_t page, int32_t head, int64_t position) {
  if (c == nullptr || c->page_size < 16 || c->page_size % 16 != 0 || head < 0 || position < 0 || position > 0x7fffffff) return SAGEKV_ERR_INVALID;
  const int entry = page_of((int)position, c->page_size, page_magic(c->page_size));
  const int64_t at = paged_row(page, c->n_pages, (int)position - entry * c->page_size, head, c->page_stride, c->head_stride, c->token_stride);
  return at < 0 ? SAGEKV_ERR_INVALID : at;
}

int sagekv_rope_plan_from(sagekv_rope_plan *plan, int32_t rotary_dim, int32_t interleaved, const double *inv_freq, float amplitude) {
  if (plan == nullptr || inv_freq == nullptr || !(amplitude >= 0.f) || !isfinite(amplitude)) return SAGEKV_ERR_INVALID;
  if (!rotary_ok(rotary_dim)) return SAGEKV_ERR_UNSUPPORTED;
  for (int i = 0; i < rotary_dim / 2; ++i)
    if (!(inv_freq[i] >= 0.0) || !isfinite(inv_freq[i])) return SAGEKV_ERR_INVALID;
  sagekv_rope_plan p = {};
  p.rotary_dim = rotary_dim;
  p.interleaved = interleaved != 0 ? 1 : 0;
  p.amplitude = amplitude;
  p.reserved = kPlanMark;
  for (int i = 0; i < rotary_dim / 2; ++i) {
    // whole revolutions per position change nothing; the fraction in two halves of 32 bits, so that none is rounded away
    const long double turns = (long double)inv_freq[i] / 6.283185307179586476925286766559005768L;
    const long double high = (turns - floorl(turns)) * 4294967296.0L, whole = floorl(high);
    const long double low = rintl((high - whole) * 4294967296.0L);             // up to 2^32: the carry goes into the upper half
    p.turns[i] = ((uint64_t)whole << 32) + (uint64_t)low;
  }
  *plan = p;
  return SAGEKV_OK;
}

int sagekv_rope_plan_init(sagekv_rope_plan *plan, int32_t rotary_dim, int32_t interleaved, double theta, const sagekv_rope_scaling *scaling,
                          double *inv_freq) {
  if (plan == nullptr || !(theta > 1.0) || !isfinite(theta)) return SAGEKV_ERR_INVALID;
  const int kind = scaling != nullptr ? scaling->kind : SAGEKV_ROPE_NONE;
  if (kind < SAGEKV_ROPE_NONE || kind > SAGEKV_ROPE_YARN) return SAGEKV_ERR_INVALID;
  if (kind != SAGEKV_ROPE_NONE && (!(scaling->factor >= 1.0) || !isfinite(scaling->factor))) return SAGEKV_ERR_INVALID;
  if (scaling != nullptr && (!(scaling->amplitude >= 0.0) || !isfinite(scaling->amplitude))) return SAGEKV_ERR_INVALID;
  if (kind >= SAGEKV_ROPE_BANDS && (!(scaling->low > 0.0) || !(scaling->high > scaling->low) || !isfinite(scaling->high) ||
                                    !(scaling->original_ctx > 0.0) || !isfinite(scaling->original_ctx)))
    return SAGEKV_ERR_INVALID;
  if (!rotary_ok(rotary_dim)) return SAGEKV_ERR_UNSUPPORTED;
  const double r = rotary_dim;
  const double factor = kind != SAGEKV_ROPE_NONE ? scaling->factor : 1.0;
  const double base = kind == SAGEKV_ROPE_BASE ? theta * pow(factor, r / (r - 2.0)) : theta;
  double f[kHeadDim / 2], amplitude = 1.0, lo = 0.0, hi = 0.0;
  if (kind == SAGEKV_ROPE_YARN) {
    lo = fmax(floor(r * log(scaling->original_ctx / (kTwoPi * scaling->high)) / (2.0 * log(theta))), 0.0);
    hi = fmin(ceil(r * log(scaling->original_ctx / (kTwoPi * scaling->low)) / (2.0 * log(theta))), r - 1.0);
    if (hi == lo) hi = lo + 0.001;
    amplitude = 0.1 * log(factor) + 1.0;
  }
  for (int i = 0; i < rotary_dim / 2; ++i) {
    f[i] = pow(base, -2.0 * i / r);
    if (kind == SAGEKV_ROPE_LINEAR) {
      f[i] /= factor;
    } else if (kind == SAGEKV_ROPE_BANDS) {
      const double turns = scaling->original_ctx * f[i] / kTwoPi;
      const double s = fmin(fmax((turns - scaling->low) / (scaling->high - scaling->low), 0.0), 1.0);
      f[i] = s * f[i] + (1.0 - s) * (f[i] / factor);
    } else if (kind == SAGEKV_ROPE_YARN) {
      const double ramp = fmin(fmax((i - lo) / (hi - lo), 0.0), 1.0);
      f[i] = ramp * (f[i] / factor) + (1.0 - ramp) * f[i];
    }
  }
  if (scaling != nullptr && scaling->amplitude > 0.0) amplitude = scaling->amplitude;
  const int code = sagekv_rope_plan_from(plan, rotary_dim, interleaved, f, (float)amplitude);
  if (code == SAGEKV_OK && inv_freq != nullptr)
    for (int i = 0; i < rotary_dim / 2; ++i) inv_freq[i] = f[i];
  return code;
}

int sagekv_rope(sagekv_ctx *ctx, const sagekv_rope_plan *plan, const void *x, sagekv_rows xs, int64_t n_tokens, int32_t n_heads,
                const int32_t *positions, void *out, sagekv_rows os, void *stream) {
  if (ctx == nullptr || plan == nullptr || !plan_ok(plan) || n_tokens < 0 || n_heads < 0) return SAGEKV_ERR_INVALID;
  if (n_tokens > 0x7fffffff || n_heads > kRopeMostHeads) return SAGEKV_ERR_UNSUPPORTED;
  if (!on_own_device(ctx)) return SAGEKV_ERR_DEVICE;
  if (n_tokens == 0 || n_heads == 0) return SAGEKV_OK;
  if (x == nullptr || out == nullptr || positions == nullptr || !rows_apart(xs, n_tokens, n_heads) || !rows_apart(os, n_tokens, n_heads))
    return SAGEKV_ERR_INVALID;
  if (!aligned16(x) || !aligned16(out) || !rows_aligned(xs) || !rows_aligned(os)) return SAGEKV_ERR_ALIGN;
  PagedAppendParams p = {};
  p.rope = rope_args(plan);
  p.c.status = ctx->status;
  p.q = static_cast<const uint16_t *>(x);
  p.q_out = static_cast<uint16_t *>(out);
  p.q_token = xs.token_stride;
  p.q_head = xs.head_stride;
  p.q_out_token = os.token_stride;
  p.q_out_head = os.head_stride;
  p.positions = positions;
  p.n_tokens = n_tokens;
  p.H_q = n_heads;
  return done(ctx, launch_rope(p, ctx->dev->n_sm, static_cast<cudaStream_t>(stream)));
}

int sagekv_paged_append(sagekv_ctx *ctx, const sagekv_paged_cache *cache, const void *k, const void *v, sagekv_rows kvs, int64_t n_tokens,
                        const int32_t *positions, const int32_t *seqs, const sagekv_rope_plan *plan, const void *q, sagekv_rows qs,
                        void *q_out, sagekv_rows qos, void *stream) {
  if (ctx == nullptr || n_tokens < 0 || (q == nullptr) != (q_out == nullptr) || (plan != nullptr && !plan_ok(plan))) return SAGEKV_ERR_INVALID;
  const int bad = sagekv_paged_check(&ctx->shape, cache);
  if (bad != SAGEKV_OK) return bad;
  if (n_tokens > 0x7fffffff) return SAGEKV_ERR_UNSUPPORTED;
  if (!on_own_device(ctx)) return SAGEKV_ERR_DEVICE;
  if (n_tokens == 0) return SAGEKV_OK;
  if (k == nullptr || v == nullptr || positions == nullptr || !rows_apart(kvs, n_tokens, ctx->shape.n_kv_heads) ||
      (q != nullptr && (!rows_apart(qs, n_tokens, ctx->shape.n_q_heads) || !rows_apart(qos, n_tokens, ctx->shape.n_q_heads))))
    return SAGEKV_ERR_INVALID;
  if (!aligned16(k) || !aligned16(v) || !rows_aligned(kvs) ||
      (q != nullptr && (!aligned16(q) || !aligned16(q_out) || !rows_aligned(qs) || !rows_aligned(qos))))
    return SAGEKV_ERR_ALIGN;
  PagedAppendParams p;
  p.rope = rope_args(plan);
  p.c = view_of(ctx, cache);
  p.k = static_cast<const uint16_t *>(k);
  p.v = static_cast<const uint16_t *>(v);
  p.q = static_cast<const uint16_t *>(q);
  p.q_out = static_cast<uint16_t *>(q_out);
  p.kv_token = kvs.token_stride;
  p.kv_head = kvs.head_stride;
  p.q_token = qs.token_stride;
  p.q_head = qs.head_stride;
  p.q_out_token = qos.token_stride;
  p.q_out_head = qos.head_stride;
  p.positions = positions;
  p.seqs = seqs;
  p.n_tokens = n_tokens;
  p.H_q = ctx->shape.n_q_heads;
  p.H_kv = ctx->shape.n_kv_heads;
  return done(ctx, launch_paged_append(p, cache->dtype, ctx->dev->n_sm, static_cast<cudaStream_t>(stream)));
}

int sagekv_paged_attn(sagekv_ctx *ctx, const void *q, int64_t q_stride, const sagekv_paged_cache *cache, void *out, float *lse, void *stream) {
  if (ctx == nullptr) return SAGEKV_ERR_INVALID;
  const int bad = sagekv_paged_check(&ctx->shape, cache);
  if (bad != SAGEKV_OK) return bad;
  if (!on_own_device(ctx)) return SAGEKV_ERR_DEVICE;
  if (cache->n_seqs == 0) return SAGEKV_OK;
  if (q == nullptr || out == nullptr || cache->seq_lens == nullptr ||
      (cache->n_seqs > 1 && q_stride < (int64_t)ctx->shape.n_q_heads * kHeadDim))
    return SAGEKV_ERR_INVALID;
  if (!aligned16(q) || !aligned16(out) || q_stride % 8 != 0) return SAGEKV_ERR_ALIGN;
  PagedAttnParams p;
  p.c = view_of(ctx, cache);
  p.q = static_cast<const uint16_t *>(q);
  p.q_stride = q_stride;
  p.out = static_cast<uint16_t *>(out);
  p.lse = lse;
  p.partials = ctx->paged_partials;
  p.tickets = ctx->paged_tickets;
  p.group_tickets = ctx->paged_tickets + (int64_t)ctx->shape.batch * ctx->shape.n_kv_heads;
  p.G = ctx->G;
  p.H_q = ctx->shape.n_q_heads;
  p.H_kv = ctx->shape.n_kv_heads;
  p.most_ctas = paged_attn_max_ctas(ctx->dev->n_sm);
  p.n_tickets = ctx->shape.batch * ctx->shape.n_kv_heads;
  p.scale_log2 = ctx->scale * kLog2e;
  return done(ctx, launch_paged_attn(p, cache->dtype, ctx->dev->n_sm, static_cast<cudaStream_t>(stream)));
}

int sagekv_paged_score(sagekv_ctx *ctx, const void *q_last, const sagekv_paged_cache *cache, int64_t n_ctx, int32_t n_init, int32_t n_recent,
                       float *scores, int64_t scores_row_stride, void *stream) {
  if (ctx == nullptr || q_last == nullptr || scores == nullptr) return SAGEKV_ERR_INVALID;
  if (n_init < 0 || n_recent < 0 || n_ctx < 1 || (int64_t)n_init + n_recent + 1 > n_ctx) return SAGEKV_ERR_INVALID;
  const int bad = sagekv_paged_check(&ctx->shape, cache);
  if (bad != SAGEKV_OK) return bad;
  if (cache->n_seqs != ctx->shape.batch || n_ctx > (int64_t)cache->max_pages * cache->page_size) return SAGEKV_ERR_INVALID;
  if (n_ctx > ctx->max_ctx) return SAGEKV_ERR_UNSUPPORTED;
  if (!on_own_device(ctx)) return SAGEKV_ERR_DEVICE;
  const int64_t E = n_ctx - 1 - n_init - n_recent;
  if (scores_row_stride < E) return SAGEKV_ERR_INVALID;
  if (!aligned16(q_last) || !aligned16(scores) || scores_row_stride % 4 != 0) return SAGEKV_ERR_ALIGN;
  ScoreParams p = {};
  p.q = static_cast<const uint16_t *>(q_last);
  p.scores = scores;
  p.row_stride = scores_row_stride;
  p.partials = ctx->score_partials;
  p.sketch = ctx->hint == 1;
  p.sketch_off = -1;
  if (ctx->hint == 2 && ctx->hint_k > 0) {
    const int64_t kq = ctx->hint_k / ctx->G;
    p.list_k_q = (int)(kq < E ? kq : E);
  }
  p.status = ctx->status;
  p.E = (int)E;
  p.S = n_init;
  p.G = ctx->G;
  p.H_q = ctx->shape.n_q_heads;
  p.H_kv = ctx->shape.n_kv_heads;
  p.B = ctx->shape.batch;
  p.scale_log2 = ctx->scale * kLog2e;
  return done(ctx, launch_paged_score(p, view_of(ctx, cache), cache->dtype, ctx->max_chunks, ctx->dev->n_sm, static_cast<cudaStream_t>(stream)));
}

int sagekv_paged_compact(sagekv_ctx *ctx, const int32_t *idx, const sagekv_paged_cache *cache, int64_t n_ctx, int32_t n_init, int32_t n_recent,
                         int32_t k, void *Kc, void *Vc, sagekv_strides cs, sagekv_cache_state *state, void *stream) {
  if (ctx == nullptr || Kc == nullptr || Vc == nullptr || state == nullptr || state->d_step == nullptr) return SAGEKV_ERR_INVALID;
  if (n_init < 0 || n_recent < 0 || k < 0 || n_ctx < 1 || (int64_t)n_init + n_recent + 1 > n_ctx || k % ctx->G != 0) return SAGEKV_ERR_INVALID;
  const int bad = sagekv_paged_check(&ctx->shape, cache);
  if (bad != SAGEKV_OK) return bad;
  if (cache->n_seqs != ctx->shape.batch || n_ctx > (int64_t)cache->max_pages * cache->page_size) return SAGEKV_ERR_INVALID;
  if (n_ctx > ctx->max_ctx || ctx->group_mode == 1) return SAGEKV_ERR_UNSUPPORTED;
  if (!on_own_device(ctx)) return SAGEKV_ERR_DEVICE;
  const int64_t E = n_ctx - 1 - n_init - n_recent;
  int64_t k_q = k / ctx->G;
  if (k_q > E) k_q = E;
  if ((k_q > 0 && idx == nullptr) || cs.token_stride < kHeadDim) return SAGEKV_ERR_INVALID;
  const int64_t L = (int64_t)n_init + ctx->G * k_q + n_recent + 1;
  if (L > ctx->max_len) return SAGEKV_ERR_UNSUPPORTED;
  if (!aligned16(Kc) || !aligned16(Vc) || cs.batch_stride % 8 != 0 || cs.head_stride % 8 != 0 || cs.token_stride % 8 != 0) return SAGEKV_ERR_ALIGN;
  PagedCompactParams p;
  p.c = view_of(ctx, cache);
  p.idx = idx;
  p.Kc = static_cast<uint16_t *>(Kc);
  p.Vc = static_cast<uint16_t *>(Vc);
  p.cs = cs;
  p.d_step = state->d_step;
  p.E = (int)E;
  p.S = n_init;
  p.R = n_recent;
  p.N = (int)n_ctx;
  p.k_q = (int)k_q;
  p.G = ctx->G;
  p.H_kv = ctx->shape.n_kv_heads;
  p.B = ctx->shape.batch;
  const cudaError_t e = launch_paged_compact(p, cache->dtype, ctx->dev->n_sm, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return cuda_fail(ctx, e);
  state->n_init = n_init;
  state->k_q = (int32_t)k_q;
  state->n_sel = (int32_t)(ctx->G * k_q);
  state->n_recent = n_recent;
  state->ring_len = n_recent + 1;
  state->len = (int32_t)L;
  return SAGEKV_OK;
}

}  // extern "C"
