// C-ABI entry points of the operators on token rows: layer norm, 8-bit codes of rows and their products, caches held in 8 bits and attention over them.
#include <cmath>
#include <string>

#include "entry.h"
#include "tokens.h"

using namespace fa;

namespace {

// The stride of an axis of one entry says nothing.
RowsPtr rows_ptr(const freqattn_rows* r, int64_t batch, int64_t rows) {
  return RowsPtr{(char*)r->data, batch > 1 ? r->batch_stride : 0, rows > 1 ? r->row_stride : 0};
}
bool given_rows(const freqattn_rows* r) { return r && r->data; }

constexpr int64_t MOST_ROWS = (int64_t)1 << 31;      // rows are counted in 32 bits

// ---- layer norm
freqattn_status norm_params(const char* who, const freqattn_norm_shape* s, NormParams& p) {
  if (!s) return fail(FREQATTN_EINVAL, who, "NULL argument");
  if (!known(s->dtype)) return fail(FREQATTN_EINVAL, who, "unknown dtype");
  if (s->batch < 0 || s->rows < 0) return fail(FREQATTN_EINVAL, who, "sizes must not be negative");
  if (s->channels < 1) return fail(FREQATTN_EINVAL, who, "channels must be positive");
  if (s->channels > NORM_MOST_CHANNELS) return fail(FREQATTN_EUNSUPPORTED, who, "channels above 16384");
  if (!(s->eps >= 0.f) || !std::isfinite(s->eps)) return fail(FREQATTN_EINVAL, who, "eps must be finite and not negative");
  const bool each = s->weights_per_batch != 0;
  if ((int64_t)s->batch * s->rows >= MOST_ROWS || (each && s->batch > 65535)) return fail(FREQATTN_EUNSUPPORTED, who, "too many rows for one call");
  p = NormParams{};
  p.groups = each ? s->batch : 1;
  p.rows = s->rows;
  p.n = each ? s->rows : (int64_t)s->batch * s->rows;
  p.channels = s->channels;
  p.eps = s->eps;
  return FREQATTN_OK;
}

}  // namespace

extern "C" freqattn_status freqattn_layer_norm(const freqattn_norm_shape* s, const freqattn_rows* x, const void* w, const void* b, const freqattn_rows* out,
                                               void* stream) {
  return guarded([&]() -> freqattn_status {
    const char* who = "freqattn_layer_norm";
    NormParams p;
    const freqattn_status fs = norm_params(who, s, p);
    if (fs != FREQATTN_OK) return fs;
    if (s->batch == 0 || s->rows == 0) return FREQATTN_OK;
    if (!given_rows(x) || !given_rows(out)) return fail(FREQATTN_EINVAL, who, "NULL argument");
    p.x = rows_ptr(x, s->batch, s->rows);
    p.y = rows_ptr(out, s->batch, s->rows);
    p.w = w;
    p.b = b;
    return launched(launch_layer_norm(p, s->dtype, compute_units(), (hipStream_t)stream), who);
  });
}

extern "C" int64_t freqattn_layer_norm_workspace(const freqattn_norm_shape* s) {
  NormParams p;
  if (guarded([&] { return norm_params("freqattn_layer_norm_workspace", s, p); }) != FREQATTN_OK) return 0;
  const int64_t blocks = p.groups > 0 ? norm_backward_blocks(p.n, p.groups, p.channels, s->dtype, compute_units()) : 0;
  return blocks > 1 ? blocks * p.groups * 2 * p.channels * 4 : 0;
}

extern "C" freqattn_status freqattn_layer_norm_backward(const freqattn_norm_shape* s, const freqattn_rows* x, const void* w, const freqattn_rows* dout,
                                                        const freqattn_rows* dx, float* dw, float* db, void* workspace, int64_t workspace_bytes,
                                                        void* stream) {
  return guarded([&]() -> freqattn_status {
    const char* who = "freqattn_layer_norm_backward";
    NormParams p;
    const freqattn_status fs = norm_params(who, s, p);
    if (fs != FREQATTN_OK) return fs;
    const bool any = s->batch > 0 && s->rows > 0;
    if (any && (!given_rows(x) || !given_rows(dout) || !given_rows(dx))) return fail(FREQATTN_EINVAL, who, "NULL argument");
    if (dw || db) {
      const int64_t need = freqattn_layer_norm_workspace(s);
      if (need > 0 && (!workspace || workspace_bytes < need)) return fail(FREQATTN_EINVAL, who, "workspace too small");
      if (need > 0 && (uintptr_t)workspace % 16) return fail(FREQATTN_EINVAL, who, "workspace must be 16-byte aligned");
    }
    if (p.groups == 0 || (!any && !dw && !db)) return FREQATTN_OK;
    // (with no rows the sums are still written: zeros)
    if (any) { p.x = rows_ptr(x, s->batch, s->rows); p.dy = rows_ptr(dout, s->batch, s->rows); p.dx = rows_ptr(dx, s->batch, s->rows); }
    p.w = w;
    p.dw = dw;
    p.db = db;
    p.part = (float*)workspace;
    return launched(launch_layer_norm_backward(p, s->dtype, compute_units(), (hipStream_t)stream), who);
  });
}

// ---- 8-bit codes of rows and their products
extern "C" freqattn_status freqattn_quantize_rows(int32_t dtype, int32_t batch, int32_t rows, int32_t channels, const freqattn_rows* x,
                                                  const freqattn_rows* codes, float* scales, void* stream) {
  return guarded([&]() -> freqattn_status {
    const char* who = "freqattn_quantize_rows";
    if (!known(dtype)) return fail(FREQATTN_EINVAL, who, "unknown dtype");
    if (batch < 0 || rows < 0) return fail(FREQATTN_EINVAL, who, "sizes must not be negative");
    if (channels < 1) return fail(FREQATTN_EINVAL, who, "channels must be positive");
    if (channels > PRODUCT_MOST_CHANNELS) return fail(FREQATTN_EUNSUPPORTED, who, "channels above 131071");
    if ((int64_t)batch * rows >= MOST_ROWS) return fail(FREQATTN_EUNSUPPORTED, who, "too many rows for one call");
    if (batch == 0 || rows == 0) return FREQATTN_OK;
    if (!given_rows(x) || !given_rows(codes) || !scales) return fail(FREQATTN_EINVAL, who, "NULL argument");
    CodeParams p = {};
    p.x = rows_ptr(x, batch, rows);
    p.codes = rows_ptr(codes, batch, rows);
    p.scales = scales;
    p.n = (int64_t)batch * rows;
    p.rows = rows;
    p.channels = channels;
    return launched(launch_quantize_rows(p, dtype, compute_units(), (hipStream_t)stream), who);
  });
}

extern "C" freqattn_status freqattn_product_i8(const freqattn_product_shape* s, const int8_t* a, int64_t a_stride, const float* a_scales, const int8_t* w,
                                               int64_t w_stride, const float* w_scales, const void* bias, void* out, int64_t out_stride,
                                               void* stream) {
  return guarded([&]() -> freqattn_status {
    const char* who = "freqattn_product_i8";
    if (!s) return fail(FREQATTN_EINVAL, who, "NULL argument");
    if (!known(s->dtype)) return fail(FREQATTN_EINVAL, who, "unknown dtype");
    if (s->rows < 0 || s->outputs < 0) return fail(FREQATTN_EINVAL, who, "sizes must not be negative");
    if (s->channels < 1) return fail(FREQATTN_EINVAL, who, "channels must be positive");
    if (s->channels > PRODUCT_MOST_CHANNELS) return fail(FREQATTN_EUNSUPPORTED, who, "channels above 131071");
    if (s->rows > (1 << 30) || s->outputs > (1 << 30)) return fail(FREQATTN_EUNSUPPORTED, who, "too many rows for one call");
    if (s->rows == 0 || s->outputs == 0) return FREQATTN_OK;
    if (!a || !a_scales || !w || !w_scales || !out) return fail(FREQATTN_EINVAL, who, "NULL argument");
    ProductParams p = {};
    p.rows = s->rows;
    p.channels = s->channels;
    p.outputs = s->outputs;
    p.a = (const char*)a;
    p.w = (const char*)w;
    p.a_rs = s->rows > 1 ? a_stride : 0;
    p.w_rs = s->outputs > 1 ? w_stride : 0;
    p.out_rs = s->rows > 1 ? out_stride : 0;
    p.a_scales = a_scales;
    p.w_scales = w_scales;
    p.bias = bias;
    p.out = (char*)out;
    p.vec = p.channels % 16 == 0 && ((uintptr_t)a | (uintptr_t)w | (uintptr_t)p.a_rs | (uintptr_t)p.w_rs) % 16 == 0;
    return launched(launch_product_i8(p, s->dtype, compute_units(), (hipStream_t)stream), who);
  });
}

// ---- caches held in 8 bits
namespace {

freqattn_status cache8_shape(const char* who, const freqattn_sequence_shape* s, const freqattn_cache8* c, int& shift) {
  if (!s || !c) return fail(FREQATTN_EINVAL, who, "NULL argument");
  for (shift = 4; shift <= 8 && c->block_rows != 1 << shift; ++shift) {}
  if (shift > 8) return fail(FREQATTN_EINVAL, who, "block_rows must be 16, 32, 64, 128 or 256");
  return FREQATTN_OK;
}

freqattn_status cache8_params(const char* who, const freqattn_sequence_shape* s, const freqattn_sequence_rows* rows, const freqattn_cache8* c,
                              const freqattn_heads* k, const freqattn_heads* v, bool append, Cache8Params& p, bool& nothing) {
  int shift;
  freqattn_status fs = cache8_shape(who, s, c, shift);
  if (fs != FREQATTN_OK) return fs;
  if (!known(s->dtype)) return fail(FREQATTN_EINVAL, who, "unknown dtype");
  if (s->sequences < 0 || s->q_rows < 0 || s->k_rows < 0) return fail(FREQATTN_EINVAL, who, "sizes must not be negative");
  if (s->kv_heads < 1 || s->head_dim < 1) return fail(FREQATTN_EINVAL, who, "kv_heads and head_dim must be positive");
  if (s->head_dim > 128) return fail(FREQATTN_EUNSUPPORTED, who, "head_dim above 128");
  if (rows && rows->k_offsets) return fail(FREQATTN_EINVAL, who, "a cache has no offsets");
  if (s->q_rows >= (1 << 30) || s->k_rows >= (1 << 30) || s->sequences >= (1 << 23) || s->kv_heads >= (1 << 23))
    return fail(FREQATTN_EUNSUPPORTED, who, "too many rows for one call");
  p = Cache8Params{};
  p.nseq = s->sequences;
  p.heads = s->kv_heads;
  p.d = s->head_dim;
  p.q_rows = s->q_rows;
  p.k_rows = s->k_rows;
  p.shift = shift;
  p.blocks = (int32_t)(((int64_t)s->k_rows + c->block_rows - 1) >> shift);
  if (rows) { p.q_off = rows->q_offsets; p.q_len = rows->q_lengths; p.k_len = rows->k_lengths; }
  nothing = s->sequences == 0 || s->k_rows == 0 || (append && s->q_rows == 0);
  if (nothing) return FREQATTN_OK;
  if (!given(k) || !given(v) || !given(&c->k) || !given(&c->v) || !c->k_scales || !c->v_scales) return fail(FREQATTN_EINVAL, who, "NULL argument");
  const int64_t batch = append && p.q_off ? 1 : p.nseq, n = append ? p.q_rows : p.k_rows;
  p.k = ptr(k, batch, n, p.heads);
  p.v = ptr(v, batch, n, p.heads);
  p.ck = ptr(&c->k, p.nseq, p.k_rows, p.heads);
  p.cv = ptr(&c->v, p.nseq, p.k_rows, p.heads);
  p.ks = c->k_scales;
  p.vs = c->v_scales;
  return FREQATTN_OK;
}

}  // namespace

extern "C" freqattn_status freqattn_cache8_append(const freqattn_sequence_shape* s, const freqattn_sequence_rows* rows, const freqattn_heads* k,
                                                  const freqattn_heads* v, const freqattn_cache8* cache, void* stream) {
  return guarded([&]() -> freqattn_status {
    const char* who = "freqattn_cache8_append";
    Cache8Params p;
    bool nothing;
    const freqattn_status fs = cache8_params(who, s, rows, cache, k, v, true, p, nothing);
    if (fs != FREQATTN_OK || nothing) return fs;
    return launched(launch_cache8_append(p, s->dtype, (hipStream_t)stream), who);
  });
}

extern "C" freqattn_status freqattn_cache8_read(const freqattn_sequence_shape* s, const freqattn_sequence_rows* rows, const freqattn_cache8* cache,
                                                const freqattn_heads* k, const freqattn_heads* v, void* stream) {
  return guarded([&]() -> freqattn_status {
    const char* who = "freqattn_cache8_read";
    Cache8Params p;
    bool nothing;
    const freqattn_status fs = cache8_params(who, s, rows, cache, k, v, false, p, nothing);
    if (fs != FREQATTN_OK || nothing) return fs;
    return launched(launch_cache8_read(p, s->dtype, (hipStream_t)stream), who);
  });
}

namespace {

freqattn_status cache8_attention_params(const char* who, const freqattn_sequence_shape* s, const freqattn_sequence_rows* rows, const freqattn_cache8* c,
                                        SeqParams& p, Cache8Scales& sc) {
  freqattn_status fs = cache8_shape(who, s, c, sc.shift);
  if (fs != FREQATTN_OK) return fs;
  if (rows && rows->k_offsets) return fail(FREQATTN_EINVAL, who, "a cache has no offsets");
  fs = seq_params(who, s, rows, p);
  if (fs != FREQATTN_OK) return fs;
  sc.k = c->k_scales;
  sc.v = c->v_scales;
  sc.blocks = (int32_t)(((int64_t)s->k_rows + c->block_rows - 1) >> sc.shift);
  return FREQATTN_OK;
}

}  // namespace

extern "C" int64_t freqattn_cache8_attention_workspace(const freqattn_sequence_shape* s, const freqattn_sequence_rows* rows) {
  SeqParams p;
  if (guarded([&] { return seq_params("freqattn_cache8_attention_workspace", s, rows, p); }) != FREQATTN_OK) return 0;
  return cache8_plan(p, s->dtype, compute_units()).workspace;
}

extern "C" freqattn_status freqattn_cache8_attention(const freqattn_sequence_shape* s, const freqattn_sequence_rows* rows, const freqattn_heads* q,
                                                     const freqattn_cache8* cache, const freqattn_heads* out, float* lse, void* workspace,
                                                     int64_t workspace_bytes, void* stream) {
  return guarded([&]() -> freqattn_status {
    const char* who = "freqattn_cache8_attention";
    SeqParams p;
    Cache8Scales sc = {};
    const freqattn_status fs = cache8_attention_params(who, s, rows, cache, p, sc);
    if (fs != FREQATTN_OK) return fs;
    if (p.lse_rows == 0 || p.nseq == 0) return FREQATTN_OK;
    if (!given(q) || !given(out) || (p.k_rows > 0 && (!given(&cache->k) || !given(&cache->v) || !sc.k || !sc.v))) return fail(FREQATTN_EINVAL, who, "NULL argument");
    const int size = size_of(s->dtype);
    p.q = q_ptr(p, q);
    p.o = q_ptr(p, out);
    p.vec = p.d % 8 == 0 && pieces16(p.q, size) && pieces16(p.o, size);
    if (p.k_rows > 0) {
      p.k = k_ptr(p, &cache->k);
      p.v = k_ptr(p, &cache->v);
    }
    p.lse = lse;
    const SeqPlan plan = cache8_plan(p, s->dtype, compute_units());
    if (plan.workspace > 0 && (!workspace || workspace_bytes < plan.workspace)) return fail(FREQATTN_EINVAL, who, "workspace too small");
    if (plan.workspace > 0 && (uintptr_t)workspace % 16) return fail(FREQATTN_EINVAL, who, "workspace must be 16-byte aligned");
    p.part = (float*)workspace;
    return launched(p.vec ? launch_cache8_attention(p, sc, plan, s->dtype, (hipStream_t)stream) : launch_cache8_generic(p, sc, s->dtype, (hipStream_t)stream), who);
  });
}
