// What the C entry points without a context share: errors, checks of arguments, addresses.
#pragma once
#include <cmath>
#include <string>

#include "heads.h"

namespace fa {

inline freqattn_status fail(freqattn_status s, const char* who, const std::string& msg) {
  context_free_error() = std::string(who) + ": " + msg;
  return s;
}

// No exception may cross the C boundary.
template <class F>
freqattn_status guarded(F&& body) {
  try {
    return body();
  } catch (...) {
    return FREQATTN_ENOMEM;   // (a string that could not be allocated is all there is)
  }
}

inline freqattn_status launched(hipError_t e, const char* who) {
  if (e == hipSuccess) return FREQATTN_OK;
  if (e == hipErrorInvalidConfiguration) return fail(FREQATTN_EUNSUPPORTED, who, "too many rows for one call");
  return fail(FREQATTN_EHIP, who, std::string("launch: ") + hipGetErrorString(e));
}

inline int compute_units() {
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) return 256;
  return n;
}

inline bool known(int32_t dtype) { return dtype == FREQATTN_F32 || dtype == FREQATTN_BF16; }
inline int size_of(int32_t dtype) { return dtype == FREQATTN_F32 ? 4 : 2; }

// The stride of an axis of one entry says nothing (and must not decide which kernel runs).
inline HeadsPtr ptr(const freqattn_heads* h, int64_t batch, int64_t rows, int64_t heads) {
  return HeadsPtr{(const char*)h->data, batch > 1 ? h->batch_stride : 0, rows > 1 ? h->row_stride : 0, heads > 1 ? h->head_stride : 0};
}
inline bool given(const freqattn_heads* h) { return h && h->data; }

// The largest launch: fewer than 2^32 threads, in workgroups of up to 512.
constexpr int64_t MAX_BLOCKS = (int64_t)1 << 23;

// ---- attention over sequences
inline freqattn_status seq_params(const char* who, const freqattn_sequence_shape* s, const freqattn_sequence_rows* rows, SeqParams& p) {
  if (!s) return fail(FREQATTN_EINVAL, who, "NULL argument");
  if (!known(s->dtype)) return fail(FREQATTN_EINVAL, who, "unknown dtype");
  if (s->sequences < 0 || s->q_rows < 0 || s->k_rows < 0) return fail(FREQATTN_EINVAL, who, "sizes must not be negative");
  if (s->q_heads < 1 || s->kv_heads < 1 || s->q_heads % s->kv_heads) return fail(FREQATTN_EINVAL, who, "q_heads must be a multiple of kv_heads");
  if (s->head_dim < 1) return fail(FREQATTN_EINVAL, who, "head_dim must be positive");
  if (s->head_dim > 128) return fail(FREQATTN_EUNSUPPORTED, who, "head_dim above 128");
  if (s->softmax_scale != s->softmax_scale || std::isinf(s->softmax_scale)) return fail(FREQATTN_EINVAL, who, "softmax_scale must be finite");
  p = SeqParams{};
  p.nseq = s->sequences;
  p.hq = s->q_heads;
  p.hk = s->kv_heads;
  p.group = s->q_heads / s->kv_heads;
  p.d = s->head_dim;
  p.q_rows = s->q_rows;
  p.k_rows = s->k_rows;
  p.causal = s->causal != 0;
  p.scale = s->softmax_scale > 0.f ? s->softmax_scale : 1.0f / std::sqrt((float)s->head_dim);
  if (rows) { p.q_off = rows->q_offsets; p.k_off = rows->k_offsets; p.q_len = rows->q_lengths; p.k_len = rows->k_lengths; }
  const int64_t qr = p.q_off ? s->q_rows : (int64_t)s->sequences * s->q_rows, kr = p.k_off ? s->k_rows : (int64_t)s->sequences * s->k_rows;
  p.lse_rows = qr;
  p.lse_k = kr;
  // row indices of one sequence's group and launch sizes stay within 31 bits
  // (sequences first: what the products behind it can come to is below 2^63 then)
  if ((int64_t)s->sequences * p.hk >= MAX_BLOCKS || (int64_t)s->q_rows * p.group >= ((int64_t)1 << 30) || s->k_rows >= (1 << 30) ||
      (qr * p.group / 32 + s->sequences) * p.hk >= MAX_BLOCKS || (kr / 32 + s->sequences) * p.hk >= MAX_BLOCKS)
    return fail(FREQATTN_EUNSUPPORTED, who, "too many rows for one call");
  return FREQATTN_OK;
}

// Eight rows lie within 2^32 bytes, as one copy of the bf16 kernels takes them.
inline bool near(const HeadsPtr& v) { return v.ts >= 0 && v.ts < ((int64_t)1 << 27); }

inline bool pieces16(const HeadsPtr& v, int size) {
  return (uintptr_t)v.p % 16 == 0 && v.bs * size % 16 == 0 && v.ts * size % 16 == 0 && v.hs * size % 16 == 0;
}
// A tensor of queries or of keys: the batch axis of a packed one is not used.
inline HeadsPtr q_ptr(const SeqParams& p, const freqattn_heads* h) { return ptr(h, p.q_off ? 1 : p.nseq, p.q_rows, p.hq); }
inline HeadsPtr k_ptr(const SeqParams& p, const freqattn_heads* h) { return ptr(h, p.k_off ? 1 : p.nseq, p.k_rows, p.hk); }

}  // namespace fa
