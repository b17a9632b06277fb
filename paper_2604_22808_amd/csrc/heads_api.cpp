// C-ABI entry points of the operators that need no context: rotary positions, norms of Q and K, attention over sequences.
#include <cmath>
#include <new>
#include <string>

#include "heads.h"

using namespace fa;

struct freqattn_rotary {
  RotTable t;
  int head_dim;
  bool grid;
  double radians[ROT_MAX_PAIRS];
  double amplitude;
};

namespace {

freqattn_status fail(freqattn_status s, const char* who, const std::string& msg) {
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

freqattn_status launched(hipError_t e, const char* who) {
  if (e == hipSuccess) return FREQATTN_OK;
  if (e == hipErrorInvalidConfiguration) return fail(FREQATTN_EUNSUPPORTED, who, "too many rows for one call");
  return fail(FREQATTN_EHIP, who, std::string("launch: ") + hipGetErrorString(e));
}

int compute_units() {
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) return 256;
  return n;
}

bool known(int32_t dtype) { return dtype == FREQATTN_F32 || dtype == FREQATTN_BF16; }
int size_of(int32_t dtype) { return dtype == FREQATTN_F32 ? 4 : 2; }

// The stride of an axis of one entry says nothing (and must not decide which kernel runs).
HeadsPtr ptr(const freqattn_heads* h, int64_t batch, int64_t rows, int64_t heads) {
  return HeadsPtr{(const char*)h->data, batch > 1 ? h->batch_stride : 0, rows > 1 ? h->row_stride : 0, heads > 1 ? h->head_stride : 0};
}
bool given(const freqattn_heads* h) { return h && h->data; }

// The largest launch: fewer than 2^32 threads, in workgroups of up to 512.
constexpr int64_t MAX_BLOCKS = (int64_t)1 << 23;

}  // namespace

extern "C" freqattn_status freqattn_rotary_create(const freqattn_rotary_cfg* c, freqattn_rotary** out) {
  return guarded([&]() -> freqattn_status {
    const char* who = "freqattn_rotary_create";
    if (!c || !out) return fail(FREQATTN_EINVAL, who, "NULL argument");
    *out = nullptr;
    if (c->head_dim < 2 || c->head_dim > 512 || c->head_dim % 2) return fail(FREQATTN_EINVAL, who, "head_dim must be even, 2..512");
    if (c->axes < 1 || c->axes > 4) return fail(FREQATTN_EINVAL, who, "1 to 4 axes");
    int64_t r = 0;
    for (int a = 0; a < c->axes; ++a) {
      if (c->axis_dim[a] < 0 || c->axis_dim[a] % 2) return fail(FREQATTN_EINVAL, who, "axis_dim must be even and not negative");
      r += c->axis_dim[a];
    }
    if (r < 2 || r > c->head_dim) return fail(FREQATTN_EINVAL, who, "the sum of axis_dim must be 2..head_dim");
    if (c->layout != FREQATTN_ROTARY_HALF && c->layout != FREQATTN_ROTARY_INTERLEAVED) return fail(FREQATTN_EINVAL, who, "unknown layout");
    if (c->scaling < FREQATTN_ROTARY_PLAIN || c->scaling > FREQATTN_ROTARY_BY_PARTS) return fail(FREQATTN_EINVAL, who, "unknown scaling");
    if (!(c->base > 1.0) || !std::isfinite(c->base)) return fail(FREQATTN_EINVAL, who, "base must be above 1");
    if (c->scaling != FREQATTN_ROTARY_PLAIN && !(c->factor > 0.0 && std::isfinite(c->factor))) return fail(FREQATTN_EINVAL, who, "factor must be positive");
    if (!(c->amplitude >= 0.0) || !std::isfinite((float)c->amplitude)) return fail(FREQATTN_EINVAL, who, "amplitude must not be negative, and finite in fp32");
    if (c->scaling == FREQATTN_ROTARY_BY_PARTS &&
        !(c->factor >= 1.0 && c->context > 0 && c->beta_slow >= 0.0 && c->beta_fast > c->beta_slow && std::isfinite(c->beta_fast)))
      return fail(FREQATTN_EINVAL, who, "scaling by parts needs factor >= 1, context > 0 and beta_fast > beta_slow >= 0");
    int extents = 0;
    for (int a = 0; a < c->axes; ++a) {
      if (c->grid[a] < 0) return fail(FREQATTN_EINVAL, who, "grid extents must not be negative");
      extents += c->grid[a] > 0;
    }
    if (extents != 0 && extents != c->axes) return fail(FREQATTN_EINVAL, who, "a grid needs an extent for every axis");
    freqattn_rotary* h = new (std::nothrow) freqattn_rotary();
    if (!h) return fail(FREQATTN_ENOMEM, who, "host allocation failed");
    h->head_dim = c->head_dim;
    h->grid = extents != 0;
    h->t.axes = c->axes;
    h->t.half = (int)(r / 2);
    h->t.interleaved = c->layout == FREQATTN_ROTARY_INTERLEAVED;
    for (int a = 0; a < 4; ++a) h->t.grid[a] = h->grid ? (a < c->axes ? (uint32_t)c->grid[a] : 1u) : 0u;
    const long double two_pi = 6.283185307179586476925286766559L;
    int at = 0;
    for (int a = 0; a < c->axes; ++a) {
      const long double n = c->axis_dim[a], f = c->factor;
      long double base = c->base;
      if (c->scaling == FREQATTN_ROTARY_NTK && c->axis_dim[a] > 2) base *= powl(f, n / (n - 2));
      for (int j = 0; j < c->axis_dim[a] / 2; ++j, ++at) {
        long double theta = powl(base, -2.0L * j / n);
        if (c->scaling == FREQATTN_ROTARY_LINEAR) theta /= f;
        if (c->scaling == FREQATTN_ROTARY_BY_PARTS) {
          const long double turns = c->context * theta / two_pi;
          long double keep = (turns - c->beta_slow) / ((long double)c->beta_fast - c->beta_slow);
          keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
          theta *= keep + (1 - keep) / f;
        }
        long double turn = theta / two_pi;
        turn -= floorl(turn);
        long double fixed = roundl(turn * 18446744073709551616.0L);
        h->t.turn[at] = fixed >= 18446744073709551616.0L ? 0 : (uint64_t)fixed;
        h->t.axis[at] = (uint8_t)a;
        h->radians[at] = (double)theta;
      }
    }
    h->amplitude = c->amplitude > 0.0 ? c->amplitude : c->scaling == FREQATTN_ROTARY_BY_PARTS ? 0.1 * std::log(c->factor) + 1.0 : 1.0;
    h->t.amplitude = (float)h->amplitude;
    *out = h;
    return FREQATTN_OK;
  });
}

extern "C" void freqattn_rotary_destroy(freqattn_rotary* h) { delete h; }   // (launches carry the table by value)

extern "C" freqattn_status freqattn_rotary_frequencies(const freqattn_rotary* h, double* radians, double* amplitude) {
  return guarded([&]() -> freqattn_status {
    if (!h || !radians || !amplitude) return fail(FREQATTN_EINVAL, "freqattn_rotary_frequencies", "NULL argument");
    for (int i = 0; i < h->t.half; ++i) radians[i] = h->radians[i];
    *amplitude = h->amplitude;
    return FREQATTN_OK;
  });
}

namespace {

// Checks that the rotation and the norms have in common, and the fields of QkParams they share.
freqattn_status qk_common(const char* who, const freqattn_rotary* rot, int32_t dtype, int32_t batch, int32_t tokens, int32_t h0, int32_t h1,
                          int32_t head_dim, const int32_t* positions, int64_t positions_stride, QkParams& p) {
  if (!known(dtype)) return fail(FREQATTN_EINVAL, who, "unknown dtype");
  if (batch < 0 || tokens < 0 || h0 < 0 || h1 < 0) return fail(FREQATTN_EINVAL, who, "sizes must not be negative");
  if (rot) {
    if (rot->head_dim != head_dim) return fail(FREQATTN_EINVAL, who, "head_dim is not the rotary's");
    if (!positions) {
      if (!rot->grid && rot->t.axes > 1) return fail(FREQATTN_EINVAL, who, "several axes and no grid: positions must be given");
      if (rot->grid) {
        int64_t n = 1;
        for (int a = 0; a < rot->t.axes && n <= tokens; ++a) n *= rot->t.grid[a];
        if (n != tokens) return fail(FREQATTN_EINVAL, who, "tokens is not the grid's size: positions must be given");
      }
    }
  }
  p = QkParams{};
  p.batch = batch;
  p.tokens = tokens;
  p.heads[0] = h0;
  p.heads[1] = h1;
  p.d = head_dim;
  p.pos = rot ? positions : nullptr;
  p.pos_bs = positions_stride;
  return FREQATTN_OK;
}

freqattn_status qk_shape_ok(const char* who, const freqattn_qk_shape* s) {
  if (!s) return fail(FREQATTN_EINVAL, who, "NULL argument");
  if (s->head_dim < 2 || s->head_dim > 512 || s->head_dim % 2) return fail(FREQATTN_EINVAL, who, "head_dim must be even, 2..512");
  if (!(s->eps >= 0.f) || !std::isfinite(s->eps)) return fail(FREQATTN_EINVAL, who, "eps must be finite and not negative");
  return FREQATTN_OK;
}

const RotTable no_rotation = {};

}  // namespace

hipError_t fa::copy_heads(int dtype, int batch, int tokens, int heads, int d, const freqattn_heads& x, const freqattn_heads& out, hipStream_t st) {
  QkParams p = {};
  p.batch = batch;
  p.tokens = tokens;
  p.heads[0] = heads;
  p.d = d;
  p.in[0] = ptr(&x, batch, tokens, heads);
  p.out[0] = ptr(&out, batch, tokens, heads);
  return launch_qk(p, no_rotation, dtype, compute_units(), st);
}

extern "C" freqattn_status freqattn_rotary_apply(const freqattn_rotary* rot, int32_t dtype, int32_t batch, int32_t tokens, int32_t heads,
                                                 const freqattn_heads* x, const int32_t* positions, int64_t positions_stride, int32_t inverse,
                                                 const freqattn_heads* out, void* stream) {
  return guarded([&]() -> freqattn_status {
    const char* who = "freqattn_rotary_apply";
    if (!rot) return fail(FREQATTN_EINVAL, who, "NULL argument");
    QkParams p;
    const freqattn_status fs = qk_common(who, rot, dtype, batch, tokens, heads, 0, rot->head_dim, positions, positions_stride, p);
    if (fs != FREQATTN_OK) return fs;
    if (batch == 0 || tokens == 0 || heads == 0) return FREQATTN_OK;
    if (!given(x) || !given(out)) return fail(FREQATTN_EINVAL, who, "NULL argument");
    p.in[0] = ptr(x, batch, tokens, heads);
    p.out[0] = ptr(out, batch, tokens, heads);
    p.inverse = inverse != 0;
    return launched(launch_qk(p, rot->t, dtype, compute_units(), (hipStream_t)stream), who);
  });
}

extern "C" freqattn_status freqattn_qk_norm(const freqattn_qk_shape* s, const freqattn_rotary* rot, const int32_t* positions, int64_t positions_stride,
                                            const freqattn_heads* q, const freqattn_heads* k, const void* w_q, const void* w_k,
                                            const freqattn_heads* q_out, const freqattn_heads* k_out, void* stream) {
  return guarded([&]() -> freqattn_status {
    const char* who = "freqattn_qk_norm";
    freqattn_status fs = qk_shape_ok(who, s);
    if (fs != FREQATTN_OK) return fs;
    QkParams p;
    fs = qk_common(who, rot, s->dtype, s->batch, s->tokens, s->q_heads, s->k_heads, s->head_dim, positions, positions_stride, p);
    if (fs != FREQATTN_OK) return fs;
    if (s->batch == 0 || s->tokens == 0 || (s->q_heads == 0 && s->k_heads == 0)) return FREQATTN_OK;
    if ((s->q_heads && (!given(q) || !given(q_out))) || (s->k_heads && (!given(k) || !given(k_out)))) return fail(FREQATTN_EINVAL, who, "NULL argument");
    auto at = [&](const freqattn_heads* h, int heads) { return ptr(h, s->batch, s->tokens, heads); };
    if (s->q_heads) { p.in[0] = at(q, s->q_heads); p.out[0] = at(q_out, s->q_heads); }
    if (s->k_heads) { p.in[1] = at(k, s->k_heads); p.out[1] = at(k_out, s->k_heads); }
    p.w[0] = w_q;
    p.w[1] = w_k;
    p.norm = 1;
    p.eps = s->eps;
    return launched(launch_qk(p, rot ? rot->t : no_rotation, s->dtype, compute_units(), (hipStream_t)stream), who);
  });
}

extern "C" int64_t freqattn_qk_norm_workspace(int32_t head_dim) {
  return head_dim < 2 || head_dim > 512 ? 0 : (int64_t)QK_BWD_BLOCKS * 2 * head_dim * 4;
}

extern "C" freqattn_status freqattn_qk_norm_backward(const freqattn_qk_shape* s, const freqattn_rotary* rot, const int32_t* positions,
                                                     int64_t positions_stride, const freqattn_heads* q, const freqattn_heads* k, const void* w_q,
                                                     const void* w_k, const freqattn_heads* dq_out, const freqattn_heads* dk_out,
                                                     const freqattn_heads* dq, const freqattn_heads* dk, float* dw_q, float* dw_k, void* workspace,
                                                     int64_t workspace_bytes, void* stream) {
  return guarded([&]() -> freqattn_status {
    const char* who = "freqattn_qk_norm_backward";
    freqattn_status fs = qk_shape_ok(who, s);
    if (fs != FREQATTN_OK) return fs;
    QkParams p;
    fs = qk_common(who, rot, s->dtype, s->batch, s->tokens, s->q_heads, s->k_heads, s->head_dim, positions, positions_stride, p);
    if (fs != FREQATTN_OK) return fs;
    if (s->q_heads < 1) return fail(FREQATTN_EINVAL, who, "q_heads must be at least 1");
    const bool any = s->batch > 0 && s->tokens > 0;
    if (any && (!given(q) || !given(dq_out) || !given(dq) || (s->k_heads && (!given(k) || !given(dk_out) || !given(dk)))))
      return fail(FREQATTN_EINVAL, who, "NULL argument");
    if (dw_q || dw_k) {
      if (!workspace || workspace_bytes < freqattn_qk_norm_workspace(s->head_dim)) return fail(FREQATTN_EINVAL, who, "workspace too small");
      if ((uintptr_t)workspace % 16) return fail(FREQATTN_EINVAL, who, "workspace must be 16-byte aligned");
      p.part = (float*)workspace;
    } else if (!any) {
      return FREQATTN_OK;
    }
    // (with no rows the sums are still written: zeros)
    auto at = [&](const freqattn_heads* h, int heads) { return ptr(h, s->batch, s->tokens, heads); };
    if (any) { p.in[0] = at(q, s->q_heads); p.dy[0] = at(dq_out, s->q_heads); p.out[0] = at(dq, s->q_heads); }
    if (any && s->k_heads) { p.in[1] = at(k, s->k_heads); p.dy[1] = at(dk_out, s->k_heads); p.out[1] = at(dk, s->k_heads); }
    p.w[0] = w_q;
    p.w[1] = w_k;
    p.norm = 1;
    p.eps = s->eps;
    float* const dw[2] = {dw_q, dw_k};
    return launched(launch_qk_backward(p, rot ? rot->t : no_rotation, s->dtype, dw, compute_units(), (hipStream_t)stream), who);
  });
}

// ---- attention over sequences ------------------------------------------------------------------------------------------
namespace {

freqattn_status seq_params(const char* who, const freqattn_sequence_shape* s, const freqattn_sequence_rows* rows, SeqParams& p) {
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
bool near(const HeadsPtr& v) { return v.ts >= 0 && v.ts < ((int64_t)1 << 27); }

bool pieces16(const HeadsPtr& v, int size) {
  return (uintptr_t)v.p % 16 == 0 && v.bs * size % 16 == 0 && v.ts * size % 16 == 0 && v.hs * size % 16 == 0;
}
// A tensor of queries or of keys: the batch axis of a packed one is not used.
HeadsPtr q_ptr(const SeqParams& p, const freqattn_heads* h) { return ptr(h, p.q_off ? 1 : p.nseq, p.q_rows, p.hq); }
HeadsPtr k_ptr(const SeqParams& p, const freqattn_heads* h) { return ptr(h, p.k_off ? 1 : p.nseq, p.k_rows, p.hk); }

}  // namespace

extern "C" int64_t freqattn_sequence_attention_workspace(const freqattn_sequence_shape* s, const freqattn_sequence_rows* rows) {
  SeqParams p;
  if (guarded([&] { return seq_params("freqattn_sequence_attention_workspace", s, rows, p); }) != FREQATTN_OK) return 0;
  return s->dtype == FREQATTN_BF16 ? seq_fwd_plan(p, compute_units()).workspace : 0;
}

extern "C" freqattn_status freqattn_sequence_attention(const freqattn_sequence_shape* s, const freqattn_sequence_rows* rows, const freqattn_heads* q,
                                                       const freqattn_heads* k, const freqattn_heads* v, const freqattn_heads* out, float* lse,
                                                       void* workspace, int64_t workspace_bytes, void* stream) {
  return guarded([&]() -> freqattn_status {
    const char* who = "freqattn_sequence_attention";
    SeqParams p;
    const freqattn_status fs = seq_params(who, s, rows, p);
    if (fs != FREQATTN_OK) return fs;
    if (p.lse_rows == 0 || p.nseq == 0) return FREQATTN_OK;
    if (!given(q) || !given(out) || (p.k_rows > 0 && (!given(k) || !given(v)))) return fail(FREQATTN_EINVAL, who, "NULL argument");
    const int size = size_of(s->dtype);
    p.q = q_ptr(p, q);
    p.o = q_ptr(p, out);
    p.vec = p.d * size % 16 == 0 && pieces16(p.q, size) && pieces16(p.o, size);
    if (p.k_rows > 0) {
      p.k = k_ptr(p, k);
      p.v = k_ptr(p, v);
      p.vec = p.vec && pieces16(p.k, size) && pieces16(p.v, size);
    }
    p.lse = lse;
    if (s->dtype != FREQATTN_BF16) return launched(launch_seq_generic_fwd(p, s->dtype, (hipStream_t)stream), who);
    const SeqPlan plan = seq_fwd_plan(p, compute_units());
    if (plan.workspace > 0 && (!workspace || workspace_bytes < plan.workspace)) return fail(FREQATTN_EINVAL, who, "workspace too small");
    if (plan.workspace > 0 && (uintptr_t)workspace % 16) return fail(FREQATTN_EINVAL, who, "workspace must be 16-byte aligned");
    p.part = (float*)workspace;
    return launched(p.vec && near(p.k) && near(p.v) ? launch_seq_fwd(p, plan, (hipStream_t)stream) : launch_seq_generic_fwd(p, s->dtype, (hipStream_t)stream), who);
  });
}

extern "C" int64_t freqattn_sequence_attention_backward_workspace(const freqattn_sequence_shape* s, const freqattn_sequence_rows* rows) {
  SeqParams p;
  if (guarded([&] { return seq_params("freqattn_sequence_attention_backward_workspace", s, rows, p); }) != FREQATTN_OK) return 0;
  return s->dtype == FREQATTN_BF16 ? seq_bwd_plan(p, compute_units()).workspace : (int64_t)p.hq * p.lse_rows * 4;
}

extern "C" freqattn_status freqattn_sequence_attention_backward(const freqattn_sequence_shape* s, const freqattn_sequence_rows* rows,
                                                                const freqattn_heads* dout, const freqattn_heads* q, const freqattn_heads* k,
                                                                const freqattn_heads* v, const freqattn_heads* out, const float* lse,
                                                                const freqattn_heads* dq, const freqattn_heads* dk, const freqattn_heads* dv,
                                                                void* workspace, int64_t workspace_bytes, void* stream) {
  return guarded([&]() -> freqattn_status {
    const char* who = "freqattn_sequence_attention_backward";
    SeqParams p;
    const freqattn_status fs = seq_params(who, s, rows, p);
    if (fs != FREQATTN_OK) return fs;
    if (p.nseq == 0) return FREQATTN_OK;
    const bool any_q = p.lse_rows > 0, any_k = p.k_rows > 0;
    if (any_q && (!given(dout) || !given(q) || !given(out) || !given(dq) || !lse)) return fail(FREQATTN_EINVAL, who, "NULL argument");
    if (any_k && (!given(k) || !given(v) || !given(dk) || !given(dv))) return fail(FREQATTN_EINVAL, who, "NULL argument");
    const int64_t need = freqattn_sequence_attention_backward_workspace(s, rows);
    if (need > 0 && (!workspace || workspace_bytes < need)) return fail(FREQATTN_EINVAL, who, "workspace too small");
    if (need > 0 && (uintptr_t)workspace % 16) return fail(FREQATTN_EINVAL, who, "workspace must be 16-byte aligned");
    const int size = size_of(s->dtype);
    p.vec = p.d * size % 16 == 0;
    if (any_q) {
      p.dout = q_ptr(p, dout); p.q = q_ptr(p, q); p.o = q_ptr(p, out); p.dq = q_ptr(p, dq);
      p.vec = p.vec && pieces16(p.dout, size) && pieces16(p.q, size) && pieces16(p.o, size) && pieces16(p.dq, size);
    }
    if (any_k) {
      p.k = k_ptr(p, k); p.v = k_ptr(p, v); p.dk = k_ptr(p, dk); p.dv = k_ptr(p, dv);
      p.vec = p.vec && pieces16(p.k, size) && pieces16(p.v, size) && pieces16(p.dk, size) && pieces16(p.dv, size);
    }
    p.lse = const_cast<float*>(lse);
    p.delta = (float*)workspace;
    const bool fast = s->dtype == FREQATTN_BF16 && p.vec && near(p.q) && near(p.dout) && near(p.k) && near(p.v);
    const SeqPlan plan = seq_bwd_plan(p, compute_units());
    p.part = (float*)((char*)workspace + plan.part_at);
    return launched(fast ? launch_seq_bwd(p, plan, (hipStream_t)stream) : launch_seq_generic_bwd(p, s->dtype, (hipStream_t)stream), who);
  });
}
