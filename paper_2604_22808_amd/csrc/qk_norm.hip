// Rotary positions and per-head norms of queries and keys, forward and backward.
//
//   r = (mean_c x_c^2 + eps)^-1/2,  y = R(p) (x r w)                 R(p): turns pair i of the channels by p * theta_i, times the amplitude
//   backward: g = R(p)^T dy,  dw = sum g x r,  dx = r (g w - x r^2 mean_c(g w x))
//
// Bound by memory (forward 409-424 us for 131,072 tokens x 32 heads x 128 in bf16, 5.1-5.25 TB/s; 166-178 for 65,536 x 48 x 64, 4.5-4.8; backward 646-720 and
// 300, 4.0-5.0; fp32, 65,536 x 32 x 128: forward 410, backward 615, both 5.2; a 2 GiB copy runs at 5.0): every element is read once (backward: x and dy) and written once.  A head's channels lie on LPR lanes, eight
// per lane: four pairs, so that no channel has to change lanes for the rotation - in the HALF layout a lane loads four channels of the first half
// and their four partners of the second.  The sums of the norm go through LPR lanes in registers.  A wave takes STEPS x 64 / LPR heads of
// one token (all its loads go out before the first is used) and computes the token's sines and cosines once for all of them.
// Angles: see RotTable; sine and cosine are Taylor sums on an eighth of a turn, |error| < 2^-23 (1.84 * 2^-24 the largest of 4 million angles).
#include <hip/hip_runtime.h>

#include "heads.h"

namespace fa {

typedef unsigned int uint2v __attribute__((ext_vector_type(2)));
typedef unsigned int uint4v __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));

struct Bf16 { uint16_t u; };

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(Bf16 x) { return __uint_as_float((uint32_t)x.u << 16); }
template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ float narrow<float>(float x) { return x; }
template <> __device__ __forceinline__ Bf16 narrow<Bf16>(float x) { return Bf16{__builtin_bit_cast(uint16_t, (__bf16)x)}; }   // to nearest, ties to even

// Sine and cosine of u / 2^32 turns, times amp.
__device__ __forceinline__ void sincos_turns(uint32_t u, float amp, float& s, float& c) {
  const uint32_t quarter = (u + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(u - (quarter << 30)) * 1.46291807926715968e-9f;   // 2 pi / 2^32: within pi / 4
  const float x2 = x * x;
  const float ps = x * (1.f + x2 * (-1.f / 6 + x2 * (1.f / 120 + x2 * (-1.f / 5040 + x2 * (1.f / 362880)))));
  const float pc = 1.f + x2 * (-0.5f + x2 * (1.f / 24 + x2 * (-1.f / 720 + x2 * (1.f / 40320 + x2 * (-1.f / 3628800)))));
  s = (quarter & 1) ? pc : ps;
  c = (quarter & 1) ? ps : pc;
  s = (quarter & 2) ? -s : s;
  c = ((quarter + 1) & 2) ? -c : c;
  s *= amp;
  c *= amp;
}

// The eight channels of a lane, as four pairs (a[j], b[j]).
struct Pairs { float4v a, b; };

// Where a lane's channels lie.  SCALAR: pair by pair, for rows that are not made of aligned pieces; else two pieces of four (HALF) or one of eight.
template <bool HALF, bool SCALAR>
struct Place {
  int ca[SCALAR ? 4 : 1], cb[SCALAR ? 4 : 1];
  __device__ __forceinline__ void set(int unit, int half_r) {
    if (SCALAR) {
#pragma unroll
      for (int j = 0; j < (SCALAR ? 4 : 1); ++j) {
        const int i = unit * 4 + j;
        ca[j] = HALF && i < half_r ? i : 2 * i;
        cb[j] = HALF && i < half_r ? i + half_r : 2 * i + 1;
      }
    } else {
      const int i = unit * 4;
      ca[0] = HALF && i < half_r ? i : 2 * i;
      cb[0] = HALF && i < half_r ? i + half_r : 2 * i + 4;
    }
  }
};

template <typename T>
__device__ __forceinline__ void load4(const T* p, float4v& x) {
  if constexpr (sizeof(T) == 4) {
    x = *(const float4v*)p;
  } else {
    const uint2v v = *(const uint2v*)p;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = __uint_as_float((j & 1) ? (v[j >> 1] & 0xffff0000u) : (v[j >> 1] << 16));
  }
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return (uint32_t)narrow<Bf16>(a).u | ((uint32_t)narrow<Bf16>(b).u << 16);
}
template <typename T>
__device__ __forceinline__ void store4(T* p, const float4v& x) {
  if constexpr (sizeof(T) == 4) {
    *(float4v*)p = x;
  } else {
    *(uint2v*)p = uint2v{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
  }
}

// valid: how many of the lane's pairs exist (4, except SCALAR at the end of a head)
template <typename T, bool HALF, bool SCALAR>
__device__ __forceinline__ Pairs load_pairs(const T* row, const Place<HALF, SCALAR>& pl, int valid) {
  Pairs x;
  if (SCALAR) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x.a[j] = j < valid ? widen(row[pl.ca[SCALAR ? j : 0]]) : 0.f;
      x.b[j] = j < valid ? widen(row[pl.cb[SCALAR ? j : 0]]) : 0.f;
    }
  } else if (HALF) {
    load4(row + pl.ca[0], x.a);
    load4(row + pl.cb[0], x.b);
    // (behind the rotated channels the two pieces are neighbours; which channel is whose partner does not matter there)
  } else {
    if constexpr (sizeof(T) == 2) {
      const uint4v v = *(const uint4v*)(row + pl.ca[0]);
#pragma unroll
      for (int j = 0; j < 4; ++j) { x.a[j] = __uint_as_float(v[j] << 16); x.b[j] = __uint_as_float(v[j] & 0xffff0000u); }
    } else {
      const float4v lo = *(const float4v*)(row + pl.ca[0]), hi = *(const float4v*)(row + pl.cb[0]);
      x.a = float4v{lo[0], lo[2], hi[0], hi[2]};
      x.b = float4v{lo[1], lo[3], hi[1], hi[3]};
    }
  }
  return x;
}
template <typename T, bool HALF, bool SCALAR>
__device__ __forceinline__ void store_pairs(T* row, const Place<HALF, SCALAR>& pl, int valid, const Pairs& x) {
  if (SCALAR) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < valid) { row[pl.ca[SCALAR ? j : 0]] = narrow<T>(x.a[j]); row[pl.cb[SCALAR ? j : 0]] = narrow<T>(x.b[j]); }
  } else if (HALF) {
    store4(row + pl.ca[0], x.a);
    store4(row + pl.cb[0], x.b);
  } else if constexpr (sizeof(T) == 2) {
    *(uint4v*)(row + pl.ca[0]) = uint4v{pack_bf16(x.a[0], x.b[0]), pack_bf16(x.a[1], x.b[1]), pack_bf16(x.a[2], x.b[2]), pack_bf16(x.a[3], x.b[3])};
  } else {
    *(float4v*)(row + pl.ca[0]) = float4v{x.a[0], x.b[0], x.a[1], x.b[1]};
    *(float4v*)(row + pl.cb[0]) = float4v{x.a[2], x.b[2], x.a[3], x.b[3]};
  }
}

// Sum over the LPR lanes of a head, on all of them.  Lanes of a quad, then of eight and sixteen (mirrored: the other half holds one value), then across.
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, true));
}
template <int LPR>
__device__ __forceinline__ float row_sum(float x) {
  x += dpp<0xb1>(x);
  x += dpp<0x4e>(x);
  if (LPR >= 8) x += dpp<0x141>(x);
  if (LPR >= 16) x += dpp<0x140>(x);
  if (LPR >= 32) {
    const auto sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  }
  if (LPR >= 64) {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  }
  return x;
}
// (mean + eps)^-1/2: the instruction is within one step, the scaled argument is a normal number unless mean and eps are both about zero
__device__ __forceinline__ float inv_norm(float ss, float inv_d, float eps) {
  const float m = __builtin_fmaf(ss, inv_d, eps);
  return m < 1e-30f ? 1.f / sqrtf(m) : __builtin_amdgcn_rsqf(m);
}

// The rotation of a lane's pairs at one token.
struct Turn { float s[4], c[4]; };

// What a lane knows of its pairs' rotation, fixed for the launch.
struct LaneRot { uint32_t lo[4], hi[4], axis; bool on[4]; };    // axis: a byte each

__device__ __forceinline__ LaneRot lane_rot(const RotTable& t, int unit) {
  LaneRot l;
  l.axis = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = unit * 4 + j;
    l.on[j] = i < t.half;
    const int at = l.on[j] ? i : 0;
    l.lo[j] = (uint32_t)t.turn[at];
    l.hi[j] = (uint32_t)(t.turn[at] >> 32);
    l.axis |= (uint32_t)t.axis[at] << (8 * j);
  }
  return l;
}

__device__ __forceinline__ Turn turn_at(const QkParams& p, const RotTable& t, const LaneRot& l, int b, int n) {
  int at[4] = {n, 0, 0, 0};
  if (p.pos) {
    const int32_t* q = p.pos + (int64_t)b * p.pos_bs + (int64_t)n * t.axes;
    at[0] = q[0];
#pragma unroll
    for (int a = 1; a < 4; ++a)
      if (a < t.axes) at[a] = q[a];
  } else if (t.axes > 1 || t.grid[0]) {
    uint32_t rest = (uint32_t)n;
#pragma unroll
    for (int a = 3; a > 0; --a)
      if (a < t.axes) { at[a] = (int)(rest % t.grid[a]); rest /= t.grid[a]; }
    at[0] = (int)rest;
  }
  Turn r;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t axis = l.axis >> (8 * j) & 3u;
    const int pos = axis == 0 ? at[0] : axis == 1 ? at[1] : axis == 2 ? at[2] : at[3];
    const uint32_t u = __umulhi((uint32_t)pos, l.lo[j]) + (uint32_t)pos * l.hi[j] - (pos < 0 ? l.lo[j] : 0u);
    sincos_turns(u, t.amplitude, r.s[j], r.c[j]);
  }
  return r;
}

__device__ __forceinline__ void rotate(Pairs& x, const Turn& t, const LaneRot& l, float sign) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (l.on[j]) {   // (channels that do not turn keep their bits, infinities too)
      const float a = x.a[j], b = x.b[j], s = sign * t.s[j];
      x.a[j] = a * t.c[j] - b * s;
      x.b[j] = b * t.c[j] + a * s;
    }
}

// A lane's pairs as they lie in memory (loads that nothing waits for yet).
template <typename T, bool HALF, bool SCALAR>
struct Raw {
  Pairs x;    // fp32 and single values: as they are
  __device__ __forceinline__ void load(const T* row, const Place<HALF, SCALAR>& pl, int valid) { x = load_pairs<T, HALF, SCALAR>(row, pl, valid); }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int j = 0; j < 4; ++j) x.a[j] = x.b[j] = 0.f;
  }
  __device__ __forceinline__ Pairs get() const { return x; }
};
template <bool HALF>
struct Raw<Bf16, HALF, false> {
  uint4v v;
  __device__ __forceinline__ void load(const Bf16* row, const Place<HALF, false>& pl, int) {
    if (HALF) {
      const uint2v a = *(const uint2v*)(row + pl.ca[0]), b = *(const uint2v*)(row + pl.cb[0]);
      v = uint4v{a[0], a[1], b[0], b[1]};
    } else {
      v = *(const uint4v*)(row + pl.ca[0]);
    }
  }
  __device__ __forceinline__ void zero() { v = uint4v{0u, 0u, 0u, 0u}; }
  __device__ __forceinline__ Pairs get() const {
    Pairs x;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (HALF) {
        x.a[j] = __uint_as_float((j & 1) ? (v[j >> 1] & 0xffff0000u) : (v[j >> 1] << 16));
        x.b[j] = __uint_as_float((j & 1) ? (v[2 + (j >> 1)] & 0xffff0000u) : (v[2 + (j >> 1)] << 16));
      } else {
        x.a[j] = __uint_as_float(v[j] << 16);
        x.b[j] = __uint_as_float(v[j] & 0xffff0000u);
      }
    }
    return x;
  }
};

template <typename T, bool HALF, bool SCALAR>
__device__ __forceinline__ Pairs load_weight(const void* w, const Place<HALF, SCALAR>& pl, int valid, bool live) {
  Pairs x;
  if (w && live) return load_pairs<T, HALF, SCALAR>((const T*)w, pl, valid);
#pragma unroll
  for (int j = 0; j < 4; ++j) x.a[j] = x.b[j] = 1.f;
  return x;
}

// How a launch cuts the work.  An item (one wave) is a token - or `tpw` tokens, where a token has fewer heads than a wave has rows - and 64 / LPR * STEPS heads of
// each tensor.  Head groups are slowest: neighbouring waves take neighbouring tokens of the same heads.
struct Items { int tpw, head_groups; uint32_t n, per_group; };
enum : int64_t { MAX_ITEMS = (int64_t)1 << 25 };   // a launch has fewer than 2^32 threads

template <typename T, int LPR, bool HALF, bool SCALAR, int STEPS>
__global__ void __launch_bounds__(256) k_qk(QkParams p, const RotTable t, Items it) {
  constexpr int RPW = 64 / LPR;
  const int lane = threadIdx.x & 63, unit = lane % LPR, hr = lane / LPR;
  const uint32_t item = blockIdx.x * 4u + (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (item >= it.n) return;
  const uint32_t hg = item / it.per_group, tg = item - hg * it.per_group;
  const int most = p.heads[0] > p.heads[1] ? p.heads[0] : p.heads[1];
  const int sub = it.tpw > 1 ? hr / most : 0, h_base = (int)hg * RPW * STEPS, h_lane = it.tpw > 1 ? hr - sub * most : h_base + hr;
  const uint32_t token = tg * (uint32_t)it.tpw + (uint32_t)sub;    // (2^25 items of at most 64 tokens)
  const int valid_pairs = p.d / 2 - unit * 4;
  const int valid = valid_pairs < 0 ? 0 : valid_pairs > 4 ? 4 : valid_pairs;
  const bool live = valid > 0 && sub < it.tpw && token < (uint32_t)p.batch * (uint32_t)p.tokens;
  const int b = live ? (int)(token / (uint32_t)p.tokens) : 0, n = live ? (int)(token - (uint32_t)b * (uint32_t)p.tokens) : 0;
  Place<HALF, SCALAR> pl;
  pl.set(unit, t.half);
  const LaneRot lr = lane_rot(t, unit);

  // all loads first (a step whose heads do not exist is skipped by the whole wave)
  Pairs x[2][STEPS];
#pragma unroll
  for (int w = 0; w < 2; ++w)
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      if (h_base + s * RPW >= p.heads[w]) continue;
      const int h = h_lane + s * RPW;
      if (live && h < p.heads[w]) {
        const HeadsPtr& v = p.in[w];
        x[w][s] = load_pairs<T, HALF, SCALAR>((const T*)v.p + (int64_t)b * v.bs + (int64_t)n * v.ts + (int64_t)h * v.hs, pl, valid);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[w][s].a[j] = x[w][s].b[j] = 0.f;
      }
    }
  Turn tn;
  if (t.half > 0) tn = turn_at(p, t, lr, b, n);
  const float sign = p.inverse ? -1.f : 1.f, inv_d = 1.f / (float)p.d;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    if (h_base >= p.heads[w]) continue;
    Pairs wt;
    if (p.norm) wt = load_weight<T, HALF, SCALAR>(p.w[w], pl, valid, live);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      if (h_base + s * RPW >= p.heads[w]) continue;
      const int h = h_lane + s * RPW;
      Pairs& y = x[w][s];
      if (p.norm) {
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) ss += y.a[j] * y.a[j] + y.b[j] * y.b[j];
        const float r = inv_norm(row_sum<LPR>(ss), inv_d, p.eps);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          y.a[j] *= r * wt.a[j];
          y.b[j] *= r * wt.b[j];
        }
      }
      if (live && h < p.heads[w]) {
        if (t.half > 0) rotate(y, tn, lr, sign);
        const HeadsPtr& v = p.out[w];
        store_pairs<T, HALF, SCALAR>((T*)v.p + (int64_t)b * v.bs + (int64_t)n * v.ts + (int64_t)h * v.hs, pl, valid, y);
      }
    }
  }
}

// Backward: waves walk items, cut as the forward pass cuts them, and keep their lanes' sums of dw in registers.  A block adds its waves' sums in a fixed order and
// stores one row of partial sums per tensor; k_qk_weights adds the rows.
template <typename T, int LPR, bool HALF, bool SCALAR, int STEPS>
__global__ void __launch_bounds__(256, 3) k_qk_backward(QkParams p, const RotTable t, Items it) {
  constexpr int RPW = 64 / LPR;
  const int lane = threadIdx.x & 63, unit = lane % LPR, hr = lane / LPR, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int most = p.heads[0] > p.heads[1] ? p.heads[0] : p.heads[1];
  const int valid_pairs = p.d / 2 - unit * 4;
  const int valid = valid_pairs < 0 ? 0 : valid_pairs > 4 ? 4 : valid_pairs;
  Place<HALF, SCALAR> pl;
  pl.set(unit, t.half);
  const LaneRot lr = lane_rot(t, unit);
  Pairs dw[2];
#pragma unroll
  for (int w = 0; w < 2; ++w)
#pragma unroll
    for (int j = 0; j < 4; ++j) dw[w].a[j] = dw[w].b[j] = 0.f;
  const int sub = it.tpw > 1 ? hr / most : 0;
  const float inv_d = 1.f / (float)p.d;

  // The rows of the next tensor or item are requested before the present ones are worked on.
  struct At { int h_base, h_lane, b, n; bool live; };
  auto place = [&](uint32_t item) {
    const uint32_t hg = item / it.per_group, tg = item - hg * it.per_group;
    const uint32_t token = tg * (uint32_t)it.tpw + (uint32_t)sub;
    At at;
    at.h_base = (int)hg * RPW * STEPS;
    at.h_lane = it.tpw > 1 ? hr - sub * most : at.h_base + hr;
    at.live = valid > 0 && sub < it.tpw && token < (uint32_t)p.batch * (uint32_t)p.tokens;
    at.b = at.live ? (int)(token / (uint32_t)p.tokens) : 0;
    at.n = at.live ? (int)(token - (uint32_t)at.b * (uint32_t)p.tokens) : 0;
    return at;
  };
  auto row = [&](const HeadsPtr& v, const At& at, int h) { return (T*)const_cast<char*>(v.p) + (int64_t)at.b * v.bs + (int64_t)at.n * v.ts + (int64_t)h * v.hs; };
  Raw<T, HALF, SCALAR> rx[2][STEPS], rg[2][STEPS];
  auto request = [&](const At& at, int w) {
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      if (at.h_base + s * RPW >= p.heads[w]) continue;
      const int h = at.h_lane + s * RPW;
      if (at.live && h < p.heads[w]) {
        rx[w][s].load(row(p.in[w], at, h), pl, valid);
        rg[w][s].load(row(p.dy[w], at, h), pl, valid);
      } else {
        rx[w][s].zero();
        rg[w][s].zero();
      }
    }
  };
  auto work = [&](const At& at, int w, const Turn& tn) {
    if (at.h_base >= p.heads[w]) return;
    const Pairs wt = load_weight<T, HALF, SCALAR>(p.w[w], pl, valid, valid > 0);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      if (at.h_base + s * RPW >= p.heads[w]) continue;
      const int h = at.h_lane + s * RPW;
      const Pairs x = rx[w][s].get();
      Pairs g = rg[w][s].get(), gw;
      if (t.half > 0) rotate(g, tn, lr, -1.f);
      float ss = 0.f, gx = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        gw.a[j] = g.a[j] * wt.a[j];
        gw.b[j] = g.b[j] * wt.b[j];
        ss += x.a[j] * x.a[j] + x.b[j] * x.b[j];
        gx += gw.a[j] * x.a[j] + gw.b[j] * x.b[j];
      }
      ss = row_sum<LPR>(ss);
      gx = row_sum<LPR>(gx);
      const float r = inv_norm(ss, inv_d, p.eps);
      const float m = r * r * (gx * inv_d);
      if (at.live && h < p.heads[w]) {
        Pairs o;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          dw[w].a[j] += g.a[j] * (x.a[j] * r);
          dw[w].b[j] += g.b[j] * (x.b[j] * r);
          o.a[j] = r * (gw.a[j] - x.a[j] * m);
          o.b[j] = r * (gw.b[j] - x.b[j] * m);
        }
        store_pairs<T, HALF, SCALAR>(row(p.out[w], at, h), pl, valid, o);
      }
    }
  };
  uint32_t item = 4u * blockIdx.x + wave;
  At at = {};
  if (item < it.n) { at = place(item); request(at, 0); }
  for (; item < it.n; item += 4u * gridDim.x) {
    const At now = at;
    request(now, 1);
    Turn tn;
    if (t.half > 0) tn = turn_at(p, t, lr, now.b, now.n);
    work(now, 0, tn);
    if (item + 4u * gridDim.x < it.n) { at = place(item + 4u * gridDim.x); request(at, 0); }
    work(now, 1, tn);
  }
  if (!p.part) return;
  __shared__ float sums[2][4][8 * LPR];
#pragma unroll
  for (int w = 0; w < 2; ++w)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int o = LPR; o < 64; o <<= 1) { dw[w].a[j] += __shfl_xor(dw[w].a[j], o); dw[w].b[j] += __shfl_xor(dw[w].b[j], o); }
      if (hr == 0) { sums[w][wave][unit * 8 + j] = dw[w].a[j]; sums[w][wave][unit * 8 + 4 + j] = dw[w].b[j]; }
    }
  __syncthreads();
  // back to channel order: slot unit*8 + j is channel a[j], + 4 its partner b[j]
  for (int i = threadIdx.x; i < 2 * p.d; i += 256) {
    const int w = i >= p.d, c = i - w * p.d;
    int pair, second;
    if (HALF && c < 2 * t.half) { second = c >= t.half; pair = c - second * t.half; }
    else if (!HALF || SCALAR) { pair = c >> 1; second = c & 1; }
    else { pair = (c >> 3) * 4 + (c & 3); second = (c >> 2) & 1; }   // (aligned pieces behind the rotated channels of the HALF layout)
    const int slot = (pair >> 2) * 8 + (pair & 3) + 4 * second;
    p.part[(int64_t)blockIdx.x * 2 * p.d + i] = (sums[w][0][slot] + sums[w][1][slot]) + (sums[w][2][slot] + sums[w][3][slot]);
  }
}

// dw[c] = sum over the blocks' rows; a block adds 32 channels of one tensor, 32 threads a channel.
__global__ void __launch_bounds__(1024) k_qk_weights(const float* __restrict__ part, int d, int blocks, float* dwq, float* dwk) {
  float* dst = blockIdx.y ? dwk : dwq;
  if (!dst) return;   // (uniform over the block)
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), row = threadIdx.x >> 5;
  float s = 0.f;
  if (c < d) {
#pragma unroll 8
    for (int i = row; i < blocks; i += 32) s += part[((int64_t)i * 2 + blockIdx.y) * d + c];
  }
  __shared__ float acc[32][33];
  acc[row][threadIdx.x & 31] = s;
  __syncthreads();
  if (row == 0 && c < d) {
    float r = 0.f;
    for (int i = 0; i < 32; ++i) r += acc[i][threadIdx.x & 31];
    dst[c] = r;
  }
}

static bool pieces(const HeadsPtr& v, int bytes, int size) {
  return (uintptr_t)v.p % bytes == 0 && (v.bs * size) % bytes == 0 && (v.ts * size) % bytes == 0 && (v.hs * size) % bytes == 0;
}

static Items make_items(int64_t tokens, int heads, int rpw, int steps) {
  Items it;
  it.tpw = heads < rpw ? rpw / heads : 1;
  it.head_groups = it.tpw > 1 ? 1 : (int)(((int64_t)heads + rpw * steps - 1) / (rpw * steps));
  const int64_t groups = (tokens + it.tpw - 1) / it.tpw;
  const bool fits = groups <= MAX_ITEMS / it.head_groups;     // (their product may pass 64 bits)
  it.per_group = groups > 0 && fits ? (uint32_t)groups : 1u;
  it.n = fits ? (uint32_t)(groups * it.head_groups) : ~0u;
  return it;
}

template <typename T, int LPR, bool HALF, bool SCALAR, int STEPS>
static hipError_t fwd_s(const QkParams& p, const RotTable& t, hipStream_t st) {
  const Items it = make_items((int64_t)p.batch * p.tokens, p.heads[0] > p.heads[1] ? p.heads[0] : p.heads[1], 64 / LPR, STEPS);
  if (it.n == ~0u) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((k_qk<T, LPR, HALF, SCALAR, STEPS>), dim3((it.n + 3) / 4), dim3(256), 0, st, p, t, it);
  return hipGetLastError();
}
template <typename T, int LPR, bool HALF, bool SCALAR>
static hipError_t fwd(const QkParams& p, const RotTable& t, int num_cu, hipStream_t st) {
  // Four steps of each tensor share a token's sines and have their loads in flight together; where that leaves fewer than 8 waves per compute unit, one
  // step per wave.
  const int64_t tokens = (int64_t)p.batch * p.tokens, most = p.heads[0] > p.heads[1] ? p.heads[0] : p.heads[1];
  const int64_t groups = (most + 4 * (64 / LPR) - 1) / (4 * (64 / LPR));
  if (most <= 64 / LPR || tokens < ((int64_t)num_cu * 8 + groups - 1) / groups) return fwd_s<T, LPR, HALF, SCALAR, 1>(p, t, st);
  return fwd_s<T, LPR, HALF, SCALAR, 4>(p, t, st);
}
template <typename T, int LPR, bool HALF, bool SCALAR>
static hipError_t bwd(const QkParams& p, const RotTable& t, float* const dw[2], int num_cu, hipStream_t st) {
  constexpr int STEPS = SCALAR ? 1 : sizeof(T) == 2 ? 4 : 2;    // (rows in flight, by the registers that they take)
  const Items it = make_items((int64_t)p.batch * p.tokens, p.heads[0] > p.heads[1] ? p.heads[0] : p.heads[1], 64 / LPR, STEPS);
  if (it.n == ~0u) return hipErrorInvalidConfiguration;
  int64_t blocks = ((int64_t)it.n + 3) / 4;     // as many as are resident, at most (see launch bounds)
  if (blocks > 3 * num_cu) blocks = 3 * num_cu;
  if (blocks > QK_BWD_BLOCKS) blocks = QK_BWD_BLOCKS;
  if (blocks < 1) blocks = 1;
  hipLaunchKernelGGL((k_qk_backward<T, LPR, HALF, SCALAR, STEPS>), dim3((unsigned)blocks), dim3(256), 0, st, p, t, it);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.part) return e;
  hipLaunchKernelGGL(k_qk_weights, dim3((unsigned)((p.d + 31) / 32), p.heads[1] > 0 ? 2u : 1u), dim3(1024), 0, st, p.part, p.d, (int)blocks, dw[0], dw[1]);
  return hipGetLastError();
}

// The variant that fits a call: lanes per head, and whether rows are made of aligned pieces.
template <typename T, bool HALF, typename F>
static hipError_t dispatch(const QkParams& p, const RotTable& t, bool backward, F&& go) {
  const int size = sizeof(T), piece = HALF ? 4 * size : 16;
  bool al = p.d % 8 == 0 && (!HALF || t.half % 4 == 0);
  for (int w = 0; w < 2; ++w)
    if (p.heads[w] > 0) {
      al = al && pieces(p.in[w], piece, size) && pieces(p.out[w], piece, size) && (!backward || pieces(p.dy[w], piece, size));
      al = al && (!p.w[w] || (uintptr_t)p.w[w] % piece == 0);
    }
  const int lanes = (p.d / 2 + 3) / 4;
#define FA_QK(L_, S_) if (lanes <= L_ && al == !S_) return go(std::integral_constant<int, L_>(), std::integral_constant<bool, S_>());
  FA_QK(4, false) FA_QK(8, false) FA_QK(16, false) FA_QK(32, false) FA_QK(64, false) FA_QK(16, true) FA_QK(64, true)
#undef FA_QK
  return hipErrorInvalidValue;
}

hipError_t launch_qk(const QkParams& p, const RotTable& t, int dtype, int num_cu, hipStream_t st) {
  auto with = [&](auto type, auto half) {
    using T = decltype(type);
    return dispatch<T, half.value>(p, t, false, [&](auto lanes, auto scalar) { return fwd<T, lanes.value, half.value, scalar.value>(p, t, num_cu, st); });
  };
  if (dtype == FREQATTN_BF16) return t.interleaved ? with(Bf16{}, std::false_type{}) : with(Bf16{}, std::true_type{});
  return t.interleaved ? with(0.f, std::false_type{}) : with(0.f, std::true_type{});
}

hipError_t launch_qk_backward(const QkParams& p, const RotTable& t, int dtype, float* const dw[2], int num_cu, hipStream_t st) {
  auto with = [&](auto type, auto half) {
    using T = decltype(type);
    return dispatch<T, half.value>(p, t, true, [&](auto lanes, auto scalar) { return bwd<T, lanes.value, half.value, scalar.value>(p, t, dw, num_cu, st); });
  };
  if (dtype == FREQATTN_BF16) return t.interleaved ? with(Bf16{}, std::false_type{}) : with(Bf16{}, std::true_type{});
  return t.interleaved ? with(0.f, std::false_type{}) : with(0.f, std::true_type{});
}

}  // namespace fa
