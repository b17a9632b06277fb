// Tiles of a cache held in 8 bits on their way into LDS, shared by the kernels of attention over such caches.
#pragma once
#include "seq_mfma.h"
#include "tokens.h"

namespace fa {

namespace seq {

typedef uint4v uint4byte __attribute__((aligned(1)));
typedef uint2v uint2byte __attribute__((aligned(1)));
#define FA_GLOBAL __attribute__((address_space(1)))    // (a choice between two addresses is a load of any address space otherwise)

// A piece of 16 codes, channels c .. c + 15 of a row of d, zeros where row or channels do not exist.  HALF: the channels end in half a piece (head_dim % 16 = 8).
template <bool HALF>
__device__ __forceinline__ uint4v load_piece(const char* p, bool in, int c, int d) {
  if constexpr (HALF) {
    const uint2v lo = *(const FA_GLOBAL uint2byte*)(in && c < d ? p : (const char*)&zero_piece);
    const uint2v hi = *(const FA_GLOBAL uint2byte*)(in && c + 8 < d ? p + 8 : (const char*)&zero_piece);
    return uint4v{lo[0], lo[1], hi[0], hi[1]};
  } else {
    return *(const FA_GLOBAL uint4byte*)(in && c < d ? p : (const char*)&zero_piece);
  }
}
// Eight codes times the scale of byte e (255: the scale is taken as infinity, with which the conversion gives NaN).
__device__ __forceinline__ uint4v widen8(uint32_t lo, uint32_t hi, int e) {
  const float s = __uint_as_float((uint32_t)e << 23);
  return uint4v{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false)),
                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true)),
                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false)),
                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true))};
}

// A tile of KT rows of codes on its way: NP pieces a thread.
template <int D, int NW, int KT, int USE, bool HALF>
struct CodeTile {
  static constexpr int PPR = D / 16, TH = 64 * NW, NP = KT * PPR / TH;
  static_assert(NP >= 1 && KT * PPR % TH == 0 && 64 / PPR <= 16, "");
  uint4v x[NP];
  int e[NP];       // bytes of the scales
  int64_t off;     // of the thread's first piece in a tile
  __device__ __forceinline__ void set(int64_t ts, int tid) { off = (int64_t)(tid / PPR) * ts + 16 * (tid % PPR); }
  // rows key0 .. of a sequence of n > key0 rows at `at` (row 0), d channels; what does not exist is zero
  __device__ __forceinline__ void load(const char* at, int64_t ts, const uint8_t* scales, int hk, int shift, int key0, int n, int d, int wave, int tid) {
    const int c = 16 * (tid % PPR);
    const char* const from = at + (int64_t)key0 * ts;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      e[i] = scales[(int64_t)(min(key0 + (i * TH + wave * 64) / PPR, n - 1) >> shift) * hk];     // (uniform over the wave)
      const char* p = from + (int64_t)(i * (TH / PPR)) * ts + off;
      const bool in = key0 + (i * TH + tid) / PPR < n;
      x[i] = load_piece<HALF>(p, in, c, d);
    }
  }
  __device__ __forceinline__ void store(uint16_t* tile, int tid) const {
    asm volatile("" : "+v"(tid));      // (addresses formed here: kept for the whole loop they would take the operands' registers)
    const int p = tid % PPR;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int r = (i * TH + tid) / PPR;
#pragma unroll
      for (int j = 0; j < 2; ++j)
        *(uint4v*)(tile + r * D + (((2 * p + j) ^ swizzle<D, USE>(r)) << 3)) = widen8(x[i][2 * j], x[i][2 * j + 1], e[i]);
    }
  }
};

// The upper 16 bits of a and b as two bf16 numbers.
__device__ __forceinline__ uint32_t high2(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); }
__device__ __forceinline__ float high(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }

// Eight fp32 numbers as three bf16 numbers each, exactly (but for what falls below the smallest numbers): t[0] + t[1] + t[2].
__device__ __forceinline__ void three_parts(const float (&v)[8], bf16x8 (&t)[3]) {
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = v[i];
#pragma unroll
  for (int term = 0; term < 3; ++term) {
    uint4v w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = high2(x[2 * j], x[2 * j + 1]);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] -= high(x[i]);
    t[term] = __builtin_bit_cast(bf16x8, w);
  }
}
// The same of numbers that may be infinite or NaN: those stay in the first term.
__device__ __forceinline__ void three_terms(const float (&v)[8], bf16x8 (&t)[3]) {
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = v[i] != v[i] ? __builtin_nanf("") : v[i];    // (a NaN that its upper bits show)
#pragma unroll
  for (int term = 0; term < 3; ++term) {
    uint4v w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = high2(x[2 * j], x[2 * j + 1]);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fabsf(x[i]) <= 3.4028235e38f ? x[i] - high(x[i]) : 0.f;
    t[term] = __builtin_bit_cast(bf16x8, w);
  }
}

// Eight values with zeros in place of those that are not finite: what the terms behind the first are multiplied by where a result was not finite.  Those may be zero where the number
// itself is not, and an infinite value counts once.
__device__ __forceinline__ bf16x8 finite8(const bf16x8& v) {
  uint4v w = __builtin_bit_cast(uint4v, v);
#pragma unroll
  for (int j = 0; j < 4; ++j)
    w[j] = ((w[j] & 0x7f80u) == 0x7f80u ? 0u : (w[j] & 0xffffu)) | ((w[j] & 0x7f800000u) == 0x7f800000u ? 0u : (w[j] & 0xffff0000u));
  return __builtin_bit_cast(bf16x8, w);
}

}  // namespace seq

}  // namespace fa
