// Rows of a token tensor in registers, shared by the kernels that walk whole rows (layer norm, 8-bit codes).
//
// A row of `channels` lies on LANES = LPR * W lanes (LPR lanes of a wave, or W whole waves), as pieces of 16 bytes: lane l holds pieces l, l + LANES, .. of the
// row, PT of them at most.  Pieces are loaded whole wherever the row starts (addresses of any element's alignment); channels behind the last whole piece are
// loaded in parts of it, and what lies behind the row's end is zero.  Rows are counted in 32 bits.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "tokens.h"

namespace fa {
namespace rows {

struct Bf16 { uint16_t u; };

typedef unsigned int uint4v __attribute__((ext_vector_type(4)));
typedef uint4v uint4any __attribute__((aligned(2)));    // at any element's address
typedef uint4v uint4byte __attribute__((aligned(1)));
typedef unsigned int uint2v __attribute__((ext_vector_type(2)));
typedef uint2v uint2any __attribute__((aligned(1)));
typedef uint2v uint2two __attribute__((aligned(2)));
typedef uint32_t u32any __attribute__((aligned(1)));
typedef uint16_t u16any __attribute__((aligned(1)));
typedef uint32_t u32two __attribute__((aligned(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float4v float4any __attribute__((aligned(4)));

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(Bf16 x) { return __uint_as_float((uint32_t)x.u << 16); }
template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ float narrow<float>(float x) { return x; }
template <> __device__ __forceinline__ Bf16 narrow<Bf16>(float x) { return Bf16{__builtin_bit_cast(uint16_t, (__bf16)x)}; }   // to nearest, ties to even

template <typename T> constexpr int PW = 16 / (int)sizeof(T);   // channels of a piece

// One piece as it lies in memory.
template <typename T>
struct Piece {
  uint4v raw;
  // channels c .. c + PW - 1 of a row of n; zeros from n on
  __device__ __forceinline__ void load(const T* row, int c, int n) {
    raw = uint4v{0u, 0u, 0u, 0u};
    if (c + PW<T> <= n) {
      raw = *(const uint4any*)(row + c);
    } else if (c < n) {      // the last channels: four, two, one
      const int left = n - c;
      const uint32_t* const at = (const uint32_t*)(row + c);
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 3; ++j)
          if (j < left) raw[j] = *(const u32two*)(at + j);
      } else {
        uint32_t two = 0, one = 0;
        if (left & 4) { const uint2v x = *(const uint2two*)at; raw[0] = x[0]; raw[1] = x[1]; }
        if (left & 2) two = *(const u32two*)(row + c + (left & 4));
        if (left & 1) one = row[c + (left & 6)].u;
        const uint32_t x = (left & 2) ? two : one, y = (left & 2) ? one : 0u;
        raw[0] = (left & 4) ? raw[0] : x;
        raw[1] = (left & 4) ? raw[1] : y;
        raw[2] = (left & 4) ? x : 0u;
        raw[3] = (left & 4) ? y : 0u;
      }
    }
  }
  __device__ __forceinline__ float get(int j) const {   // (j a constant)
    if constexpr (sizeof(T) == 4) return __uint_as_float(raw[j]);
    else return __uint_as_float((j & 1) ? (raw[j >> 1] & 0xffff0000u) : (raw[j >> 1] << 16));
  }
  __device__ __forceinline__ void set(int j, float a, float b) {   // channels j, j + 1, j even
    if constexpr (sizeof(T) == 4) {
      raw[j] = __float_as_uint(a);
      raw[j + 1] = __float_as_uint(b);
    } else {
      raw[j >> 1] = (uint32_t)narrow<T>(a).u | ((uint32_t)narrow<T>(b).u << 16);
    }
  }
  __device__ __forceinline__ void store(T* row, int c, int n) const {
    if (c + PW<T> <= n) {
      *(uint4any*)(row + c) = raw;
    } else if (c < n) {
      const int left = n - c;
      uint32_t* const at = (uint32_t*)(row + c);
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 3; ++j)
          if (j < left) *(u32two*)(at + j) = raw[j];
      } else {
        if (left & 4) *(uint2two*)at = uint2v{raw[0], raw[1]};
        const uint32_t x = (left & 4) ? raw[2] : raw[0], y = (left & 4) ? raw[3] : raw[1];
        if (left & 2) *(u32two*)(row + c + (left & 4)) = x;
        if (left & 1) row[c + (left & 6)].u = (uint16_t)((left & 2) ? y : x);
      }
    }
  }
};

// Sums over the LPR lanes of a row in a wave: neighbours through the data-parallel primitives of the vector unit, halves through swaps.
template <int LPR, typename F>
__device__ __forceinline__ float over_lanes(float x, F&& f) {
#define FA_STEP(CTRL) x = f(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true)))
  if constexpr (LPR >= 2) FA_STEP(0xb1);     // lane ^ 1
  if constexpr (LPR >= 4) FA_STEP(0x4e);     // lane ^ 2
  if constexpr (LPR >= 8) FA_STEP(0x141);    // the other half of 8 (mirrored; its lanes agree)
  if constexpr (LPR >= 16) FA_STEP(0x140);   // the other half of 16
#undef FA_STEP
  if constexpr (LPR >= 32) {
    const uint32_t b = __float_as_uint(x);
    const auto s = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    x = f(__uint_as_float(s[0]), __uint_as_float(s[1]));
  }
  if constexpr (LPR >= 64) {
    const uint32_t b = __float_as_uint(x);
    const auto s = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    x = f(__uint_as_float(s[0]), __uint_as_float(s[1]));
  }
  return x;
}
__device__ __forceinline__ float add(float a, float b) { return a + b; }

// A lane's place: which row of the workgroup's step, which pieces of it.
template <typename T, int LPR, int W, int PT>
struct Place {
  static constexpr bool AHEAD = PT * PW<T> <= 24;    // the next row is requested ahead (longer shares leave no registers for it)
  static constexpr int LANES = LPR * W, STEP = W == 1 ? 4 * (64 / LPR) : 1, THREADS = W == 1 ? 256 : 64 * W;
  int lane, row;     // within the row's lanes; row of the step
  __device__ __forceinline__ void set() {
    lane = W == 1 ? (int)(threadIdx.x % LPR) : (int)threadIdx.x;
    row = W == 1 ? (int)(threadIdx.x / LPR) : 0;
  }
  __device__ __forceinline__ int channel(int i) const { return (lane + i * LANES) * PW<T>; }
};

// Row i of a tensor of batch * rows rows.
template <typename T>
__device__ __forceinline__ T* row_of(const RowsPtr& v, int rows, int64_t i) {
  const int64_t b = (int64_t)((uint32_t)i / (uint32_t)rows);
  return (T*)v.p + b * v.bs + (i - b * rows) * v.rs;
}

// How rows lie.  SPREAD: up to 512 channels on as many lanes as there are pieces of eight.  PACKED: up to 768 on half as many or fewer, two or three such pieces each, so that a wave's sums
// over lanes are of more rows: that gains where vector work bounds them (spread / packed: norm of 60,000 x 173 bf16 19.2 / 13.4 us, 60,000 x 768 36 / 31, 300,000 x 128 27.1 / 25.5; codes of
// the same 18.1 / 11.5, 33 / 26, 34 / 23.5, of 200,000 x 99 fp32 22.4 / 21.0), and loses elsewhere (norm of 200,000 x 99 fp32 28 / 31, 30,000 x 700 30.5 / 33.3).  HALF_PACKED: the
// backward pass, whose registers are more (spread / packed: 60,000 x 173 bf16 33 / 37, 100,000 x 250 fp32 58 / 80, but 60,000 x 768 bf16 87 / 52, 40,000 x 640 53 / 41, 30,000 x 600 fp32 50 / 46).
// Rows of two and four waves likewise: both take three pieces a lane for more than 2048 and 4096 channels, as far as that reaches (20,000 x 2500 bf16 forward 47 / 41, backward 146 / 99, codes 38 / 32; 8000 x 6000
// fp32 forward 74 / 84, backward 143 / 129, codes 40 / 35).
enum Lay { SPREAD, PACKED, HALF_PACKED };
// The variant whose lanes hold a row: go(LPR, W, PT).
template <typename T, Lay LAY, typename F>
auto for_channels(int channels, F&& go) {
  constexpr int U = 8 / PW<T>;      // pieces of eight channels
  const int eights = (channels + 7) / 8;
#define FA_ROWS(L_, W_, P_) if (eights <= (L_) * (W_) * (P_)) return go(std::integral_constant<int, L_>(), std::integral_constant<int, W_>(), std::integral_constant<int, (P_) * U>());
  FA_ROWS(8, 1, 1)
  if constexpr (LAY == PACKED) { FA_ROWS(8, 1, 2) FA_ROWS(8, 1, 3) FA_ROWS(16, 1, 2) FA_ROWS(16, 1, 3) FA_ROWS(32, 1, 2) }
  else { FA_ROWS(16, 1, 1) FA_ROWS(32, 1, 1) FA_ROWS(64, 1, 1) }
  if constexpr (LAY != SPREAD) { FA_ROWS(32, 1, 3) }
  FA_ROWS(64, 1, 2) FA_ROWS(64, 1, 3)
  FA_ROWS(64, 2, 2)
  if constexpr (LAY != SPREAD) { FA_ROWS(64, 2, 3) }
  FA_ROWS(64, 4, 2)
  if constexpr (LAY != SPREAD) { FA_ROWS(64, 4, 3) }
  FA_ROWS(64, 8, 2)
#undef FA_ROWS
  return go(std::integral_constant<int, 64>(), std::integral_constant<int, 8>(), std::integral_constant<int, 4 * U>());
}

// Workgroups of a launch: `waves` for each compute unit, shared by the groups.
inline int64_t blocks_of(int64_t n, int64_t groups, int step, int threads, int waves, int num_cu) {
  const int64_t most = ((int64_t)num_cu * waves * 64 / threads + groups - 1) / groups, all = (n + step - 1) / step;
  return all < most ? all : most;
}

}  // namespace rows
}  // namespace fa
