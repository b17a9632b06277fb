// 8-bit codes of token rows: a = max_c |x_c|, code_c = 127 x_c / a to the nearest whole number, ties to even, scale = a / 127.
//
// Codes are exact: what fp32 leaves within 10^-4 of the border between two codes is decided in fp64, where 254 |x| and (2 k + 1) a have no rounding.  (x = a / 2
// lies on a border, at 63.5, and is no rare value in bf16.)  Bound by memory: a row is read once, into registers, and its codes are written; only rows of more than
// 16,384 channels are read twice.  131,072 x 2048 bf16 143 us (5.6 TB/s), 65,536 x 1536 57 (5.3), 65,536 x 2048 fp32 116 (5.8), 300,000 x 301 fp32 101 (4.5).
#include "rows.h"
#include "tokens.h"

namespace fa {

using namespace rows;

namespace {

constexpr uint32_t INF_BITS = 0x7f800000u;

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }   // (orders as unsigned numbers, NaN last)
__device__ __forceinline__ float larger(float a, float b) {
  const uint32_t u = __float_as_uint(a), v = __float_as_uint(b);
  return __uint_as_float(u > v ? u : v);
}

// What the codes of a row are made with.
struct Coder {
  float up, inv, scale;
  double top;
  __device__ __forceinline__ void set(uint32_t bits) {
    const float a = __uint_as_float(bits);
    const bool odd = bits >= INF_BITS, some = bits > 0 && !odd;
    scale = odd ? __builtin_nanf("") : a / 127.f;
    up = a < 0x1p-60f ? 0x1p64f : 1.f;                 // 127 / a stays finite
    inv = some ? 127.f / (a * up) : 0.f;
    top = a;
  }
};

template <typename T>
__device__ __forceinline__ void store_codes(int8_t* row, int c, int n, const Piece<T>& x, const Coder& k) {
  float q[PW<T>];
  bool close = false;
#pragma unroll
  for (int j = 0; j < PW<T>; ++j) {
    const float t = k.inv == 0.f ? 0.f : x.get(j) * k.up * k.inv;    // (rows of zeros, or with an infinity or NaN: zeros)
    q[j] = rintf(t);
    close = close || fabsf(t - q[j]) > 0.4999f;
  }
  if (close) {
#pragma unroll
    for (int j = 0; j < PW<T>; ++j) {
      const float t = fabsf(x.get(j) * k.up * k.inv);
      if (fabsf(t - rintf(t)) > 0.4999f) {
        const float lower = floorf(t);
        const double a = 254.0 * fabs((double)x.get(j)), b = (2.0 * lower + 1.0) * k.top;
        const float whole = a > b || (a == b && ((int)lower & 1)) ? lower + 1.f : lower;
        q[j] = x.get(j) < 0.f ? -whole : whole;
      }
    }
  }
  uint32_t w[PW<T> / 4];
#pragma unroll
  for (int i = 0; i < PW<T> / 4; ++i) {
    w[i] = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[i] |= ((uint32_t)(int)q[4 * i + j] & 0xffu) << (8 * j);
  }
  if (c + PW<T> <= n) {
    if constexpr (PW<T> == 8) *(uint2any*)(row + c) = uint2v{w[0], w[1]};
    else *(u32any*)(row + c) = w[0];
  } else if (c < n) {      // the last codes: four, two, one
    const int left = n - c;
    uint32_t x = w[0];
    if (PW<T> == 8 && (left & 4)) { *(u32any*)(row + c) = x; x = w[PW<T> / 4 - 1]; }
    if (left & 2) { *(u16any*)(row + c + (left & 4)) = (uint16_t)x; x >>= 16; }
    if (left & 1) row[c + (left & 6)] = (int8_t)x;
  }
}

template <typename T, int LPR, int W, int PT>
__global__ void __launch_bounds__((Place<T, LPR, W, PT>::THREADS)) k_quantize_rows(CodeParams p) {
  using At = Place<T, LPR, W, PT>;
  __shared__ uint32_t lds[2][W];
  At at;
  at.set();
  const int n = p.channels;
  int turn = 0;
  Piece<T> x[PT];
  for (int64_t i = (int64_t)blockIdx.x * At::STEP; i < p.n; i += (int64_t)gridDim.x * At::STEP) {
    const int64_t r = i + at.row;
    const bool live = r < p.n;
    const T* row = row_of<T>(p.x, p.rows, live ? r : 0);
    uint32_t bits = 0;
#pragma unroll
    for (int k = 0; k < PT; ++k) {
      x[k].load(row, at.channel(k), live ? n : 0);
#pragma unroll
      for (int j = 0; j < PW<T>; ++j) bits = max(bits, magnitude(x[k].get(j)));
    }
    bits = __float_as_uint(over_lanes<LPR>(__uint_as_float(bits), larger));
    if constexpr (W > 1) {
      if ((threadIdx.x & 63) == 0) lds[turn][threadIdx.x >> 6] = bits;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < W; ++w) bits = max(bits, lds[turn][w]);
      turn ^= 1;
    }
    Coder k;
    k.set(bits);
    if (!live) continue;
    int8_t* to = row_of<int8_t>(p.codes, p.rows, r);
#pragma unroll
    for (int i2 = 0; i2 < PT; ++i2) store_codes<T>(to, at.channel(i2), n, x[i2], k);
    if (at.lane == 0) p.scales[r] = k.scale;
  }
}

// Rows that no registers hold: read twice.
template <typename T>
__global__ void __launch_bounds__(1024) k_quantize_long(CodeParams p) {
  __shared__ uint32_t lds[16];
  const int n = p.channels;
  for (int64_t r = blockIdx.x; r < p.n; r += gridDim.x) {
    const T* row = row_of<T>(p.x, p.rows, r);
    uint32_t bits = 0;
    Piece<T> x;
    for (int c = threadIdx.x * PW<T>; c < n; c += 1024 * PW<T>) {
      x.load(row, c, n);
#pragma unroll
      for (int j = 0; j < PW<T>; ++j) bits = max(bits, magnitude(x.get(j)));
    }
    bits = __float_as_uint(over_lanes<64>(__uint_as_float(bits), larger));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = bits;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 16; ++w) bits = max(bits, lds[w]);
    Coder k;
    k.set(bits);
    int8_t* to = row_of<int8_t>(p.codes, p.rows, r);
    for (int c = threadIdx.x * PW<T>; c < n; c += 1024 * PW<T>) {
      x.load(row, c, n);
      store_codes<T>(to, c, n, x, k);
    }
    if (threadIdx.x == 0) p.scales[r] = k.scale;
  }
}

// Waves for each compute unit, at most: rows that are dealt out as workgroups end keep memory busier than fixed shares (32 / 256 waves: 131,072 x 2048 bf16 156 / 143 us, 65,536 x 4096
// 184 / 145, 100,000 x 1024 64 / 58).
constexpr int WAVES = 256;

template <typename T>
hipError_t go(const CodeParams& p, int num_cu, hipStream_t st) {
  if (p.channels > NORM_MOST_CHANNELS) {
    const int64_t blocks = blocks_of(p.n, 1, 1, 1024, WAVES, num_cu);
    hipLaunchKernelGGL(k_quantize_long<T>, dim3((unsigned)blocks), dim3(1024), 0, st, p);
    return hipGetLastError();
  }
  auto launch = [&](auto l, auto w, auto pt) {
    using At = Place<T, l.value, w.value, pt.value>;
    const int64_t blocks = blocks_of(p.n, 1, At::STEP, At::THREADS, WAVES, num_cu);
    hipLaunchKernelGGL((k_quantize_rows<T, l.value, w.value, pt.value>), dim3((unsigned)blocks), dim3(At::THREADS), 0, st, p);
    return hipGetLastError();
  };
  constexpr int U = 8 / PW<T>;
  using std::integral_constant;
  // (one wave with four pieces a lane here too, without a barrier: 131,072 x 2048 bf16 182 us on two waves, 156 on one)
  if (p.channels > 1536 && p.channels <= 2048) return launch(integral_constant<int, 64>(), integral_constant<int, 1>(), integral_constant<int, 4 * U>());
  return for_channels<T, PACKED>(p.channels, launch);
}

}  // namespace

hipError_t launch_quantize_rows(const CodeParams& p, int dtype, int num_cu, hipStream_t st) {
  return dtype == FREQATTN_BF16 ? go<Bf16>(p, num_cu, st) : go<float>(p, num_cu, st);
}

}  // namespace fa
