// Products of rows of 8-bit codes: out[m][n] = s_a[m] s_w[n] sum_k a[m][k] w[n][k] + bias[n], k adjacent in both.  Sums are whole numbers of 32 bits, exact up to 131,071
// channels, so neither their order nor their cut shows in the result; scaling and bias are fp32, rounded once to the output's type.
//
// Three kernels.  Operands are fed to the matrix cores as 16 bytes a lane, k = 16 g .. 16 g + 15 of a product's channels on lane group g; both sides use the same order, so any
// order of the channels will do.
#include "rows.h"
#include "tokens.h"

namespace fa {

using namespace rows;

namespace {

typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int16v __attribute__((ext_vector_type(16)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float4v float4any __attribute__((aligned(4)));

static __device__ const int4v zero_piece = {0, 0, 0, 0};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ unsigned lds_at(const void* p) { return (unsigned)uniform((int)(unsigned)(uintptr_t)(const __attribute__((address_space(3))) void*)p); }
// One wave-wide copy into LDS, 16 bytes a lane, to bytes dst + 16 lane.  Written as assembly because the compiler orders every LDS read behind a copy of this
// kind that it knows of; the kernels wait for their copies themselves.
__device__ __forceinline__ void copy16(const void* src, unsigned dst) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "s"(dst) : "memory", "m0");
}

// Eight results of a row, columns c .. c + 7.
template <typename T>
__device__ __forceinline__ void store8(const ProductParams& p, int64_t row, int c, const int (&acc)[8], float sa) {
  float o[8];
  T* to = (T*)p.out + row * p.out_rs;
  if (c + 8 <= p.outputs) {
    const float4v s0 = *(const float4any*)(p.w_scales + c), s1 = *(const float4any*)(p.w_scales + c + 4);
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = (float)acc[j] * sa * (j < 4 ? s0[j & 3] : s1[j & 3]);
    if (p.bias) {
#pragma unroll
      for (int i = 0; i < 8 / PW<T>; ++i) {
        Piece<T> b;
        b.raw = *(const uint4any*)((const T*)p.bias + c + i * PW<T>);
#pragma unroll
        for (int j = 0; j < PW<T>; ++j) o[i * PW<T> + j] += b.get(j);
      }
    }
#pragma unroll
    for (int i = 0; i < 8 / PW<T>; ++i) {
      Piece<T> x;
#pragma unroll
      for (int j = 0; j < PW<T>; j += 2) x.set(j, o[i * PW<T> + j], o[i * PW<T> + j + 1]);
      *(uint4any*)(to + c + i * PW<T>) = x.raw;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (c + j < p.outputs) {
        const float x = (float)acc[j] * sa * p.w_scales[c + j];
        to[c + j] = narrow<T>(p.bias ? x + widen(((const T*)p.bias)[c + j]) : x);
      }
  }
}

// The accumulators of a 32 x 32 product hold one row a lane and the columns 8 (r / 4) + 4 g + r % 4: after a swap of registers with lane ^ 32 (the same row) a lane has
// 8 neighbouring columns.
template <typename T>
__device__ __forceinline__ void store_tile(const ProductParams& p, const int16v& acc, int64_t row, int col, int g, float sa, bool live) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    int o[8];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const auto sw = __builtin_amdgcn_permlane32_swap((unsigned)acc[8 * j + b], (unsigned)acc[8 * j + 4 + b], false, false);
      o[b] = (int)sw[0];
      o[4 + b] = (int)sw[1];
    }
    const int c = col + j * 16 + g * 8;
    if (live && c < p.outputs) store8<T>(p, row, c, o, sa);
  }
}

__device__ __forceinline__ int16v zero16() {
  int16v z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0;
  return z;
}

// ---- any addresses: 64 x 64 tiles, codes fetched byte by byte where a row's piece of 16 is not whole or the rows not aligned --------------------------------
constexpr int AM = 64, AK = 64, AS = AK + 16;    // rows of a tile, channels of a step, bytes of a row in LDS

template <typename T>
__global__ void __launch_bounds__(256) k_product_any(ProductParams p, int tiles_n) {
  __shared__ __attribute__((aligned(16))) int8_t As[AM * AS], Ws[AM * AS];
  const int lane = threadIdx.x & 63, nn = lane & 31, g = lane >> 5, wave = threadIdx.x >> 6;
  const int64_t m0 = (int64_t)(blockIdx.x / (unsigned)tiles_n) * AM;
  const int n0 = (int)(blockIdx.x % (unsigned)tiles_n) * AM;
  const int r = threadIdx.x >> 2, c0 = (threadIdx.x & 3) * 16;     // the piece of 16 codes that this thread fetches of either tile
  auto fetch = [&](const char* row, bool live, int k) {
    int4v x = {0, 0, 0, 0};
    if (live && k + 16 <= p.channels) x = __builtin_bit_cast(int4v, *(const uint4byte*)(row + k));
    else if (live) {
#pragma unroll
      for (int j = 0; j < 15; ++j)
        if (k + j < p.channels) x[j >> 2] |= (int)((uint32_t)(uint8_t)row[k + j] << (8 * (j & 3)));
    }
    return x;
  };
  const bool a_live = m0 + r < p.rows, w_live = n0 + r < p.outputs;
  const char *a_row = p.a + (a_live ? m0 + r : 0) * p.a_rs, *w_row = p.w + (int64_t)(w_live ? n0 + r : 0) * p.w_rs;
  int16v acc = zero16();
  for (int k0 = 0; k0 < p.channels; k0 += AK) {
    const int4v a = fetch(a_row, a_live, k0 + c0), w = fetch(w_row, w_live, k0 + c0);
    __syncthreads();
    *(int4v*)(As + r * AS + c0) = a;
    *(int4v*)(Ws + r * AS + c0) = w;
    __syncthreads();
#pragma unroll
    for (int s = 0; s < AK / 32; ++s) {
      const int4v rows_ = *(const int4v*)(As + ((wave & 1) * 32 + nn) * AS + s * 32 + g * 16);
      const int4v cols = *(const int4v*)(Ws + ((wave >> 1) * 32 + nn) * AS + s * 32 + g * 16);
      acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(cols, rows_, acc, 0, 0, 0);
    }
  }
  const int64_t row = m0 + (wave & 1) * 32 + nn;
  const bool live = row < p.rows;
  store_tile<T>(p, acc, row, n0 + (wave >> 1) * 32, g, live ? p.a_scales[row] : 0.f, live);
}

// ---- few rows: 16 columns of the output a workgroup, whose waves share the sum -------------------------------------------------------------------------------
// The weights' bytes are all that counts: each is loaded once, straight into the registers that the product takes it from (16 x 16 x 64: lane l holds row l % 16), the rows' codes
// come from the caches.  A step is 128 channels, lane group g taking 32 g .. 32 g + 31, so that a row of a step is a whole line.  The waves' sums meet in LDS.
constexpr int FEW_WAVES = 8;

template <typename T, int MT>
__global__ void __launch_bounds__(64 * FEW_WAVES) k_product_few(ProductParams p) {
  const int lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4, wave = uniform(threadIdx.x >> 6);
  const int n0 = blockIdx.x * 16;
  const char* w_row = p.w + (int64_t)min(n0 + l, p.outputs - 1) * p.w_rs;
  const char* a_row[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) a_row[t] = p.a + (int64_t)min(t * 16 + l, p.rows - 1) * p.a_rs;
  int4v acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t] = int4v{0, 0, 0, 0};
  const int steps = (p.channels + 127) / 128;
  auto piece = [&](const char* row, int k) { return k < p.channels ? *(const int4v*)(row + k) : int4v{0, 0, 0, 0}; };
#pragma unroll 2
  for (int s = wave; s < steps; s += FEW_WAVES) {
    const int k = s * 128 + g * 32;
    int4v w[2], a[MT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      w[h] = piece(w_row, k + 16 * h);
#pragma unroll
      for (int t = 0; t < MT; ++t) a[t][h] = piece(a_row[t], k + 16 * h);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int t = 0; t < MT; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[h], a[t][h], acc[t], 0, 0, 0);
  }
  __shared__ int4v sums[FEW_WAVES][MT][64];
#pragma unroll
  for (int t = 0; t < MT; ++t) sums[wave][t][lane] = acc[t];
  __syncthreads();
  // a thread finishes one row's four columns 4 g .. 4 g + 3
  if (wave >= MT) return;
  int4v s = {0, 0, 0, 0};
#pragma unroll
  for (int w = 0; w < FEW_WAVES; ++w) s += sums[w][wave][lane];
  const int row = wave * 16 + l, c = n0 + 4 * g;
  if (row >= p.rows) return;
  const float sa = p.a_scales[row];
  T* to = (T*)p.out + (int64_t)row * p.out_rs;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (c + j < p.outputs) {
      const float x = (float)s[j] * sa * p.w_scales[c + j];
      to[c + j] = narrow<T>(p.bias ? x + widen(((const T*)p.bias)[c + j]) : x);
    }
}

// ---- tiles: TM x TN results a workgroup of four waves, steps of 128 channels copied straight into LDS, one step ahead -----------------------------------------
// Rows of a step are 128 bytes in LDS; 16-byte chunk c of row r sits at c ^ ((r >> 1) & 7), through the source address, so that the operand reads of 16 rows
// fall on 16 different bank groups.
template <typename T, int TM, int TN>
__global__ void __launch_bounds__(256) k_product_tile(ProductParams p, int tiles_m, int tiles_n) {
  constexpr int MI = TM / 64, NI = TN / 64;     // 32 x 32 products of a wave: its rows TM / 2, its columns TN / 2
  __shared__ __attribute__((aligned(16))) int8_t As[2][TM * 128], Ws[2][TN * 128];
  const int xcd = blockIdx.x & 7, seq = blockIdx.x >> 3;
  const int mt = (seq / tiles_n) * 8 + xcd;
  if (mt >= tiles_m) return;
  const int m0 = mt * TM, n0 = (seq % tiles_n) * TN;
  const int lane = threadIdx.x & 63, nn = lane & 31, g = lane >> 5, wave = uniform(threadIdx.x >> 6);
  const int wm = wave & 1, wn = wave >> 1;
  const int lr = lane >> 3, lc = lane & 7;
  // copy i of a wave: rows (wave * N + i) * 8 .. + 7 of a tile, N = rows / 32
  auto stage = [&](int k0, int buf) {
#pragma unroll
    for (int i = 0; i < TM / 32; ++i) {
      const int r = (wave * (TM / 32) + i) * 8 + lr, k = k0 + ((lc ^ ((r >> 1) & 7)) << 4);
      const char* at = p.a + (int64_t)min(m0 + r, p.rows - 1) * p.a_rs + k;
      copy16(k < p.channels ? (const void*)at : (const void*)&zero_piece, lds_at(As[buf] + (wave * (TM / 32) + i) * 8 * 128));
    }
#pragma unroll
    for (int i = 0; i < TN / 32; ++i) {
      const int r = (wave * (TN / 32) + i) * 8 + lr, k = k0 + ((lc ^ ((r >> 1) & 7)) << 4);
      const char* at = p.w + (int64_t)min(n0 + r, p.outputs - 1) * p.w_rs + k;
      copy16(k < p.channels ? (const void*)at : (const void*)&zero_piece, lds_at(Ws[buf] + (wave * (TN / 32) + i) * 8 * 128));
    }
  };
  int16v acc[NI][MI];
#pragma unroll
  for (int n = 0; n < NI; ++n)
#pragma unroll
    for (int m = 0; m < MI; ++m) acc[n][m] = zero16();
  const int steps = (p.channels + 127) / 128;
  stage(0, 0);
  for (int s = 0; s < steps; ++s) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (s + 1 < steps) stage((s + 1) * 128, (s + 1) & 1);
    const int8_t *Ab = As[s & 1] + (wm * (TM / 2) + nn) * 128, *Wb = Ws[s & 1] + (wn * (TN / 2) + nn) * 128;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      const int pos = ((2 * ks + g) ^ ((nn >> 1) & 7)) << 4;
      int4v a[MI], w[NI];
#pragma unroll
      for (int m = 0; m < MI; ++m) a[m] = *(const int4v*)(Ab + m * 32 * 128 + pos);
#pragma unroll
      for (int n = 0; n < NI; ++n) w[n] = *(const int4v*)(Wb + n * 32 * 128 + pos);
#pragma unroll
      for (int n = 0; n < NI; ++n)
#pragma unroll
        for (int m = 0; m < MI; ++m) acc[n][m] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[n], a[m], acc[n][m], 0, 0, 0);
    }
  }
#pragma unroll
  for (int m = 0; m < MI; ++m) {
    const int row = m0 + wm * (TM / 2) + m * 32 + nn;
    const bool live = row < p.rows;
    const float sa = live ? p.a_scales[row] : 0.f;
#pragma unroll
    for (int n = 0; n < NI; ++n) store_tile<T>(p, acc[n][m], row, n0 + wn * (TN / 2) + n * 32, g, sa, live);
  }
}

enum { ANY, FEW, TILE };

template <typename T, int TM, int TN>
hipError_t tile(const ProductParams& p, hipStream_t st) {
  const int tiles_m = (int)(((int64_t)p.rows + TM - 1) / TM), tiles_n = (int)(((int64_t)p.outputs + TN - 1) / TN);
  const int64_t blocks = ((int64_t)tiles_m + 7) / 8 * 8 * tiles_n;
  if (blocks >= ((int64_t)1 << 23)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((k_product_tile<T, TM, TN>), dim3((unsigned)blocks), dim3(256), 0, st, p, tiles_m, tiles_n);
  return hipGetLastError();
}

template <typename T>
hipError_t go(const ProductParams& p, const ProductPlan& s, hipStream_t st) {
  if (s.kind == ANY) {
    const int64_t tiles_n = ((int64_t)p.outputs + AM - 1) / AM, blocks = ((int64_t)p.rows + AM - 1) / AM * tiles_n;
    if (blocks >= ((int64_t)1 << 23)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(k_product_any<T>, dim3((unsigned)blocks), dim3(256), 0, st, p, (int)tiles_n);
    return hipGetLastError();
  }
  if (s.kind == FEW) {
    const dim3 grid((unsigned)(((int64_t)p.outputs + 15) / 16)), block(64 * FEW_WAVES);
    if (((int64_t)p.outputs + 15) / 16 >= ((int64_t)1 << 23)) return hipErrorInvalidConfiguration;
    if (p.rows <= 16) hipLaunchKernelGGL((k_product_few<T, 1>), grid, block, 0, st, p);
    else if (p.rows <= 32) hipLaunchKernelGGL((k_product_few<T, 2>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((k_product_few<T, 4>), grid, block, 0, st, p);
    return hipGetLastError();
  }
  return s.tile_m == 64 ? tile<T, 64, 64>(p, st) : tile<T, 128, 128>(p, st);
}

}  // namespace

ProductPlan product_plan(const ProductParams& p, int num_cu) {
  ProductPlan s = {};
  s.pieces = 1;
  if (!p.vec) { s.kind = ANY; return s; }
  if (p.rows <= 64) { s.kind = FEW; return s; }
  s.kind = TILE;
  s.tile_m = s.tile_n = ((int64_t)p.rows + 127) / 128 * (((int64_t)p.outputs + 127) / 128) >= 2 * (int64_t)num_cu ? 128 : 64;
  return s;
}

hipError_t launch_product_i8(ProductParams p, const ProductPlan& s, int dtype, hipStream_t st) {
  return dtype == FREQATTN_BF16 ? go<Bf16>(p, s, st) : go<float>(p, s, st);
}

}  // namespace fa
