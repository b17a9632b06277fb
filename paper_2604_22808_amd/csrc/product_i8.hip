// Products of rows of 8-bit codes: out[m][n] = s_a[m] s_w[n] sum_k a[m][k] w[n][k] + bias[n], k adjacent in both.  Sums are whole numbers of 32 bits, exact up to 131,071
// channels, so neither their order nor their cut shows in the result; scaling and bias are fp32, rounded once to the output's type.
//
// Long products run on 256 x 256 tiles, whose round of the chip takes about 11 us whatever the channels and 13 ns more for each of them (65,536 rows, 4096 outputs: 128 channels 12.2 us a
// round, 1024 24.6, 2048 37.8, 8192 117, which is 2.3 POPS): during the first copies of a tile, and while its results go out, the compute unit's only workgroup multiplies nothing.
// 65,536 x 1536 -> 4608 533 us (1.74 POPS; a library's product without scales 557; fp32 results 585), 131,072 x 2048 -> 2048 605-619 (1.8; 589; 675), 16,384 x 4096 -> 4096 252 (2.18; fp32
// results 270), 8192 x 4096 -> 4096 130; in a run with counters the second took 660 us, matrix cores busy 45 % of the cycles.  A few rows are bound by the weights' bytes and latency.
//
// Operands are fed to the matrix cores as 16 bytes a lane, k = 16 g .. 16 g + 15 of a product's channels on lane group g; both sides use the same order, so any
// order of the channels will do.
#include <algorithm>

#include "rows.h"
#include "tokens.h"

namespace fa {

using namespace rows;

namespace {

typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int16v __attribute__((ext_vector_type(16)));

static __device__ const int4v zero_piece = {0, 0, 0, 0};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ unsigned lds_at(const void* p) { return (unsigned)uniform((int)(unsigned)(uintptr_t)(const __attribute__((address_space(3))) void*)p); }
// One wave-wide copy into LDS, 16 bytes a lane, to bytes dst + 16 lane.  Written as assembly because the compiler orders every LDS read behind a copy of this
// kind that it knows of; the kernels wait for their copies themselves.
__device__ __forceinline__ void copy16(const void* src, unsigned dst) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "s"(dst) : "memory", "m0");
}

// A sum in the value's units.  Beyond 2^96 a row's scale times the sum may leave fp32 where the other scale would have brought it back: that one comes first then.  (If
// both are so large, what is not zero has no value in fp32 either way.)
__device__ __forceinline__ bool far_scale(float sa) { return sa > 0x1p96f; }
__device__ __forceinline__ float scaled(int sum, float sa, float sw) { return far_scale(sa) ? (float)sum * sw * sa : (float)sum * sa * sw; }

// Eight results of a row, columns c .. c + 7 (zeros where there is no column), as pieces of the output.
template <typename T>
__device__ __forceinline__ void finish8(const ProductParams& p, int c, const int (&acc)[8], float sa, Piece<T> (&x)[8 / PW<T>]) {
  float o[8];
  if (c + 8 <= p.outputs) {
    const float4v s0 = *(const float4any*)(p.w_scales + c), s1 = *(const float4any*)(p.w_scales + c + 4);
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = (float)acc[j] * sa * (j < 4 ? s0[j & 3] : s1[j & 3]);
    if (far_scale(sa)) {
      asm volatile("");      // (a branch, not selects for everyone)
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = scaled(acc[j], sa, j < 4 ? s0[j & 3] : s1[j & 3]);
    }
    if (p.bias) {
#pragma unroll
      for (int i = 0; i < 8 / PW<T>; ++i) {
        Piece<T> b;
        b.raw = *(const uint4any*)((const T*)p.bias + c + i * PW<T>);
#pragma unroll
        for (int j = 0; j < PW<T>; ++j) o[i * PW<T> + j] += b.get(j);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      o[j] = 0.f;
      if (c + j < p.outputs) {
        o[j] = scaled(acc[j], sa, p.w_scales[c + j]);
        if (p.bias) o[j] += widen(((const T*)p.bias)[c + j]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 8 / PW<T>; ++i)
#pragma unroll
    for (int j = 0; j < PW<T>; j += 2) x[i].set(j, o[i * PW<T> + j], o[i * PW<T> + j + 1]);
}

// The accumulators of a 32 x 32 product hold one row a lane and the columns 8 (r / 4) + 4 g + r % 4: after a swap of registers with lane ^ 32 (the same row) a lane has
// 8 neighbouring columns.
__device__ __forceinline__ void neighbours(const int16v& acc, int j, int (&o)[8]) {
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const auto sw = __builtin_amdgcn_permlane32_swap((unsigned)acc[8 * j + b], (unsigned)acc[8 * j + 4 + b], false, false);
    o[b] = (int)sw[0];
    o[4 + b] = (int)sw[1];
  }
}
template <typename T>
__device__ __forceinline__ void store_tile(const ProductParams& p, const int16v& acc, int64_t row, int col, int g, float sa, bool live) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    int o[8];
    neighbours(acc, j, o);
    const int c = col + j * 16 + g * 8;
    if (live && c < p.outputs) {
      Piece<T> x[8 / PW<T>];
      finish8<T>(p, c, o, sa, x);
#pragma unroll
      for (int i = 0; i < 8 / PW<T>; ++i) x[i].store((T*)p.out + row * p.out_rs, c + i * PW<T>, p.outputs);
    }
  }
}

// 32 rows x 64 columns, two products side by side, through a wave's 8 KB (fp32; bf16: 4) of LDS, so that a store covers whole lines of a few rows instead of 32 bytes of each
// (100,000 x 96 -> 4096 338 / 282 us, 65,536 x 256 -> 4096 270 / 235, 65,536 x 1536 -> 4608 543 / 536).
template <typename T>
__device__ __forceinline__ void store_wide(const ProductParams& p, const int16v& left, const int16v& right, int first, int col, int lane, uint4v* mine) {
  constexpr int CH = 64 / PW<T>, STORES = 32 * CH / 64;      // pieces of such a row; stores of a lane
  const int nn = lane & 31, g = lane >> 5;
  const float sa = p.a_scales[min(first + nn, p.rows - 1)];
  // (lanes read what others wrote: a wave's accesses to LDS stay in order, and the waits keep the compiler from moving one past another whose address it can tell apart within a lane)
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
  for (int c2 = 0; c2 < 2; ++c2)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      int o[8];
      neighbours(c2 ? right : left, j, o);
      Piece<T> x[8 / PW<T>];
      finish8<T>(p, col + 32 * c2 + 16 * j + 8 * g, o, sa, x);
#pragma unroll
      for (int i = 0; i < 8 / PW<T>; ++i) mine[nn * CH + (((4 * c2 + 2 * j + g) * (8 / PW<T>) + i) ^ (nn & 7))] = x[i].raw;
    }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
  for (int i = 0; i < STORES; ++i) {
    const int r = i * (64 / CH) + lane / CH, ch = lane % CH;
    Piece<T> x;
    x.raw = mine[r * CH + (ch ^ (r & 7))];
    if (first + r < p.rows) x.store((T*)p.out + (int64_t)(first + r) * p.out_rs, col + ch * PW<T>, p.outputs);
  }
}

__device__ __forceinline__ int16v zero16() {
  int16v z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0;
  return z;
}

// The tile of a workgroup.  Workgroups are dealt to the 8 XCDs in turn and each XCD has an L2 of its own: XCD x takes the x-th eighth of the tiles, in an order that goes through
// GROUP rows of tiles column by column, so that the tiles that run at the same time share few rows and columns.
constexpr int GROUP = 4;
__device__ __forceinline__ bool tile_of(int tiles_m, int tiles_n, int& mt, int& nt) {
  const unsigned all = (unsigned)tiles_m * (unsigned)tiles_n, each = (all + 7) / 8;
  const unsigned id = (blockIdx.x & 7) * each + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= each || id >= all) return false;
  const unsigned group = id / (GROUP * (unsigned)tiles_n), in = id - group * GROUP * (unsigned)tiles_n;
  const unsigned rows_ = min((unsigned)GROUP, (unsigned)tiles_m - group * GROUP);
  nt = (int)(in / rows_);
  mt = (int)(group * GROUP + in - (unsigned)nt * rows_);
  return true;
}

// ---- any addresses: TM x TM tiles, codes through registers into LDS, two steps ahead of the products ---------------------------------------------------------
// (333 x 1000 -> 1100 7.1 us; 64 x 2049 -> 6144 12.5, with nothing requested ahead 17.7; 14,599 x 1999 -> 2000 137, 0.85 POPS)
constexpr int AK = 64, AS = AK + 16;    // channels of a step, bytes of a row in LDS

// Codes k .. k + 15 of a row of n, zeros from n on.
__device__ __forceinline__ int4v row_piece(const char* row, int k, int n) {
  if (k >= n) return int4v{0, 0, 0, 0};
  if (k + 16 <= n) return __builtin_bit_cast(int4v, *(const uint4byte*)(row + k));
  if (n >= 16) {      // the row's last 16, shifted down
    typedef uint64_t long2 __attribute__((ext_vector_type(2)));
    const long2 x = __builtin_bit_cast(long2, *(const uint4byte*)(row + n - 16));
    const int down = 8 * (k + 16 - n);      // 8 .. 120
    const long2 y = down >= 64 ? long2{x[1] >> (down - 64), 0} : long2{x[0] >> down | x[1] << (64 - down), x[1] >> down};
    return __builtin_bit_cast(int4v, y);
  }
  int4v x = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < 15; ++j)
    if (k + j < n) x[j >> 2] |= (int)((uint32_t)(uint8_t)row[k + j] << (8 * (j & 3)));
  return x;
}

template <typename T, int TM>
__global__ void __launch_bounds__(256) k_product_any(ProductParams p, int tiles_m, int tiles_n) {
  constexpr int MI = TM / 64;      // 32 x 32 products of a wave each way; pieces of 16 codes of a thread and operand
  __shared__ __attribute__((aligned(16))) int8_t both[4][TM * AS];
  int8_t(*const As)[TM * AS] = both, (*const Ws)[TM * AS] = both + 2;
  int mt, nt;
  if (!tile_of(tiles_m, tiles_n, mt, nt)) return;
  const int64_t m0 = (int64_t)mt * TM;
  const int n0 = nt * TM;
  const int lane = threadIdx.x & 63, nn = lane & 31, g = lane >> 5, wave = threadIdx.x >> 6, wm = wave & 1, wn = wave >> 1;
  const int r = threadIdx.x >> 2, c0 = (threadIdx.x & 3) * 16;
  const char *a_row[MI], *w_row[MI];      // (rows that do not exist: the last one, and nobody stores what comes of it)
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    a_row[i] = p.a + min(m0 + r + 64 * i, (int64_t)p.rows - 1) * p.a_rs + c0;
    w_row[i] = p.w + (int64_t)min(n0 + r + 64 * i, p.outputs - 1) * p.w_rs + c0;
  }
  int16v acc[MI][MI];
#pragma unroll
  for (int n = 0; n < MI; ++n)
#pragma unroll
    for (int m = 0; m < MI; ++m) acc[n][m] = zero16();
  struct Step { int4v a[MI], w[MI]; };
  auto fetch = [&](Step& x, int k0) {
    if (k0 + AK <= p.channels) {
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        x.a[i] = __builtin_bit_cast(int4v, *(const uint4byte*)(a_row[i] + k0));
        x.w[i] = __builtin_bit_cast(int4v, *(const uint4byte*)(w_row[i] + k0));
      }
    } else if (k0 < p.channels) {
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        x.a[i] = row_piece(a_row[i] - c0, k0 + c0, p.channels);
        x.w[i] = row_piece(w_row[i] - c0, k0 + c0, p.channels);
      }
    }
  };
  auto store = [&](const Step& x, int buf) {
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      *(int4v*)(As[buf] + (r + 64 * i) * AS + c0) = x.a[i];
      *(int4v*)(Ws[buf] + (r + 64 * i) * AS + c0) = x.w[i];
    }
  };
  auto multiply = [&](int buf) {
#pragma unroll
    for (int s = 0; s < AK / 32; ++s) {
      int4v rows_[MI], cols[MI];
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        rows_[i] = *(const int4v*)(As[buf] + (wm * (TM / 2) + i * 32 + nn) * AS + s * 32 + g * 16);
        cols[i] = *(const int4v*)(Ws[buf] + (wn * (TM / 2) + i * 32 + nn) * AS + s * 32 + g * 16);
      }
#pragma unroll
      for (int n = 0; n < MI; ++n)
#pragma unroll
        for (int m = 0; m < MI; ++m) acc[n][m] = __builtin_amdgcn_mfma_i32_32x32x32_i8(cols[n], rows_[m], acc[n][m], 0, 0, 0);
    }
  };
  // two steps under way in registers, one in LDS
  Step even, odd;
  fetch(even, 0);
  fetch(odd, AK);
  for (int k0 = 0; k0 < p.channels; k0 += 2 * AK) {
    store(even, 0);
    fetch(even, k0 + 2 * AK);
    __syncthreads();
    multiply(0);
    if (k0 + AK < p.channels) {
      store(odd, 1);
      fetch(odd, k0 + 3 * AK);
      __syncthreads();
      multiply(1);
    }
  }
  if constexpr (MI == 2) {
    static_assert(MI == 1 || 4 * TM * AS >= 4 * 8192, "");
    __syncthreads();
#pragma unroll
    for (int m = 0; m < MI; ++m) store_wide<T>(p, acc[0][m], acc[1][m], (int)m0 + wm * (TM / 2) + m * 32, n0 + wn * (TM / 2), lane, (uint4v*)(both[0] + wave * 8192));
  } else {
    const int64_t row = m0 + wm * (TM / 2) + nn;
    const bool live = row < p.rows;
    store_tile<T>(p, acc[0][0], row, n0 + wn * (TM / 2), g, live ? p.a_scales[row] : 0.f, live);
  }
}

// ---- few rows: 16 columns of the output a workgroup, whose waves share the sum -------------------------------------------------------------------------------
// The weights' bytes are all that counts: each is loaded once, straight into the registers that the product takes it from (16 x 16 x 64: lane l holds row l % 16), the rows' codes
// come from the caches.  A step is 128 channels, lane group g taking 32 g .. 32 g + 31, so that a row of a step is a whole line.  The waves' sums meet in LDS.
// 2048 -> 6144: one row 4.6 us (2.7 TB/s), 16 rows 6.1.
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
      const float x = scaled(s[j], sa, p.w_scales[c + j]);
      to[c + j] = narrow<T>(p.bias ? x + widen(((const T*)p.bias)[c + j]) : x);
    }
}

// ---- tiles: TM x TN results a workgroup of four waves, steps of 128 channels copied straight into LDS, S - 1 steps ahead -------------------------------------
// Rows of a step are 128 bytes in LDS; 16-byte chunk c of row r sits at c ^ ((r >> 1) & 7), through the source address, so that the operand reads of 16 rows
// fall on 16 different bank groups.
// G groups of four waves take every G-th step, with tiles of their own in LDS, and add their sums up there.
template <typename T, int TM, int TN, int S, int G>
__global__ void __launch_bounds__(256 * G) k_product_tile(ProductParams p, int tiles_m, int tiles_n) {
  constexpr int MI = TM / 64, NI = TN / 64;     // 32 x 32 products of a wave: its rows TM / 2, its columns TN / 2
  constexpr int COPIES = TM / 32 + TN / 32;     // of a wave and step
  static_assert(G * S * (TM + TN) * 128 <= 160 * 1024 && (S - 2) * COPIES < 64, "");
  static_assert(NI == 1 ? MI == 1 : NI == 2 && G * S * TM * 128 >= 4 * 8192, "");
  static_assert(G == 1 || (MI * NI == 1 && (G - 1) * 4 * 64 * 64 <= G * S * TM * 128), "");
  __shared__ __attribute__((aligned(16))) int8_t all_a[G][S][TM * 128], all_w[G][S][TN * 128];
  int mt, nt;
  if (!tile_of(tiles_m, tiles_n, mt, nt)) return;      // (uniform over the workgroup)
  const int m0 = mt * TM, n0 = nt * TN;
  const int lane = threadIdx.x & 63, nn = lane & 31, g = lane >> 5, group = G == 1 ? 0 : uniform(threadIdx.x >> 8), wave = uniform(threadIdx.x >> 6) & 3;
  const int wm = wave & 1, wn = wave >> 1;
  const int lr = lane >> 3, lc = lane & 7;
  int8_t(*const As)[TM * 128] = all_a[group];
  int8_t(*const Ws)[TN * 128] = all_w[group];
  // copy i of a wave: rows (wave * N + i) * 8 .. + 7 of a tile, N = rows / 32; channels behind the last one are zeros
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
  const int steps = (p.channels + 128 * G - 1) / (128 * G);      // of a group
#pragma unroll
  for (int s = 0; s < S - 1; ++s) stage((s * G + group) * 128, s);       // (steps behind the last one are zeros too: the count of copies under way stays the same)
  int buf = 0;
  for (int s = 0; s < steps; ++s) {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((S - 2) * COPIES) : "memory");    // step s is there for everybody, and step s - 1 has been read
    stage(((s + S - 1) * G + group) * 128, buf == 0 ? S - 1 : buf - 1);
    const int8_t *Ab = As[buf] + (wm * (TM / 2) + nn) * 128, *Wb = Ws[buf] + (wn * (TN / 2) + nn) * 128;
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
    buf = buf == S - 1 ? 0 : buf + 1;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // (copies into this workgroup's LDS)
  if constexpr (G > 1) {
    __syncthreads();
    int4v* const sums = (int4v*)all_a;
    if (group > 0) {
#pragma unroll
      for (int j = 0; j < 4; ++j) sums[(((group - 1) * 4 + j) * 4 + wave) * 64 + lane] = int4v{acc[0][0][4 * j], acc[0][0][4 * j + 1], acc[0][0][4 * j + 2], acc[0][0][4 * j + 3]};
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int o = 0; o < G - 1; ++o)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int4v x = sums[((o * 4 + j) * 4 + wave) * 64 + lane];
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[0][0][4 * j + k] += x[k];
      }
  }
  if constexpr (NI == 2) {
    __syncthreads();
#pragma unroll
    for (int m = 0; m < MI; ++m) store_wide<T>(p, acc[0][m], acc[1][m], m0 + wm * (TM / 2) + m * 32, n0 + wn * (TN / 2), lane, (uint4v*)(all_a[0][0] + wave * 8192));
  } else {
    const int row = m0 + wm * (TM / 2) + nn;
    const bool live = row < p.rows;
    store_tile<T>(p, acc[0][0], row, n0 + wn * (TN / 2), g, live ? p.a_scales[row] : 0.f, live);
  }
}

// ---- wide tiles: 256 x 256 results a workgroup of eight waves, one workgroup a compute unit ---------------------------------------------------------------
// The tiles of a step of 128 channels are halves of 128 rows, 16 KB each in LDS, two copies of everything (128 KB).  A wave owns 32 rows of either half of A and 64
// columns of either half of W, and a step is four phases of 8 products, one per pair of halves, in an order in which every phase changes one half only: A0 W0, A0 W1, A1 W1,
// A1 W0, then (next step) A0 W1, A0 W0, A1 W0, A1 W1.  So half number j of the sequence A0 W0 W1 A1 | A0 W1 W0 A1 | A0 W0 .. is, in phase
//   j - 9   copied from memory into the place of half j - 8, which every wave has read in phase j - 10,
//   j - 2   read into registers by every wave, beside the products of that phase,
//   j - 1 .. j + 2   multiplied.
// A copy has seven phases to arrive, six of them are always in flight, and no wait in the loop is for the latest ones.
constexpr int WM = 256, HALF = 128 * 128;

// TAIL: the channels end inside a step.
template <typename T, bool TAIL>
__global__ void __launch_bounds__(512, 2) k_product_wide(ProductParams p, int tiles_m, int tiles_n) {
  __shared__ __attribute__((aligned(16))) int8_t lds[4][2][HALF];   // [A0, A1, W0, W1][step & 1]
  int mt, nt;
  if (!tile_of(tiles_m, tiles_n, mt, nt)) return;
  const int m0 = mt * WM, n0 = nt * WM;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), nn = lane & 31, g = lane >> 5;
  const int wm = wave & 3, wn = wave >> 2;              // this wave's 32 rows and 64 columns of every half
  // 16-byte chunk c of row r sits at c ^ ((r >> 1) & 7); the copies: wave w moves rows 16 w .. 16 w + 15 of a half, 8 per instruction
  int lr = lane >> 3, chunk = ((lane & 7) ^ ((lane >> 4) & 3)) << 4;   // this lane's row and (even instructions) its chunk
  const int steps = (p.channels + 127) / 128;
  int k_i = 0;                                          // the step that is copied next
  const unsigned copy_at = lds_at(lds[0][0] + 16 * wave * 128);
  auto copy = [&](int buf, int which) {   // 0, 1: A0, A1; 2, 3: W0, W1
    const int h = which & 1;
    const bool w = which >= 2;
    const char* base = (w ? p.w + (int64_t)n0 * p.w_rs : p.a + (int64_t)m0 * p.a_rs) + k_i;   // wave-uniform
    const int last = (w ? p.outputs - n0 : p.rows - m0) - 1, first = 128 * h + 16 * wave;     // (rows clamped to what exists)
    const uint32_t rs = (uint32_t)(w ? p.w_rs : p.a_rs);
    asm volatile("" : "+v"(lr), "+v"(chunk));   // (addresses formed here: kept for the whole loop they would take the operands' registers)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int c = chunk ^ (i * 64);
      const char* at = base + (uint32_t)((uint32_t)min(first + 8 * i + lr, last) * rs + (uint32_t)c);
      if (TAIL) at = k_i + c < p.channels ? at : (const char*)&zero_piece;
      copy16(at, copy_at + (which * 2 + buf) * HALF + 8 * i * 128);
    }
  };
  auto advance = [&]() {   // (behind the last step: that step again, into places that nobody reads)
    if (k_i + 128 < p.channels) k_i += 128;
  };

  int16v acc[4][2];   // [column tile: half of W, 32 columns][row tile: half of A]
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) acc[ct][rt] = zero16();
  int4v ra[2][4], rw[2][4][2];   // operands: halves of A and of W
  const int8_t* const a_at = lds[0][0] + (32 * wm + nn) * 128;
  const int8_t* const w_at = lds[2][0] + (64 * wn + nn) * 128;
  auto read = [&](int buf, int which) {
    const int h = which & 1;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      const int pos = ((2 * ks + g) ^ ((nn >> 1) & 7)) << 4;
      if (which < 2) {
        ra[h][ks] = *(const int4v*)(a_at + (2 * h + buf) * HALF + pos);
      } else {
#pragma unroll
        for (int c = 0; c < 2; ++c) rw[h][ks][c] = *(const int4v*)(w_at + (2 * h + buf) * HALF + c * 32 * 128 + pos);
      }
    }
  };
  // One phase: half `a` of A and half `w` of W multiplied; the half `rd` read; the half `cp` copied.
  auto phase = [&](int a, int w, int rd_buf, int rd, int cp_buf, int cp) {
    // The half to be read has landed (this wave's part; with the barrier, everybody's), and everybody has the half that was read last.
    asm volatile("s_waitcnt vmcnt(12) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    copy(cp_buf, cp);
    read(rd_buf, rd);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int c = 0; c < 2; ++c) acc[2 * w + c][a] = __builtin_amdgcn_mfma_i32_32x32x32_i8(rw[w][ks][c], ra[a][ks], acc[2 * w + c][a], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  };

  copy(0, 0); copy(0, 2); copy(0, 3); copy(0, 1); advance();   // halves 0 .. 3
  copy(1, 0); copy(1, 3); copy(1, 2); copy(1, 1); advance();   // 4 .. 7
  asm volatile("s_waitcnt vmcnt(12)\n\ts_barrier" ::: "memory");
  read(0, 0); read(0, 2);
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  copy(0, 0);                                                   // 8
  for (int step = 1; step < steps; step += 2) {
    phase(0, 0, 0, 3, 0, 2);
    phase(0, 1, 0, 1, 0, 3);
    phase(1, 1, 1, 0, 0, 1); advance();
    phase(1, 0, 1, 3, 1, 0);
    phase(0, 1, 1, 2, 1, 3);
    phase(0, 0, 1, 1, 1, 2);
    phase(1, 0, 0, 0, 1, 1); advance();
    phase(1, 1, 0, 2, 0, 0);
  }
  if (steps & 1) {
    phase(0, 0, 0, 3, 0, 2);
    phase(0, 1, 0, 1, 0, 3);
    phase(1, 1, 1, 0, 0, 1);
    phase(1, 0, 1, 3, 1, 0);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (copies into this workgroup's LDS)
  __syncthreads();
#pragma unroll
  for (int rt = 0; rt < 2; ++rt)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      store_wide<T>(p, acc[2 * h][rt], acc[2 * h + 1][rt], m0 + 128 * rt + 32 * wm, n0 + 64 * wn + 128 * h, lane, (uint4v*)(lds[0][0] + wave * HALF));
      __builtin_amdgcn_sched_barrier(0);
    }
}

template <typename T, int TM, int TN, int S, int G>
hipError_t tile(const ProductParams& p, hipStream_t st) {
  const int tiles_m = (int)(((int64_t)p.rows + TM - 1) / TM), tiles_n = (int)(((int64_t)p.outputs + TN - 1) / TN);
  const int64_t blocks = ((int64_t)tiles_m * tiles_n + 7) / 8 * 8;
  if (blocks >= ((int64_t)1 << 23)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((k_product_tile<T, TM, TN, S, G>), dim3((unsigned)blocks), dim3(256 * G), 0, st, p, tiles_m, tiles_n);
  return hipGetLastError();
}

template <typename T>
hipError_t wide(const ProductParams& p, hipStream_t st) {
  const int tiles_m = (int)(((int64_t)p.rows + WM - 1) / WM), tiles_n = (int)(((int64_t)p.outputs + WM - 1) / WM);
  const int64_t blocks = ((int64_t)tiles_m * tiles_n + 7) / 8 * 8;
  if (blocks >= ((int64_t)1 << 23)) return hipErrorInvalidConfiguration;
  if (p.channels % 128) hipLaunchKernelGGL((k_product_wide<T, true>), dim3((unsigned)blocks), dim3(512), 0, st, p, tiles_m, tiles_n);
  else hipLaunchKernelGGL((k_product_wide<T, false>), dim3((unsigned)blocks), dim3(512), 0, st, p, tiles_m, tiles_n);
  return hipGetLastError();
}

template <typename T, int TM>
hipError_t any(const ProductParams& p, hipStream_t st) {
  const int tiles_m = (int)(((int64_t)p.rows + TM - 1) / TM), tiles_n = (int)(((int64_t)p.outputs + TM - 1) / TM);
  const int64_t blocks = ((int64_t)tiles_m * tiles_n + 7) / 8 * 8;
  if (blocks >= ((int64_t)1 << 23)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((k_product_any<T, TM>), dim3((unsigned)blocks), dim3(256), 0, st, p, tiles_m, tiles_n);
  return hipGetLastError();
}

template <typename T>
hipError_t few(const ProductParams& p, hipStream_t st) {
  const int64_t blocks = ((int64_t)p.outputs + 15) / 16;
  if (blocks >= ((int64_t)1 << 23)) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)blocks), block(64 * FEW_WAVES);
  if (p.rows <= 16) hipLaunchKernelGGL((k_product_few<T, 1>), grid, block, 0, st, p);
  else hipLaunchKernelGGL((k_product_few<T, 2>), grid, block, 0, st, p);
  return hipGetLastError();
}

// Stages of the copies by tile.
//
// The kernel of few rows takes up to 32 of them where its workgroups run side by side, one a compute unit for 17 to 32 rows and two for up to 16 (or few channels): each reads all rows' codes,
// which more workgroups wait for one after the other, while 64 x 64 tiles read them once for 64 outputs.  Here / on tiles, 32 rows: 2048 -> 4096 5.5 / 6.2 us, 4112 7.9 / 6.2, 6144 8.2 / 6.2,
// 4096 -> 4096 8.5 / 9.1, 6144 13.7 / 9.2, 8192 -> 1024 13.1 / 15.3, 8192 24.6 / 15.8, 1024 -> 1024 4.1 / 4.6; 17 rows: 2048 -> 4096 4.8 / 6.1, 6144 6.8 / 6.1, 8192 -> 8192 19.6 / 15.7.  16
// rows: 2048 -> 8192 6.2 / 6.2, 16,384 10.4 / 6.9, 4096 -> 6144 10.0 / 9.1, 12,288 13.9 / 10.7, 8192 -> 1024 9.4 / 15.2; one row: 2048 -> 8192 4.7 / 6.2, 16,384 7.5 / 7.0, 4096 -> 12,288 10.3 /
// 10.4, 512 -> 12,288 3.4 / 3.9 (16 rows 4.2 / 4.0).  64 rows: 2048 -> 6144 12.1 / 6.4, 8192 -> 1024 20.5 / 15.2.
// On 64 x 64 tiles of a single round two groups share the steps: one / two / four of them, 64 rows 2048 -> 6144 7.7 / 6.4 / 6.5 us, 8192 -> 1024 21.3 / 15.2 / 13.7, 512 rows 8192 -> 1024
// 22.2 / 16.6 / 16.7, 6250 rows 8000 -> 96 22.5 / 18.8 / 22.6; in more rounds 2048 x 1536 -> 1536 11.6 / 15.3 / 16.1.
constexpr int S64 = 3, S128 = 2, FEW_ROWS = 32, FEW_CHANNELS = 512;
bool few_rows(const ProductParams& p, int num_cu) {
  const int64_t blocks = ((int64_t)p.outputs + 15) / 16;
  return p.rows <= 16 ? blocks <= 2 * (int64_t)num_cu || p.channels <= FEW_CHANNELS : p.rows <= FEW_ROWS && blocks <= num_cu;
}

template <typename T>
hipError_t go(const ProductParams& p, int num_cu, hipStream_t st) {
  if (!p.vec) {
    // by the time of the launch, us at 2048 channels: tiles of 64 take 7.2 on a full compute unit and 13 alone, of 128 19 and 25 (14,599 x 1999 -> 2000 206 / 137, 2000 x 3001 -> 1000
    // 23 / 34, 333 x 1000 -> 1100 7.1 / 13.5)
    auto time = [&](int64_t n, float each, float alone) {
      return std::max(alone, each * (float)(((int64_t)p.rows + n - 1) / n * (((int64_t)p.outputs + n - 1) / n)) / (float)num_cu);
    };
    return time(128, 19.f, 25.f) < time(64, 7.2f, 13.f) ? any<T, 128>(p, st) : any<T, 64>(p, st);
  }
  if (few_rows(p, num_cu)) return few<T>(p, st);
  // The kernel whose rounds of the chip take the shortest, us at 2048 channels (others in proportion): a compute unit holds three workgroups of 64 x 64 tiles (one of them alone 9, or 7 in
  // two groups, two 12, three 13), two of 128 x 128 (16, 28) or one of 256 x 256 (29).  Measured as tiles of 64 / 128 / 256: 1024 x 2048 -> 2048 11.6 / 16.6 / 29.5, 2048 x 2048 -> 2048 21.6 / 18.2 /
  // 30.5, 4096 x 2048 -> 2048 36 / 27.6 / 33, 2048 x 1536 -> 4608 33.6 / 32.2 / 28.5, 3000 x 4096 -> 4096 91 / 70 / 57, 100,000 x 1024 -> 128 35 / 32 / 39.5.
  auto cost = [&](int64_t n, int resident, const int (&us)[4]) {
    const int64_t tiles = ((int64_t)p.rows + n - 1) / n * (((int64_t)p.outputs + n - 1) / n), round = (int64_t)num_cu * resident;
    return tiles / round * us[resident] + us[(tiles % round + num_cu - 1) / num_cu];
  };
  const bool one = ((int64_t)p.rows + 63) / 64 * (((int64_t)p.outputs + 63) / 64) <= num_cu;
  const int64_t c64 = one ? 7 : cost(64, 3, {0, 9, 12, 13}), c128 = cost(128, 2, {0, 16, 28, 0}), c256 = cost(256, 1, {0, 29, 0, 0});
  // (the wide kernel's rows lie within 2^31 bytes of their tile's first)
  const bool near = p.a_rs >= 0 && p.a_rs < (1 << 22) && p.w_rs >= 0 && p.w_rs < (1 << 22);
  if (near && c256 <= c128 && c256 <= c64) return wide<T>(p, st);
  if (c128 <= c64) return tile<T, 128, 128, S128, 1>(p, st);
  return one ? tile<T, 64, 64, S64, 2>(p, st) : tile<T, 64, 64, S64, 1>(p, st);
}

}  // namespace

hipError_t launch_product_i8(const ProductParams& p, int dtype, int num_cu, hipStream_t st) {
  return dtype == FREQATTN_BF16 ? go<Bf16>(p, num_cu, st) : go<float>(p, num_cu, st);
}

}  // namespace fa
