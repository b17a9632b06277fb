// What the bf16 kernels of attention over sequences share: operand types, tiles in LDS and the copies that fill them.
//
// A tile is KT rows of D channels, row-major without padding.  Rows are copied straight from global memory into LDS, 16 bytes a lane; lane
// l of a copy fills bytes 16 l of 1 KB, so that the order inside LDS is fixed and bank conflicts are avoided through the global address: 16-byte
// chunk c of row r sits at position c ^ f(r).  Two kinds of operands are read from a tile:
//   rows     lane = row (32 of them), 8 consecutive channels           (one 16-byte read)
//   columns  lane = channel (32), 8 rows in the order of a product's accumulator registers   (two transposing reads, ds_read_b64_tr_b16)
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "seq_common.h"

namespace fa {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef unsigned int uint4v __attribute__((ext_vector_type(4)));
typedef unsigned int uint2v __attribute__((ext_vector_type(2)));
typedef short short4v __attribute__((ext_vector_type(4)));

namespace seq {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// 16 bytes of zeros that copies of rows and channels that do not exist read.
static __device__ const uint4v zero_piece = {0u, 0u, 0u, 0u};

// (values that every lane holds alike, said to the compiler)
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ const void* uniform(const void* x) {
  const uint64_t v = (uint64_t)x;
  return (const void*)(((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32) | (uint32_t)uniform((int)(uint32_t)v));
}
__device__ __forceinline__ SeqRange uniform(SeqRange r) { return SeqRange{uniform(r.seq), uniform(r.base), uniform(r.n)}; }

// One wave-wide copy, 16 bytes a lane, to LDS bytes dst + 16 lane (dst wave-uniform).  Written as assembly because the compiler orders every LDS
// read behind a copy of this kind that it knows of; the kernels wait for their copies themselves (vmcnt) in front of the barrier that publishes a tile.
__device__ __forceinline__ void copy16(const void* base, unsigned off, unsigned dst) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(uniform(base)), "s"(uniform((int)dst))
               : "memory", "m0");
}
__device__ __forceinline__ void copy16_any(const void* addr, unsigned dst) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(addr), "s"(uniform((int)dst)) : "memory", "m0");
}
__device__ __forceinline__ unsigned lds_address(const uint16_t* p) {
  return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) uint16_t*)p;
}

// Stands at the start of a branch that is rarely taken: without it the compiler turns a branch of selects into selects for everyone.
__device__ __forceinline__ void really_branch() { asm volatile(""); }

__device__ __forceinline__ float16v zero16() {
  float16v z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(float2v{a, b}, bf16x2));   // v_cvt_pk_bf16_f32: to nearest, ties to even
}
__device__ __forceinline__ float16v mfma(const bf16x8& a, const bf16x8& b, const float16v& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float other_half(float x) {   // the value of lane ^ 32
  const uint32_t b = __float_as_uint(x);
  const auto sw = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return __uint_as_float((threadIdx.x & 32) ? sw[0] : sw[1]);
}
__device__ __forceinline__ float max_halves(float x) {
  const uint32_t b = __float_as_uint(x);
  const auto sw = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}

// Where 16-byte chunk c of row r sits.  ROWS tiles are read as row operands, by 16 consecutive rows at a time.  COLS tiles are read through transposing
// reads, which hand lane i of a 16-lane group, for k = 0..3, element i % 4 of the 8-byte piece named by lane 4 k + i / 4: four rows of 32 bytes.
// BOTH serves both without conflicts: 16 rows in 16 places, four neighbouring ones 64 bytes apart.
enum { ROWS = 0, COLS = 1, BOTH = 2 };
template <int D, int USE>
__device__ __forceinline__ int swizzle(int r) {
  if (USE == ROWS) return D == 128 ? (r & 15) : ((r >> 1) & 7);
  const int apart = D == 128 ? ((r & 3) << 2) : (((r >> 1) & 1) << 2);
  return USE == COLS ? apart : apart | ((r >> 2) & 3);
}

// Copies of KT rows into a tile by NW waves.
template <int D, int NW, int KT, int USE>
struct TileCopy {
  static constexpr int CPR = D / 8, RPI = 64 / CPR, NI = KT / (RPI * NW);   // chunks a row, rows a copy, copies a wave
  static_assert(NI >= 1, "");
  // (the swizzle of a row repeats after 16 rows at most, so copies whose first rows agree modulo 16 use the same lane offsets)
  static constexpr int NOFF = USE == COLS ? 1 : (16 / RPI < NI ? 16 / RPI : NI);
  unsigned off[NOFF];
  __device__ __forceinline__ void set(int64_t row_bytes, int wave, int lane) {
    const int lr = lane / CPR, c = lane % CPR;
#pragma unroll
    for (int i = 0; i < NOFF; ++i) off[i] = (unsigned)(lr * row_bytes) + ((c ^ swizzle<D, USE>((wave * NI + i) * RPI + lr)) << 4);
  }
  // The copies of one tile, in order: a cursor steps through the tensor with the scalar unit.  (The empty assembly keeps the compiler from holding one
  // address per copy in registers over the whole loop.)
  struct Cursor {
    const char* at;
    __device__ __forceinline__ void step(int64_t bytes) {
      at = (const char*)uniform(at + bytes);
      asm("" : "+s"(at));
    }
  };
  __device__ __forceinline__ Cursor begin(const char* tile, int64_t row_bytes, int wave) const {
    return Cursor{(const char*)uniform(tile + (int64_t)(wave * NI * RPI) * row_bytes)};
  }
  // copy i of this wave, all rows and channels exist
  __device__ __forceinline__ void whole(Cursor& cur, int64_t row_bytes, unsigned dst, int wave, int i) const {
    copy16(cur.at, off[i % NOFF], dst + (wave * NI + i) * RPI * D * 2);
    cur.step(RPI * row_bytes);
  }
  // the same where rows of the tile from n on, or chunks from `chunks` on, do not exist: they become zero
  __device__ __forceinline__ void part(Cursor& cur, int64_t row_bytes, unsigned dst, int wave, int lane, int i, int n, int chunks) const {
    asm volatile("" : "+v"(lane));
    const int row = (wave * NI + i) * RPI, lr = lane / CPR, c = (lane % CPR) ^ swizzle<D, USE>(row + lr);
    const char* at = cur.at + (int64_t)lr * row_bytes + (c << 4);
    copy16_any(row + lr < n && c < chunks ? at : (const char*)&zero_piece, dst + row * D * 2);
    cur.step(RPI * row_bytes);
  }
};

// Operand addresses (LDS bytes) of a lane in a tile that starts at a multiple of a row.  The swizzles are exclusive-ors, so that one register holds the
// address and a constant flips the bits of step, channel tile and half.
template <int D>
struct RowRead {    // rows 32 t + nn, channels 16 s + 8 g .. + 7
  unsigned at;
  template <int USE> __device__ __forceinline__ void set(int nn, int g) { at = nn * D * 2 + ((g ^ swizzle<D, USE>(nn)) << 4); }   // (row 32 t + nn has nn's swizzle)
  __device__ __forceinline__ bf16x8 get(unsigned tile, int t, int s) const {
    return *(const __attribute__((address_space(3))) bf16x8*)(uintptr_t)(((tile + at) ^ (s << 5)) + t * 32 * D * 2);
  }
};
// channels 32 dt + nn, rows 16 s + 8 h + 4 g + 0..3 for h = 0, 1: the rows that a lane half g holds in registers 8 (s % 2) .. + 7 of the product
// over rows 32 (s / 2) .. + 31.
template <int D, int USE>
struct ColRead {
  static_assert(USE != ROWS, "");
  unsigned at;
  __device__ __forceinline__ void set(int lane) {
    const int g = lane >> 5, sl = lane & 15, g1 = (lane >> 4) & 1, row = 4 * g + (sl >> 2);
    at = row * D * 2 + (sl & 1) * 8 + (((2 * g1 + ((sl & 3) >> 1)) ^ swizzle<D, USE>(row)) << 4);
  }
  __device__ __forceinline__ bf16x8 get(unsigned tile, int dt, int s) const {
    uint4v r;
#pragma unroll
    for (int h = 0; h < 2; ++h) {   // (eight rows on, a BOTH tile's swizzle has one more bit)
      const unsigned p = ((tile + at) ^ ((dt << 6) | (USE == BOTH ? h << 5 : 0))) + (s * 16 + 8 * h) * D * 2;
      const uint2v u = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4v __attribute__((address_space(3)))*)(uintptr_t)p));
      r[2 * h] = u[0];
      r[2 * h + 1] = u[1];
    }
    return __builtin_bit_cast(bf16x8, r);
  }
};

// Bit i: does f hold of row i of 32, rows as two lane halves hold them in the registers of a product (f(r): of register r, row 8 (r / 4) + 4 g + r % 4).
template <typename F>
__device__ __forceinline__ uint32_t row_bits(int g, F&& f) {
  uint32_t b = 0;
#pragma unroll
  for (int r = 0; r < 16; ++r) b |= f(r) ? 1u << (8 * (r >> 2) + (r & 3)) : 0u;
  b <<= 4 * g;
  const auto sw = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return sw[0] | sw[1];
}

// Masked probabilities are exactly zero, but zero times a value that is not finite is not.  Run where a result came out not finite: the products of 32 rows' such
// values are added for the pairs that are seen, and the values taken out of the tile before its product.  The rows' factors are `none` (row_bits) zero, and
// positive elsewhere: an infinity stays what it is, or becomes NaN.  (Factors that are NaN spoil the product itself.)
template <int D, int USE, typename F>
__device__ __forceinline__ void set_aside(float16v (&acc)[D / 32], uint16_t* tile, int g, uint32_t none, F&& seen) {
  constexpr int KT = 32;
  uint32_t* t32 = (uint32_t*)tile;
  bool odd = false;
  for (int i = threadIdx.x; i < KT * D / 2; i += blockDim.x) odd = odd || (t32[i] & 0x7f80u) == 0x7f80u || (t32[i] & 0x7f800000u) == 0x7f800000u;
  if (!uniform(__syncthreads_or(odd))) return;
#pragma nounroll
  for (int i = 0; i < KT; ++i) {
    const bool s = seen(i);
    const float zero = (none >> i & 1) ? 0.f : 1.f;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint2v x = *(const uint2v*)(tile + i * D + (((4 * dt + q) ^ swizzle<D, USE>(i)) << 3) + 4 * g);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float v = __uint_as_float((j & 1) ? (x[j >> 1] & 0xffff0000u) : (x[j >> 1] << 16));
          if (s && !(fabsf(v) <= 3.4028235e38f)) acc[dt][4 * q + j] += zero * v;
        }
      }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < KT * D / 2; i += blockDim.x) {
    const uint32_t x = t32[i];
    t32[i] = ((x & 0x7f80u) == 0x7f80u ? 0u : (x & 0xffffu)) | ((x & 0x7f800000u) == 0x7f800000u ? 0u : (x & 0xffff0000u));
  }
  __syncthreads();
}
// Not zero where any of the values is not finite.
template <int N>
__device__ __forceinline__ bool any_odd(const float16v (&x)[N]) {
  float probe = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) probe = __builtin_fmaf(x[i][r], 0.f, probe);
  return probe != 0.f;
}

// N products of which product i takes an operand load(i), requested PF products ahead.
template <int N, int PF, typename L, typename M>
__device__ __forceinline__ void products(L&& load, M&& mul) {
  decltype(load(0)) A[PF];
#pragma unroll
  for (int i = 0; i < PF; ++i) A[i] = load(i);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const auto a = A[i % PF];
    if (i + PF < N) A[i % PF] = load(i + PF);
    mul(i, a);
  }
}
// The order of such a run: the reads of PF operands, then one product and one operand's reads in turn.
template <int N, int PF, int READS>
__device__ __forceinline__ void in_turn() {
  __builtin_amdgcn_sched_group_barrier(0x100, PF * READS, 0);
#pragma unroll
  for (int i = 0; i < N - PF; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, PF, 0);
}

// Stores a row of which two lane halves hold the channels as accumulators, times f.  Per 16 channels a lane holds two groups of four that interleave with its
// partner's: after swapping one each it has 8 consecutive channels.  put(c, o): channels c .. c + 7.
template <int DT, typename F>
__device__ __forceinline__ void each_piece(const float16v (&acc)[DT], float f, int g, F&& put) {
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float o[8];
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[dt][8 * j + b] * f), __float_as_uint(acc[dt][8 * j + 4 + b] * f), false, false);
        o[b] = __uint_as_float(sw[0]);
        o[4 + b] = __uint_as_float(sw[1]);
      }
      put(dt * 32 + j * 16 + g * 8, o);
    }
}
__device__ __forceinline__ uint4v pack8(const float (&o)[8]) { return uint4v{pack2(o[0], o[1]), pack2(o[2], o[3]), pack2(o[4], o[5]), pack2(o[6], o[7])}; }

struct Row { bool live; int token, head, last; };   // last: the last key the row sees, -1 none

__device__ __forceinline__ int last_key(int causal, int token, int nq, int nk) {
  return causal ? (token + nk - nq < nk - 1 ? token + nk - nq : nk - 1) : nk - 1;
}
__device__ __forceinline__ Row query_row(const SeqParams& p, int kvh, int r, int nq, int nk) {
  Row w;
  w.live = r < nq * p.group;
  w.token = w.live ? (int)((unsigned)r / (unsigned)p.group) : 0;
  w.head = kvh * p.group + (w.live ? r - w.token * p.group : 0);
  w.last = w.live ? last_key(p.causal, w.token, nq, nk) : -1;
  return w;
}

}  // namespace seq
}  // namespace fa
