// Attention over sequences with fp32 products (v_mfma_f32_32x32x2_f32), forward and backward: FREQATTN_F32 tensors, and bf16 ones that
// the bf16 kernels do not take (rows that are not whole aligned 16-byte pieces).
//
//   S = scale Q K^T,  O = softmax(S) V,  lse = log sum exp S;  delta = rowsum(dO O),  P = exp(S - lse),  dS = P (dO V^T - delta),
//   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
//
// A wave owns 32 rows - query rows in the forward and dQ kernels, key rows in the dK / dV kernel - as columns of transposed products: S^T = K Q^T
// leaves a column (a query) on two lanes, whose accumulator registers are then the B operand of O^T += V^T P^T as they stand: step
// r of v_mfma_f32_32x32x2 takes k = 8 (r / 4) + r % 4 + 4 g from lane half g, which is where register r of the product before it lies.
// The other side passes through LDS in tiles of 32 rows, widened to fp32.  A workgroup owns 32 rows; its waves take the other side's tiles in turn, each through
// LDS of its own (no barrier until their sums are joined at the end), in the forward and dQ kernels with the next tile's loads under way in registers: fp32 products are slow
// enough that a tile per 32 rows is no burden on the caches, and short sequences still give every wave something to do.  The sums over keys (dQ) and over queries (dK, dV) are taken by
// different kernels, each by one workgroup in a fixed order, instead of by atomics: 7 products instead of 5, equal bits every time.
// Bound, on long rows: 8 heads of 4096 rows, full, run at 85 TFLOP/s forward (404 us, head_dim 64; 71 at 128, 964 us) and 100 backward, counting its own seven products (1202 us; 89
// and 2715), of the 134 that a large library product reaches, with one workgroup of four or eight waves a compute unit (LDS).  Short sequences by the
// longest row's chain of tiles (three sequences of 701, 333 and 100 rows, 6 / 3 heads of 48: forward 28 us, dQ 34, dK and dV 71; with four waves and the next rows in
// registers dK and dV took 89).  The other side is not cut into pieces: one token against a cache of 16,384 rows, 32 / 8 heads of 128, runs on 8 workgroups and takes
// 929 us, 32 such tokens on 256 take 955 (4.5 TB/s).
#include <hip/hip_runtime.h>

#include "seq_common.h"
#include "tokens.h"

namespace fa {

typedef float float4v __attribute__((ext_vector_type(4)));
typedef int int4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef unsigned int uint2v __attribute__((ext_vector_type(2)));

namespace {

struct Bf16 { uint16_t u; };
struct E4m3 { uint8_t u; };    // a code of a cache held in 8 bits
__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(E4m3 x) { return __builtin_amdgcn_cvt_f32_fp8((int)x.u, 0); }
__device__ __forceinline__ float widen(Bf16 x) { return __uint_as_float((uint32_t)x.u << 16); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(Bf16* p, float x) { p->u = __builtin_bit_cast(uint16_t, (__bf16)x); }

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int TR = 32;    // rows of a tile

__device__ __forceinline__ float16v zero16() {
  float16v z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}

// A wave's LDS writes are done before what follows reads them (LDS of one wave needs no barrier).
__device__ __forceinline__ void wave_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

template <typename T>
__device__ __forceinline__ const T* row_of(const HeadsPtr& v, int seq, int64_t row, int head) {
  return (const T*)v.p + (int64_t)seq * v.bs + row * v.ts + (int64_t)head * v.hs;
}
template <typename T>
__device__ __forceinline__ T* row_of_out(const HeadsPtr& v, int seq, int64_t row, int head) {
  return (T*)const_cast<char*>(v.p) + (int64_t)seq * v.bs + row * v.ts + (int64_t)head * v.hs;
}

// Four channels c .. c + 3 of a row, zero from d on.
template <typename T>
__device__ __forceinline__ float4v chunk(const T* row, int c, int d, bool live, int vec) {
  float4v x = {0.f, 0.f, 0.f, 0.f};
  if (!live || c >= d) return x;
  if (vec && sizeof(T) > 1) {
    if constexpr (sizeof(T) == 4) return *(const float4v*)(row + c);
    const uint2v u = *(const uint2v*)(row + c);
    return float4v{__uint_as_float(u[0] << 16), __uint_as_float(u[0] & 0xffff0000u), __uint_as_float(u[1] << 16), __uint_as_float(u[1] & 0xffff0000u)};
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (c + j < d) x[j] = widen(row[c + j]);
  return x;
}

// The lane's share of a row as an operand over the channels: chunk s holds channels 8 s + 4 g .. + 3.
template <typename T, int D>
struct RowOperand {
  float4v x[D / 8];
  __device__ __forceinline__ void load(const T* row, int g, int d, bool live, int vec) {
#pragma unroll
    for (int s = 0; s < D / 8; ++s) x[s] = chunk(row, 8 * s + 4 * g, d, live, vec);
  }
};

// tile (32 rows, LDS, stride D + 4) x operand: rows of the tile on registers, the operand's row on the lane
template <typename T, int D>
__device__ __forceinline__ float16v product(const float* tile, const RowOperand<T, D>& b, int nn, int g) {
  float16v acc = zero16();
#pragma unroll
  for (int s = 0; s < D / 8; ++s) {
    const float4v a = *(const float4v*)(tile + nn * (D + 4) + 8 * s + 4 * g);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b.x[s][j], acc, 0, 0, 0);
  }
  return acc;
}

// acc[dt] (channels on registers) += tile^T x w, w: one value per tile row on the registers, as product() leaves them
template <int D>
__device__ __forceinline__ void accumulate(float16v (&acc)[D / 32], const float* tile, const float16v& w, int nn, int g) {
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const float* row = tile + (8 * (r >> 2) + (r & 3) + 4 * g) * (D + 4);
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) acc[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(row[dt * 32 + nn], w[r], acc[dt], 0, 0, 0);
  }
}

// A product of a probability that is exactly zero and a value that is not finite is NaN on the matrix core, but a masked pair contributes nothing.  So where a
// tile has masked pairs and values that are not finite, their products are added to the rows that do see them and they are taken out of the tile.  Rare:
// tiles without them pay one comparison per value.  `seen(i)`: does the lane's row see row i of the tile.  w: the products' factors; an infinity
// stays what it is where its factor is positive, and becomes NaN where it is zero - or `zero` says so of all: a key or a query that is not finite has scores of +inf
// or NaN, whose row is NaN anyway, or of -inf, and dS zero.  (Factors that are NaN spoil the product itself.)
template <int D, typename F>
__device__ __forceinline__ void set_aside(float16v (&acc)[D / 32], float* tile, int lane, int g, const float16v& w, bool zero, F&& seen) {
  bool odd = false;
  for (int i = lane; i < TR * D; i += 64) odd = odd || !(fabsf(tile[i / D * (D + 4) + i % D]) <= 3.4028235e38f);
  if (__builtin_amdgcn_ballot_w64(odd) == 0) return;
  uint32_t none = 0;     // bit i: row i's factor is zero (the lane halves hold four rows each in turn)
#pragma unroll
  for (int r = 0; r < 16; ++r) none |= zero || !(w[r] != 0.f) ? 1u << (8 * (r >> 2) + (r & 3)) : 0u;
  none <<= 4 * g;
  none |= (uint32_t)__shfl_xor((int)none, 32);
#pragma nounroll
  for (int i = 0; i < TR; ++i) {
    const bool s = seen(i);
    const float f = (none >> i & 1) ? 0.f : 1.f;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float x = tile[i * (D + 4) + dt * 32 + 8 * (r >> 2) + 4 * g + (r & 3)];
        if (s && !(fabsf(x) <= 3.4028235e38f)) acc[dt][r] += f * x;
      }
  }
  wave_lds();
  for (int i = lane; i < TR * D; i += 64) {
    float& x = tile[i / D * (D + 4) + i % D];
    if (!(fabsf(x) <= 3.4028235e38f)) x = 0.f;
  }
  wave_lds();
}

// What a query row is: token, head, and the last key it sees.
struct Row { bool live; int token, head, last; };

__device__ __forceinline__ Row query_row(const SeqParams& p, int kvh, int r, int nq, int nk) {
  Row w;
  w.live = r < nq * p.group;
  w.token = w.live ? r / p.group : 0;
  w.head = kvh * p.group + (w.live ? r - w.token * p.group : 0);
  w.last = !w.live ? -1 : p.causal ? (w.token + nk - nq < nk - 1 ? w.token + nk - nq : nk - 1) : nk - 1;
  return w;
}

// 32 rows of the other side on their way into the wave's tile; row(i) gives the address of row i, nullptr where there is none.
template <typename T, int D>
struct Fetch {
  float4v x[TR * D / 256];
  template <typename F> __device__ __forceinline__ void load(int lane, int d, int vec, F&& row) {
#pragma unroll
    for (int j = 0; j < TR * D / 256; ++j) {
      const int i = j * 64 + lane, r = i / (D / 4), c = i % (D / 4) * 4;
      const T* at = row(r);
      x[j] = chunk(at, c, d, at != nullptr, vec);
    }
  }
  // codes to values: times the scale 2^(byte - 127) of their row, by(r) the byte (255: NaN)
  template <typename F> __device__ __forceinline__ void scale(int lane, F&& by) {
#pragma unroll
    for (int j = 0; j < TR * D / 256; ++j) {
      const int e = by((j * 64 + lane) / (D / 4));
#pragma unroll
      for (int k = 0; k < 4; ++k) x[j][k] = e == 255 ? __builtin_nanf("") : __builtin_amdgcn_ldexpf(x[j][k], e - 127);
    }
  }
  __device__ __forceinline__ void store(float* tile, int lane) {
#pragma unroll
    for (int j = 0; j < TR * D / 256; ++j) {
      const int i = j * 64 + lane, r = i / (D / 4), c = i % (D / 4) * 4;
      *(float4v*)(tile + r * (D + 4) + c) = x[j];
    }
  }
};

// Waves of a workgroup, by the LDS that their tiles take.
template <int D> constexpr int waves() { return D == 64 ? 8 : 4; }
template <int D> constexpr int tile_floats() { return TR * (D + 4); }

// Adds the waves' accumulators up in the order of the waves, each wave a share of the registers, and hands the sums out: put(register, sum) with
// register dt * 16 + r.  `weight(w)`: factor of wave w's values.  lds holds waves * D * 32 floats.
template <int D, int NW, typename W, typename P>
__device__ __forceinline__ void join_waves(const float16v (&acc)[D / 32], float* lds, int wave, int lane, W&& weight, P&& put) {
  constexpr int N = D / 2;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) lds[(wave * N + dt * 16 + r) * 64 + lane] = acc[dt][r];
  __syncthreads();
  for (int i = wave * (N / NW); i < (wave + 1) * (N / NW); ++i) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) s += weight(w) * lds[(w * N + i) * 64 + lane];
    put(i, s);
  }
}
__device__ __forceinline__ int channel_of(int reg, int g) { return (reg >> 4) * 32 + 8 * ((reg & 15) >> 2) + 4 * g + (reg & 3); }

// KV: type of the keys and values; E4m3 takes them from a cache held in 8 bits with the scales `sc`.
template <typename T, int D, typename KV = T>
__global__ void __launch_bounds__(64 * waves<D>(), 1) k_seq_generic_fwd(SeqParams p, Cache8Scales sc) {
  constexpr int NW = waves<D>(), TF = tile_floats<D>();
  __shared__ __attribute__((aligned(16))) float tiles[NW][2 * TF];
  __shared__ float ms[NW][64], ls[NW][64];
  const int lane = threadIdx.x & 63, nn = lane & 31, g = lane >> 5, wave = threadIdx.x >> 6;
  const int kvh = (int)(blockIdx.x % (unsigned)p.hk);
  int seq, tile;
  if (!seq_query_tile(p, TR, lane, (int)(blockIdx.x / (unsigned)p.hk), seq, tile)) return;
  const SeqRange q = seq_range(p.q_off, p.q_len, p.q_rows, seq), k = seq_range(p.k_off, p.k_len, p.k_rows, seq);
  if ((int64_t)tile * TR >= (int64_t)q.n * p.group) return;
  const Row row = query_row(p, kvh, tile * TR + nn, q.n, k.n);
  RowOperand<T, D> Q;
  Q.load(row_of<T>(p.q, q.seq, q.base + row.token, row.head), g, p.d, row.live, p.vec);
  const int last = query_row(p, kvh, min(tile * TR + TR - 1, q.n * p.group - 1), q.n, k.n).last;    // of the tile: its last row sees the most
  const int first_last = query_row(p, kvh, tile * TR, q.n, k.n).last;
  const float c2 = p.scale * LOG2E;
  float *Ks = tiles[wave], *Vs = tiles[wave] + TF;
  Fetch<KV, D> fk, fv;
  auto fetch = [&](int key0) {
    fk.load(lane, p.d, p.vec, [&](int r) { return key0 + r < k.n ? row_of<KV>(p.k, k.seq, k.base + key0 + r, kvh) : nullptr; });
    fv.load(lane, p.d, p.vec, [&](int r) { return key0 + r < k.n ? row_of<KV>(p.v, k.seq, k.base + key0 + r, kvh) : nullptr; });
    if constexpr (sizeof(KV) == 1) {
      const int64_t at = (int64_t)k.seq * sc.blocks * p.hk + kvh;
      auto byte = [&](const uint8_t* s, int r) { return key0 + r < k.n ? (int)s[at + (int64_t)((key0 + r) >> sc.shift) * p.hk] : 127; };
      fk.scale(lane, [&](int r) { return byte(sc.k, r); });
      fv.scale(lane, [&](int r) { return byte(sc.v, r); });
    }
  };
  float16v O[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) O[dt] = zero16();
  float m = -INFINITY, l = 0.f;
  if (wave * TR <= last) fetch(wave * TR);
  for (int key0 = wave * TR; key0 <= last; key0 += NW * TR) {
    fk.store(Ks, lane);
    fv.store(Vs, lane);
    wave_lds();
    if (key0 + NW * TR <= last) fetch(key0 + NW * TR);
    float16v S = product<T, D>(Ks, Q, nn, g);
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int key = key0 + 8 * (r >> 2) + 4 * g + (r & 3);
      S[r] = key <= row.last ? S[r] * c2 : -INFINITY;
      mx = fmaxf(mx, S[r]);
    }
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float mn = fmaxf(m, mx), ref = mn == -INFINITY ? 0.f : mn;
    const float alpha = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - ref);
    m = mn;
    l *= alpha;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) O[dt][r] *= alpha;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      S[r] = __builtin_amdgcn_exp2f(S[r] - ref);      // (0 where masked)
      l += S[r];
    }
    if (p.causal && key0 + TR - 1 > first_last) set_aside<D>(O, Vs, lane, g, S, false, [&](int i) { return key0 + i <= row.last; });
    accumulate<D>(O, Vs, S, nn, g);
    wave_lds();
  }
  l += __shfl_xor(l, 32);
  ms[wave][lane] = m;
  ls[wave][lane] = l;
  __syncthreads();
  float top = -INFINITY, sum = 0.f, w[NW];
#pragma unroll
  for (int i = 0; i < NW; ++i) top = fmaxf(top, ms[i][lane]);
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    w[i] = ls[i][lane] == 0.f ? 0.f : __builtin_amdgcn_exp2f(ms[i][lane] - top);
    sum += w[i] * ls[i][lane];
  }
  T* dst = row_of_out<T>(p.o, q.seq, q.base + row.token, row.head);
  const float inv = row.last < 0 ? 0.f : 1.f / sum;
  join_waves<D, NW>(O, tiles[0], wave, lane, [&](int i) { return w[i]; }, [&](int i, float x) {
    const int c = channel_of(i, g);
    if (row.live && c < p.d) put(dst + c, x * inv);
  });
  if (row.live && p.lse && g == 0 && wave == 0)
    p.lse[(int64_t)row.head * p.lse_rows + (p.q_off ? q.base : (int64_t)seq * p.q_rows) + row.token] = row.last < 0 ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * LN2;
}

// dQ, and the row sums delta that the other kernel reads.
template <typename T, int D>
__global__ void __launch_bounds__(64 * waves<D>(), 1) k_seq_generic_dq(SeqParams p) {
  constexpr int NW = waves<D>(), TF = tile_floats<D>();
  __shared__ __attribute__((aligned(16))) float tiles[NW][2 * TF];
  const int lane = threadIdx.x & 63, nn = lane & 31, g = lane >> 5, wave = threadIdx.x >> 6;
  const int kvh = (int)(blockIdx.x % (unsigned)p.hk);
  int seq, tile;
  if (!seq_query_tile(p, TR, lane, (int)(blockIdx.x / (unsigned)p.hk), seq, tile)) return;
  const SeqRange q = seq_range(p.q_off, p.q_len, p.q_rows, seq), k = seq_range(p.k_off, p.k_len, p.k_rows, seq);
  if ((int64_t)tile * TR >= (int64_t)q.n * p.group) return;
  const Row row = query_row(p, kvh, tile * TR + nn, q.n, k.n);
  RowOperand<T, D> Q, dO;
  Q.load(row_of<T>(p.q, q.seq, q.base + row.token, row.head), g, p.d, row.live, p.vec);
  dO.load(row_of<T>(p.dout, q.seq, q.base + row.token, row.head), g, p.d, row.live, p.vec);
  float delta = 0.f;
  {
    const T* o = row_of<T>(p.o, q.seq, q.base + row.token, row.head);
#pragma unroll
    for (int s = 0; s < D / 8; ++s) {
      const float4v x = chunk(o, 8 * s + 4 * g, p.d, row.live && row.last >= 0, p.vec);
#pragma unroll
      for (int j = 0; j < 4; ++j) delta += row.last >= 0 ? x[j] * dO.x[s][j] : 0.f;
    }
    delta += __shfl_xor(delta, 32);
  }
  const int64_t at = (int64_t)row.head * p.lse_rows + (p.q_off ? q.base : (int64_t)seq * p.q_rows) + row.token;
  const float lse2 = row.live && row.last >= 0 ? p.lse[at] * LOG2E : 0.f;
  const int last = query_row(p, kvh, min(tile * TR + TR - 1, q.n * p.group - 1), q.n, k.n).last;
  const int first_last = query_row(p, kvh, tile * TR, q.n, k.n).last;
  const float c2 = p.scale * LOG2E;
  float *Ks = tiles[wave], *Vs = tiles[wave] + TF;
  Fetch<T, D> fk, fv;
  auto fetch = [&](int key0) {
    fk.load(lane, p.d, p.vec, [&](int r) { return key0 + r < k.n ? row_of<T>(p.k, k.seq, k.base + key0 + r, kvh) : nullptr; });
    fv.load(lane, p.d, p.vec, [&](int r) { return key0 + r < k.n ? row_of<T>(p.v, k.seq, k.base + key0 + r, kvh) : nullptr; });
  };
  if (sizeof(T) == 2 && first_last < SHORT_ROW && last >= 0) {    // short rows of bf16: delta from the probabilities
    __shared__ float sums[NW][TR];
    static_assert(NW * TR >= SHORT_ROW, "");
    float sum = 0.f;
    const int key0 = wave * TR;
    if (key0 < SHORT_ROW && key0 <= last) {
      fetch(key0);
      fk.store(Ks, lane);
      fv.store(Vs, lane);
      wave_lds();
      const float16v S = product<T, D>(Ks, Q, nn, g), dP = product<T, D>(Vs, dO, nn, g);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float x = __builtin_amdgcn_exp2f(S[r] * c2 - lse2) * dP[r];
        sum += key0 + 8 * (r >> 2) + 4 * g + (r & 3) <= row.last ? x : 0.f;
      }
      sum += __shfl_xor(sum, 32);
      wave_lds();
    }
    if (g == 0) sums[wave][nn] = sum;
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < SHORT_ROW / TR; ++w) sum += sums[w][nn];
    if (row.last < SHORT_ROW) delta = sum;
  }
  if (row.live && g == 0 && wave == 0) p.delta[at] = delta;
  float16v A[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) A[dt] = zero16();
  if (wave * TR <= last) fetch(wave * TR);
  for (int key0 = wave * TR; key0 <= last; key0 += NW * TR) {
    fk.store(Ks, lane);
    fv.store(Vs, lane);
    wave_lds();
    if (key0 + NW * TR <= last) fetch(key0 + NW * TR);
    float16v S = product<T, D>(Ks, Q, nn, g);
    const float16v dP = product<T, D>(Vs, dO, nn, g);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int key = key0 + 8 * (r >> 2) + 4 * g + (r & 3);
      const float x = __builtin_amdgcn_exp2f(S[r] * c2 - lse2) * (dP[r] - delta);
      S[r] = key <= row.last ? x : 0.f;
    }
    if (p.causal && key0 + TR - 1 > first_last) set_aside<D>(A, Ks, lane, g, S, true, [&](int i) { return key0 + i <= row.last; });
    accumulate<D>(A, Ks, S, nn, g);
    wave_lds();
  }
  __syncthreads();
  T* dst = row_of_out<T>(p.dq, q.seq, q.base + row.token, row.head);
  join_waves<D, NW>(A, tiles[0], wave, lane, [](int) { return 1.f; }, [&](int i, float x) {
    const int c = channel_of(i, g);
    if (row.live && c < p.d) put(dst + c, x * p.scale);
  });
}

// dK and dV of 32 keys, over all query rows of the sequence and group that see any of them.
template <typename T, int D>
__global__ void __launch_bounds__(64 * waves<D>(), 1) k_seq_generic_dkv(SeqParams p) {
  constexpr int NW = waves<D>(), TF = tile_floats<D>();
  __shared__ __attribute__((aligned(16))) float tiles[NW][2 * TF];
  __shared__ __attribute__((aligned(16))) float Ls[NW][TR], Ds[NW][TR];
  __shared__ __attribute__((aligned(16))) int Last[NW][TR];
  const int lane = threadIdx.x & 63, nn = lane & 31, g = lane >> 5, wave = threadIdx.x >> 6;
  const int kvh = (int)(blockIdx.x % (unsigned)p.hk);
  int seq, tile;
  if (!seq_key_tile(p, TR, lane, (int)(blockIdx.x / (unsigned)p.hk), seq, tile)) return;
  const SeqRange q = seq_range(p.q_off, p.q_len, p.q_rows, seq), k = seq_range(p.k_off, p.k_len, p.k_rows, seq);
  if ((int64_t)tile * TR >= k.n) return;
  const int key = tile * TR + nn;
  const bool live = key < k.n;
  RowOperand<T, D> K, V;
  K.load(row_of<T>(p.k, k.seq, k.base + (live ? key : 0), kvh), g, p.d, live, p.vec);
  V.load(row_of<T>(p.v, k.seq, k.base + (live ? key : 0), kvh), g, p.d, live, p.vec);
  float16v dK[D / 32], dV[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) { dK[dt] = zero16(); dV[dt] = zero16(); }
  const float c2 = p.scale * LOG2E;
  const int64_t rows = (int64_t)q.n * p.group;
  // the first token that sees the tile's first key
  int first = p.causal ? tile * TR - (k.n - q.n) : 0;
  if (first < 0) first = 0;
  const int last_key = min(tile * TR + TR - 1, k.n - 1);
  float *Qs = tiles[wave], *Gs = tiles[wave] + TF;
  const float per_group = 1.f / (float)p.group;
  auto fetch = [&](int r0) {
    // tokens of the tile's rows from the first row's: what is left to divide is below group + 32
    const int t0 = __builtin_amdgcn_readfirstlane((int)((unsigned)r0 / (unsigned)p.group)), rem = r0 - t0 * p.group;
    const auto row_at = [&](int r) {
      const int up = (int)(((float)(rem + r) + 0.5f) * per_group);
      Row w;
      w.live = r0 + r < rows;
      w.token = t0 + up;
      w.head = kvh * p.group + rem + r - up * p.group;
      w.last = !w.live ? -1 : p.causal ? min(w.token + k.n - q.n, k.n - 1) : k.n - 1;
      return w;
    };
    const auto at = [&](const HeadsPtr& v, int r) -> const T* {
      const Row row = row_at(r);
      return row.live ? row_of<T>(v, q.seq, q.base + row.token, row.head) : nullptr;
    };
    Fetch<T, D> f;
    f.load(lane, p.d, p.vec, [&](int r) { return at(p.q, r); });
    f.store(Qs, lane);
    f.load(lane, p.d, p.vec, [&](int r) { return at(p.dout, r); });
    f.store(Gs, lane);
    const Row row = row_at(nn);
    const int64_t i = (int64_t)row.head * p.lse_rows + (p.q_off ? q.base : (int64_t)seq * p.q_rows) + row.token;
    const bool some = row.live && row.last >= 0;
    if (g == 0) {
      Ls[wave][nn] = some ? p.lse[i] * LOG2E : 0.f;
      Ds[wave][nn] = some ? p.delta[i] : 0.f;
      Last[wave][nn] = row.last;
    }
  };
  const int64_t start = (int64_t)first * p.group / TR * TR + wave * TR;
  for (int64_t r0 = start; r0 < rows; r0 += NW * TR) {
    fetch((int)r0);      // (the registers are full without the next tile's rows; the other waves fill the wait)
    wave_lds();
    float16v S = product<T, D>(Qs, K, nn, g);
    float16v dP = product<T, D>(Gs, V, nn, g);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4v lse = *(const float4v*)&Ls[wave][8 * i + 4 * g], del = *(const float4v*)&Ds[wave][8 * i + 4 * g];
      const int4v last = *(const int4v*)&Last[wave][8 * i + 4 * g];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = 4 * i + j;
        const float x = __builtin_amdgcn_exp2f(S[r] * c2 - lse[j]), y = x * (dP[r] - del[j]);
        const bool seen = live && key <= last[j];
        S[r] = seen ? x : 0.f;
        dP[r] = seen ? y : 0.f;
      }
    }
    if (Last[wave][0] < last_key || Last[wave][TR - 1] < last_key) {   // some pair is masked: queries before the diagonal, rows behind the last query
      set_aside<D>(dV, Gs, lane, g, S, false, [&](int i) { return live && key <= Last[wave][i]; });
      set_aside<D>(dK, Qs, lane, g, dP, true, [&](int i) { return live && key <= Last[wave][i]; });
    }
    accumulate<D>(dV, Gs, S, nn, g);
    accumulate<D>(dK, Qs, dP, nn, g);
    wave_lds();
  }
  __syncthreads();
  const auto store = [&](const HeadsPtr& v, const float16v (&acc)[D / 32], float f) {
    T* dst = row_of_out<T>(v, k.seq, k.base + (live ? key : 0), kvh);
    join_waves<D, NW>(acc, tiles[0], wave, lane, [](int) { return 1.f; }, [&](int i, float x) {
      const int c = channel_of(i, g);
      if (live && c < p.d) put(dst + c, x * f);
    });
  };
  store(p.dk, dK, p.scale);
  __syncthreads();
  store(p.dv, dV, 1.f);
}

template <typename T, int D, typename KV = T>
hipError_t fwd(SeqParams p, hipStream_t st, const Cache8Scales& sc = {}) {
  p.slots = (int)seq_slots(p.q_off != nullptr, p.q_rows, p.nseq, p.group, TR);
  if (p.slots == 0) return hipSuccess;
  hipLaunchKernelGGL((k_seq_generic_fwd<T, D, KV>), dim3((unsigned)p.slots * (unsigned)p.hk), dim3(64 * waves<D>()), 0, st, p, sc);
  return hipGetLastError();
}
template <typename T, int D>
hipError_t bwd(SeqParams p, hipStream_t st) {
  p.slots = (int)seq_slots(p.q_off != nullptr, p.q_rows, p.nseq, p.group, TR);
  if (p.slots > 0) hipLaunchKernelGGL((k_seq_generic_dq<T, D>), dim3((unsigned)p.slots * (unsigned)p.hk), dim3(64 * waves<D>()), 0, st, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  p.slots = (int)seq_slots(p.k_off != nullptr, p.k_rows, p.nseq, 1, TR);
  if (p.slots > 0) hipLaunchKernelGGL((k_seq_generic_dkv<T, D>), dim3((unsigned)p.slots * (unsigned)p.hk), dim3(64 * waves<D>()), 0, st, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_seq_generic_fwd(const SeqParams& p, int dtype, hipStream_t st) {
  if (dtype == FREQATTN_BF16) return p.d <= 64 ? fwd<Bf16, 64>(p, st) : fwd<Bf16, 128>(p, st);
  return p.d <= 64 ? fwd<float, 64>(p, st) : fwd<float, 128>(p, st);
}
hipError_t launch_cache8_generic(const SeqParams& p, const Cache8Scales& sc, int dtype, hipStream_t st) {
  if (dtype == FREQATTN_BF16) return p.d <= 64 ? fwd<Bf16, 64, E4m3>(p, st, sc) : fwd<Bf16, 128, E4m3>(p, st, sc);
  return p.d <= 64 ? fwd<float, 64, E4m3>(p, st, sc) : fwd<float, 128, E4m3>(p, st, sc);
}
hipError_t launch_seq_generic_bwd(const SeqParams& p, int dtype, hipStream_t st) {
  if (dtype == FREQATTN_BF16) return p.d <= 64 ? bwd<Bf16, 64>(p, st) : bwd<Bf16, 128>(p, st);
  return p.d <= 64 ? bwd<float, 64>(p, st) : bwd<float, 128>(p, st);
}

}  // namespace fa
