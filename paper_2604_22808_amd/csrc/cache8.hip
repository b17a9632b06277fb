// Caches held in 8 bits: new rows appended, values read back.
//
// A block of 2^shift rows of a sequence and head has one scale 2^(e - 127), the smallest that brings its largest value to 448 or less (the largest e4m3 value); a code
// is x 2^(127 - e) to the nearest e4m3 value, ties to even.  Scales are powers of two so that a value in e4m3 keeps its bits when a block's scale grows:
// only values that fall among the subnormal codes are rounded again.  With no smaller byte than 10 every value is a normal number in fp32 and exact in bf16.
//
// Bound by memory: 16 x 4096 packed rows of 8 heads of 128 take 83 us to append (4.8 TB/s; blocks of 16 rows 81), 80 to read back (5.0).  A workgroup, or a wave, appends to one block
// of one head of K or V (nobody else writes there): largest value of the new rows, then codes; rows that the block holds already are rewritten only where its scale has grown.
#include "rows.h"
#include "seq_common.h"
#include "tokens.h"

namespace fa {

using namespace rows;

namespace {

constexpr int LEAST = 10;      // byte of the smallest scale
constexpr uint32_t INF_BITS = 0x7f800000u;

typedef float float2v __attribute__((ext_vector_type(2)));

// The smallest byte e with top <= 448 * 2^(e - 127) = 1.75 * 2^(e - 119), top by its bits.
__device__ __forceinline__ int least_byte(uint32_t top) {
  const int e = (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e > LEAST ? e : LEAST;
}

__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  int x = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, x, true);
}
__device__ __forceinline__ float coded(float x, int e) {   // what is coded: infinities become NaN
  return (__float_as_uint(x) & 0x7fffffffu) >= INF_BITS ? __builtin_nanf("") : __builtin_amdgcn_ldexpf(x, 127 - e);
}
__device__ __forceinline__ void values4(uint32_t codes, float (&x)[4]) {
  const float2v a = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
}

// Eight codes, channels c .. c + 7 of a row of d.
__device__ __forceinline__ uint2v load_codes(const uint8_t* row, int c, int d) {
  uint2v x = {0u, 0u};
  if (c + 8 <= d) return *(const uint2any*)(row + c);
#pragma unroll
  for (int j = 0; j < 7; ++j)
    if (c + j < d) x[j >> 2] |= (uint32_t)row[c + j] << (8 * (j & 3));
  return x;
}
__device__ __forceinline__ void store_codes(uint8_t* row, int c, int d, uint2v x) {
  if (c + 8 <= d) { *(uint2any*)(row + c) = x; return; }
#pragma unroll
  for (int j = 0; j < 7; ++j)
    if (c + j < d) row[c + j] = (uint8_t)(x[j >> 2] >> (8 * (j & 3)));
}

// Blocks that n new rows touch start at slot floor(offset / rows of a block) + 2 i of a launch: they are floor(n / rows) + 2 at most.
__device__ __forceinline__ void touched(const Cache8Params& p, int slot, int& seq, int& nth, SeqRange& q, int& length) {
  if (p.q_off && p.nseq <= 64) {      // a sequence a lane: everything about them in one load each, not in a chain of loads (16 x 4096 rows of 8 x 128 92 / 83 us)
    const int lane = threadIdx.x & 63, mine = min(lane, p.nseq - 1);
    const SeqRange r = seq_range(p.q_off, p.q_len, p.q_rows, mine);
    const int filled = p.k_len ? seq_clamp(p.k_len[mine], 0, p.k_rows) : p.k_rows, at = (r.base >> p.shift) + 2 * mine;
    const uint64_t before = __builtin_amdgcn_ballot_w64(lane < p.nseq && at <= slot);
    seq = before ? 63 - __builtin_clzll(before) : 0;
    nth = slot - __builtin_amdgcn_readlane(at, seq);
    q = SeqRange{0, __builtin_amdgcn_readlane(r.base, seq), __builtin_amdgcn_readlane(r.n, seq)};
    length = __builtin_amdgcn_readlane(filled, seq);
    return;
  }
  if (!p.q_off) {
    const int per = ((p.q_rows + (1 << p.shift) - 2) >> p.shift) + 1;
    seq = slot / per;
    nth = slot - seq * per;
  } else {
    int lo = 0, hi = p.nseq - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if ((seq_clamp(p.q_off[mid], 0, p.q_rows) >> p.shift) + 2 * mid <= slot) lo = mid; else hi = mid - 1;
    }
    seq = lo;
    nth = slot - ((seq_clamp(p.q_off[lo], 0, p.q_rows) >> p.shift) + 2 * lo);
  }
  q = seq_range(p.q_off, p.q_len, p.q_rows, seq);
  length = p.k_len ? seq_clamp(p.k_len[seq], 0, p.k_rows) : p.k_rows;
}

constexpr int THREADS = 256;

// W waves append to one block and head, IT pieces of eight channels a lane, which stay in registers between the two passes over them (and are all there are: block rows * pieces of a
// row <= 64 W IT).
template <typename T, int W, int IT>
__global__ void __launch_bounds__(THREADS) k_cache8_append(Cache8Params p, unsigned units) {
  __shared__ uint32_t tops[W];
  constexpr int LANES = 64 * W, EACH = THREADS / LANES;
  const int t = threadIdx.x % LANES;
  unsigned id = blockIdx.x * EACH + threadIdx.x / LANES;
  if (id >= units) return;
  const int head = (int)(id % (unsigned)p.heads);
  id /= (unsigned)p.heads;
  const bool is_v = id & 1;
  int seq, nth, length;
  SeqRange q;
  touched(p, (int)(id >> 1), seq, nth, q, length);
  if (nth < 0 || nth > (q.n >> p.shift) + 1) return;       // (offsets that do not ascend; slots that nobody's rows reach: the row numbers below stay within 31 bits)
  const int first = length - q.n, from = first > 0 ? first : 0;      // cache rows from .. length - 1 are new
  const int block = (from >> p.shift) + nth, lo = block << p.shift;
  if (q.n == 0 || lo >= length) return;                    // (of W waves all, or none)
  const int hi = min(lo + (1 << p.shift), length), start = max(lo, from);
  const HeadsPtr& in = is_v ? p.v : p.k;
  const HeadsPtr& out = is_v ? p.cv : p.ck;
  uint8_t* scale = (is_v ? p.vs : p.ks) + ((int64_t)seq * p.blocks + block) * p.heads + head;
  const int was = *scale, chunks = (p.d + 7) >> 3, items = (hi - start) * chunks;
  const T* src = (const T*)in.p + (int64_t)q.seq * in.bs + (int64_t)head * in.hs + (int64_t)(q.base + start - first) * in.ts;
  uint8_t* dst = (uint8_t*)const_cast<char*>(out.p) + (int64_t)seq * out.bs + (int64_t)head * out.hs;
  constexpr int N = 8 / PW<T>;
  Piece<T> x[IT][N];
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < IT; ++k) {
    const int i = t + k * LANES, r = i / chunks, c = (i - r * chunks) * 8;
    if (k > 0 && k * LANES >= items) break;                // (uniform)
#pragma unroll
    for (int h = 0; h < N; ++h) x[k][h].load(src + (int64_t)r * in.ts, c + h * PW<T>, i < items ? p.d : 0);
  }
#pragma unroll
  for (int k = 0; k < IT; ++k) {
    if (k > 0 && k * LANES >= items) break;
#pragma unroll
    for (int h = 0; h < N; ++h)
#pragma unroll
      for (int j = 0; j < PW<T>; ++j) {
        const uint32_t b = __float_as_uint(x[k][h].get(j)) & 0x7fffffffu;
        top = max(top, b < INF_BITS ? b : 0u);
      }
  }
  top = __float_as_uint(over_lanes<64>(__uint_as_float(top), [](float a, float b) { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); }));
  if constexpr (W > 1) {
    static_assert(EACH == 1, "");      // (a barrier for all waves of the workgroup)
    if ((t & 63) == 0) tops[t >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) top = max(top, tops[w]);
  }
  const int need = least_byte(top), e = start > lo ? max(was, need) : need;
#pragma unroll
  for (int k = 0; k < IT; ++k) {
    if (k > 0 && k * LANES >= items) break;
    const int i = t + k * LANES, r = i / chunks, c = (i - r * chunks) * 8;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = coded(x[k][j / PW<T>].get(j % PW<T>), e);
    if (i < items) store_codes(dst + (int64_t)(start + r) * out.ts, c, p.d, uint2v{codes4(v[0], v[1], v[2], v[3]), codes4(v[4], v[5], v[6], v[7])});
  }
  if (start > lo && e != was) {
    for (int i = t; i < (start - lo) * chunks; i += LANES) {
      const int r = i / chunks, c = (i - r * chunks) * 8;
      uint8_t* row = dst + (int64_t)(lo + r) * out.ts;
      const uint2v was_codes = load_codes(row, c, p.d);
      uint2v now;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float v[4];
        values4(was_codes[h], v);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __builtin_amdgcn_ldexpf(v[j], was - e);
        now[h] = codes4(v[0], v[1], v[2], v[3]);
      }
      store_codes(row, c, p.d, now);
    }
  }
  if (W > 1) __syncthreads();      // (every wave has the byte that it found)
  if (t == 0) *scale = (uint8_t)e;
}

template <typename T>
__global__ void __launch_bounds__(THREADS) k_cache8_read(Cache8Params p, int per) {
  unsigned id = blockIdx.x;
  const int part = (int)(id % (unsigned)per);
  id /= (unsigned)per;
  const bool is_v = id & 1;
  const int seq = (int)(id >> 1);
  const int length = p.k_len ? seq_clamp(p.k_len[seq], 0, p.k_rows) : p.k_rows;
  const unsigned chunks = (unsigned)(p.d + 7) >> 3, row_items = chunks * (unsigned)p.heads;
  const int64_t i = (int64_t)part * THREADS + threadIdx.x;
  if (i >= (int64_t)length * row_items) return;
  const int r = (int)(i / row_items);
  const unsigned in_row = (unsigned)(i - (int64_t)r * row_items);
  const int head = (int)(in_row / chunks), c = (int)(in_row - (unsigned)head * chunks) * 8;
  const HeadsPtr& from = is_v ? p.cv : p.ck;
  const HeadsPtr& to = is_v ? p.v : p.k;
  const int e = (is_v ? p.vs : p.ks)[((int64_t)seq * p.blocks + (r >> p.shift)) * p.heads + head];
  const uint2v codes = load_codes((const uint8_t*)from.p + (int64_t)seq * from.bs + (int64_t)r * from.ts + (int64_t)head * from.hs, c, p.d);
  float x[8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float y[4];
    values4(codes[h], y);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[4 * h + j] = e == 255 ? __builtin_nanf("") : __builtin_amdgcn_ldexpf(y[j], e - 127);
  }
  T* row = (T*)const_cast<char*>(to.p) + (int64_t)seq * to.bs + (int64_t)r * to.ts + (int64_t)head * to.hs;
#pragma unroll
  for (int h = 0; h < 8 / PW<T>; ++h) {
    Piece<T> o;
#pragma unroll
    for (int j = 0; j < PW<T>; j += 2) o.set(j, x[h * PW<T> + j], x[h * PW<T> + j + 1]);
    o.store(row, c + h * PW<T>, p.d);
  }
}

constexpr int64_t MOST_BLOCKS = (int64_t)1 << 23;

}  // namespace

hipError_t launch_cache8_append(const Cache8Params& p, int dtype, hipStream_t st) {
  const int64_t rows = (int64_t)1 << p.shift;
  const int64_t slots = p.q_off ? p.q_rows / rows + 2 * (int64_t)p.nseq : (int64_t)p.nseq * ((p.q_rows + rows - 2) / rows + 1);
  if (p.q_rows == 0 || slots == 0) return hipSuccess;
  if (slots >= MOST_BLOCKS || slots * 2 * p.heads >= MOST_BLOCKS) return hipErrorInvalidConfiguration;
  // a block and head a wave, four in a workgroup, up to 512 pieces; more are shared by four waves (blocks of 16 rows, 8 heads of 128, 16 x 4096 rows: 157 us by four waves each, 92 by one)
  const int64_t units = slots * 2 * p.heads, pieces = rows * ((p.d + 7) / 8);
  auto go = [&](auto type, auto w, auto it) {
    constexpr int each = THREADS / (64 * w.value);
    hipLaunchKernelGGL((k_cache8_append<decltype(type), w.value, it.value>), dim3((unsigned)((units + each - 1) / each)), dim3(THREADS), 0, st, p, (unsigned)units);
    return hipGetLastError();
  };
  auto with = [&](auto type) {
    using std::integral_constant;
    if (pieces <= 256) return go(type, integral_constant<int, 1>{}, integral_constant<int, 4>{});
    if (pieces <= 512) return go(type, integral_constant<int, 1>{}, integral_constant<int, 8>{});
    if (pieces <= 1024) return go(type, integral_constant<int, 4>{}, integral_constant<int, 4>{});
    return go(type, integral_constant<int, 4>{}, integral_constant<int, 16>{});
  };
  return dtype == FREQATTN_BF16 ? with(Bf16{}) : with(0.f);
}

hipError_t launch_cache8_read(const Cache8Params& p, int dtype, hipStream_t st) {
  const int64_t chunks = (p.d + 7) / 8, per = ((int64_t)p.k_rows * chunks * p.heads + THREADS - 1) / THREADS;
  if (per == 0 || p.nseq == 0) return hipSuccess;
  if (per >= MOST_BLOCKS || per * 2 * p.nseq >= MOST_BLOCKS) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)(per * 2 * p.nseq));
  if (dtype == FREQATTN_BF16) hipLaunchKernelGGL(k_cache8_read<Bf16>, grid, dim3(THREADS), 0, st, p, (int)per);
  else hipLaunchKernelGGL(k_cache8_read<float>, grid, dim3(THREADS), 0, st, p, (int)per);
  return hipGetLastError();
}

}  // namespace fa
