// Layer norm over the channels of token rows, forward and backward.
//
//   m = mean_c x_c,  r = (mean_c (x_c - m)^2 + eps)^-1/2,  h = (x - m) r,  y = h w + b
//   backward: g = dy w,  dx = r (g - mean g - h mean(g h)),  dw = sum over rows of dy h,  db = sum over rows of dy
//
// Bound by memory: the forward pass reads a row and writes one, the backward pass reads two and writes one.  A row lies in the registers of LPR lanes, or of W
// waves where it is longer than one wave holds, so that mean and centred squares are taken one after the other from one read; the next row is requested before the
// present one is worked on.  The mean as it comes out of fp32 is off by some of its steps, which rows far from zero would feel: the sum of the
// centred values, taken beside their squares, puts that right.  A wave keeps the weights and, in the backward pass, its share of dw and db in registers over all its rows;
// a workgroup adds its waves' shares in their order and stores one row of partial sums, k_norm_weights adds those: no atomics, equal calls give equal bits.
//
// Measured (us, bf16 unless said): 131,072 x 2048 forward 182 (5.9 TB/s), backward 326 (4.95); 2 x 65,536 x 1536 with weights each 142 and 235; 10,007 x 999 fp32 16 and 30, of which adding up
// dw and db 4 (rows of odd length start at any element); 60,000 x 173 13 and 33, bound by vector work and the loads' number, not their bytes; a single row 3 and 4.
#include <algorithm>

#include "rows.h"
#include "tokens.h"

namespace fa {

using namespace rows;

namespace {

// (var + eps)^-1/2: the instruction is within one step, which every channel of a row would have alike, so half of a Newton step goes on top.
__device__ __forceinline__ float inv_root(float v) {
  const float r = __builtin_amdgcn_rsqf(v);
  return __builtin_fmaf(0.5f * r, __builtin_fmaf(-v * r, r, 1.f), r);
}
// Not so: squares that have left fp32, or are about to.  Such a row is taken again in a scale of its own (own_scale).
__device__ __forceinline__ bool out_of_range(float v) { return v < 1e-30f || !(v < 3e38f); }

// Sums of N values over a row's lanes; those of W waves meet in LDS, in the order of the waves.  `turn` alternates between two places, so that one barrier a sum
// is enough.
template <int LPR, int W, int N>
__device__ __forceinline__ void row_sums(float (&x)[N], float (*lds)[W][4], int& turn, int wave) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = over_lanes<LPR>(x[i], add);
  if constexpr (W > 1) {
    float (*at)[4] = lds[turn];
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) at[wave][i] = x[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s = at[0][i];
#pragma unroll
      for (int w = 1; w < W; ++w) s += at[w][i];
      x[i] = s;
    }
  }
}

template <typename T>
__device__ __forceinline__ T* row_at(const RowsPtr& v, const NormParams& p, int64_t i) {
  return p.groups == 1 ? row_of<T>(v, p.rows, i) : (T*)v.p + (int64_t)blockIdx.y * v.bs + i * v.rs;
}

// Centred values d of a row's pieces times `times` (zero where there is no channel); mean: of the row times `times`.
template <typename T, int LPR, int W, int PT>
__device__ __forceinline__ void centre(const Piece<T> (&x)[PT], float (&d)[PT][PW<T>], const Place<T, LPR, W, PT>& at, int n, float mean, float times) {
#pragma unroll
  for (int i = 0; i < PT; ++i) {
    const int c = at.channel(i);
    const float m = c < n ? mean : 0.f;
#pragma unroll
    for (int j = 0; j < PW<T>; ++j) d[i][j] = __builtin_fmaf(x[i].get(j), times, -m);
    if (c < n && c + PW<T> > n) {
#pragma unroll
      for (int j = 1; j < PW<T>; ++j) d[i][j] = c + j < n ? d[i][j] : 0.f;
    }
  }
}

template <typename T, int PT>
__device__ __forceinline__ float sum_of(const Piece<T> (&x)[PT]) {
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < PT; ++i)
#pragma unroll
    for (int j = 0; j < PW<T>; ++j) s[j & 3] += x[i].get(j);
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// The largest magnitude of a row, by its bits (a NaN counts as the largest).
template <int LPR, int W>
__device__ __forceinline__ uint32_t row_top(float x, float (*lds)[W][4], int& turn, int wave) {
  auto larger = [](float a, float b) { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); };
  x = over_lanes<LPR>(__uint_as_float(__float_as_uint(x) & 0x7fffffffu), larger);
  if constexpr (W > 1) {
    float (*at)[4] = lds[turn];
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) at[wave][0] = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) x = larger(x, at[w][0]);
  }
  return __float_as_uint(x);
}

// How the centred values d = x times - mean of a row are taken.  eps: in their units.  back: the power of two that they are times the row's own.
struct Scale { float times, mean, eps, back; };

// A row whose variance v is out_of_range gets a scale of its own: the power of two by which its largest centred value, or eps^1/2 where that is larger, lies in 2^16 .. 2^17, so that neither
// sums nor squares leave fp32 and eps counts for what it is.  (A large row comes down first, since its sum has to stay.)  The mean is found twice, by division: what the first leaves of a
// row of equal values are a few steps of them, whose sum and mean have no rounding, so that such a row becomes zero exactly.  The row is read again piece by piece, which takes no
// registers; `count`: its channels, 0 of a row that does not exist.  Other rows of the wave stay as they are.
template <typename T, int LPR, int W, int PT>
__device__ __forceinline__ void own_scale(const T* row, const Place<T, LPR, W, PT>& at, int count, int n, float v, float (*lds)[W][4], int& turn, int wave, Scale& sc) {
  const float down = v < 3e38f ? 1.f : 0x1p-20f;
  float mean = 0.f;
  uint32_t top = 0;
  int pieces = PT;
  if constexpr (PT == 1) asm volatile("" : "+s"(pieces));      // (a loop all the same: nothing of it is moved up)
#pragma nounroll
  for (int pass = 0; pass < 3; ++pass) {      // sum, what is left of it, largest centred value
    float s[1] = {0.f};
    top = 0;
#pragma nounroll
    for (int k = 0; k < pieces; ++k) {
      asm volatile("" ::: "memory");
      Piece<T> x;
      const int c = at.channel(k);
      x.load(row, c, count);
#pragma unroll
      for (int j = 0; j < PW<T>; ++j) {
        const float y = c + j < count ? __builtin_fmaf(x.get(j), down, -mean) : 0.f;
        s[0] += y;
        top = max(top, __float_as_uint(y) & 0x7fffffffu);
      }
    }
    row_sums<LPR, W>(s, lds, turn, wave);
    top = row_top<LPR, W>(__uint_as_float(top), lds, turn, wave);
    if (pass < 2) mean += s[0] / (float)n;
  }
  const int e = (int)(max(top, __float_as_uint(sqrtf(sc.eps) * down)) >> 23);
  const float up = __uint_as_float((uint32_t)min(270 - e, 247) << 23), all = down * up;      // 2^120 at most: the smallest numbers are 2^-29 then
  // (equal values are zeros in any scale, also where their mean would leave fp32 in the scale of eps)
  if (out_of_range(v)) sc = Scale{top ? all : 0.f, top ? mean * up : 0.f, sc.eps * all * all, all};
}

template <typename T, int LPR, int W, int PT>
__global__ void __launch_bounds__((Place<T, LPR, W, PT>::THREADS)) k_layer_norm(NormParams p) {
  using At = Place<T, LPR, W, PT>;
  __shared__ float lds[2][W][4];
  At at;
  at.set();
  const int n = p.channels, wave = threadIdx.x >> 6;
  const float inv_n = 1.f / (float)n;
  int turn = 0;
  Piece<T> w[PT], b[PT], x[PT], next[PT];
#pragma unroll
  for (int i = 0; i < PT; ++i) {
    const int c = at.channel(i);
    w[i].load((const T*)p.w + (int64_t)blockIdx.y * n, c, p.w ? n : 0);
    if (!p.w) {
#pragma unroll
      for (int j = 0; j < PW<T>; j += 2) w[i].set(j, 1.f, 1.f);
    }
    b[i].load((const T*)p.b + (int64_t)blockIdx.y * n, c, p.b ? n : 0);
  }
  auto request = [&](int64_t i) {
    const T* row = row_at<T>(p.x, p, i < p.n ? i : 0);
#pragma unroll
    for (int k = 0; k < PT; ++k) next[k].load(row, at.channel(k), i < p.n ? n : 0);
  };
  auto again = [&](Piece<T> (&to)[PT], int64_t i) {
    asm volatile("" ::: "memory");      // (not the registers that hold it)
    const T* row = row_at<T>(p.x, p, i < p.n ? i : 0);
#pragma unroll
    for (int k = 0; k < PT; ++k) to[k].load(row, at.channel(k), i < p.n ? n : 0);
  };
  const int64_t step = (int64_t)gridDim.x * At::STEP;
  int64_t i = (int64_t)blockIdx.x * At::STEP;
  if (At::AHEAD) request(i + at.row);
  for (; i < p.n; i += step) {
    if (!At::AHEAD) request(i + at.row);
#pragma unroll
    for (int k = 0; k < PT; ++k) x[k] = next[k];
    if (At::AHEAD && i + step < p.n) request(i + step + at.row);
    float d[PT][PW<T>], dm, v;
    float s[1] = {sum_of<T, PT>(x)};
    row_sums<LPR, W>(s, lds, turn, wave);
    Scale sc = {1.f, s[0] * inv_n, p.eps, 1.f};
    auto spread = [&](float times, float mean, float eps) {
      centre<T, LPR, W, PT>(x, d, at, n, mean, times);
      float q[2] = {0.f, 0.f};
#pragma unroll
      for (int k = 0; k < PT; ++k)
#pragma unroll
        for (int j = 0; j < PW<T>; ++j) {
          q[0] += d[k][j];
          q[1] = __builtin_fmaf(d[k][j], d[k][j], q[1]);
        }
      row_sums<LPR, W>(q, lds, turn, wave);
      dm = q[0] * inv_n;
      v = __builtin_fmaxf(__builtin_fmaf(-dm, dm, q[1] * inv_n), 0.f) + eps;
      v = q[1] < INFINITY ? v : q[1];      // (the maximum drops a NaN, which a mean beyond fp32 leaves too)
    };
    spread(1.f, sc.mean, p.eps);
    if (__builtin_amdgcn_ballot_w64(out_of_range(v)) != 0) {      // (all waves of a row find the same)
      const bool in = i + at.row < p.n;
      own_scale<T, LPR, W, PT>(row_at<T>(p.x, p, in ? i + at.row : 0), at, in ? n : 0, n, v, lds, turn, wave, sc);
      again(x, i + at.row);      // (kept for this it would take registers)
      spread(sc.times, sc.mean, sc.eps);
    }
    const float r = out_of_range(v) ? 1.f / sqrtf(v) : inv_root(v), k0 = -dm * r;      // (out of range still: zero or NaN)
    if (i + at.row < p.n) {
      T* row = row_at<T>(p.y, p, i + at.row);
#pragma unroll
      for (int k = 0; k < PT; ++k) {
        Piece<T> o;
#pragma unroll
        for (int j = 0; j < PW<T>; j += 2)
          o.set(j, __builtin_fmaf(__builtin_fmaf(d[k][j], r, k0), w[k].get(j), b[k].get(j)),
                __builtin_fmaf(__builtin_fmaf(d[k][j + 1], r, k0), w[k].get(j + 1), b[k].get(j + 1)));
        o.store(row, at.channel(k), n);
      }
    }
  }
}

template <typename T, int LPR, int W, int PT>
__global__ void __launch_bounds__((Place<T, LPR, W, PT>::THREADS)) k_layer_norm_backward(NormParams p) {
  using At = Place<T, LPR, W, PT>;
  __shared__ float lds[2][W][4];
  At at;
  at.set();
  const int n = p.channels, wave = threadIdx.x >> 6;
  const float inv_n = 1.f / (float)n;
  int turn = 0;
  Piece<T> w[PT], x[PT], dy[PT], nx[PT], ny[PT];
  float dw[PT][PW<T>], db[PT][PW<T>];
#pragma unroll
  for (int i = 0; i < PT; ++i) {
    w[i].load((const T*)p.w + (int64_t)blockIdx.y * n, at.channel(i), p.w ? n : 0);
    if (!p.w) {
#pragma unroll
      for (int j = 0; j < PW<T>; j += 2) w[i].set(j, 1.f, 1.f);
    }
#pragma unroll
    for (int j = 0; j < PW<T>; ++j) dw[i][j] = db[i][j] = 0.f;
  }
  auto request = [&](int64_t i) {
    const T *rx = row_at<T>(p.x, p, i < p.n ? i : 0), *ry = row_at<T>(p.dy, p, i < p.n ? i : 0);
#pragma unroll
    for (int k = 0; k < PT; ++k) {
      nx[k].load(rx, at.channel(k), i < p.n ? n : 0);
      ny[k].load(ry, at.channel(k), i < p.n ? n : 0);
    }
  };
  auto again = [&](Piece<T> (&to)[PT], int64_t i) {
    asm volatile("" ::: "memory");      // (not the registers that hold it)
    const T* row = row_at<T>(p.x, p, i < p.n ? i : 0);
#pragma unroll
    for (int k = 0; k < PT; ++k) to[k].load(row, at.channel(k), i < p.n ? n : 0);
  };
  const int64_t step = (int64_t)gridDim.x * At::STEP;
  int64_t i = (int64_t)blockIdx.x * At::STEP;
  if (At::AHEAD && i < p.n) request(i + at.row);
  for (; i < p.n; i += step) {
    if (!At::AHEAD) request(i + at.row);
#pragma unroll
    for (int k = 0; k < PT; ++k) { x[k] = nx[k]; dy[k] = ny[k]; }
    if (At::AHEAD && i + step < p.n) request(i + step + at.row);
    float d[PT][PW<T>], q[4], v;     // q: sums of d, d^2, g, g d
    float s[1] = {sum_of<T, PT>(x)};
    row_sums<LPR, W>(s, lds, turn, wave);
    Scale sc = {1.f, s[0] * inv_n, p.eps, 1.f};
    auto spread = [&](float times, float mean, float eps) {
      centre<T, LPR, W, PT>(x, d, at, n, mean, times);
#pragma unroll
      for (int k = 0; k < 4; ++k) q[k] = 0.f;
#pragma unroll
      for (int k = 0; k < PT; ++k)
#pragma unroll
        for (int j = 0; j < PW<T>; ++j) {
          const float g = dy[k].get(j) * w[k].get(j);
          q[0] += d[k][j];
          q[1] = __builtin_fmaf(d[k][j], d[k][j], q[1]);
          q[2] += g;
          q[3] = __builtin_fmaf(g, d[k][j], q[3]);
        }
      row_sums<LPR, W>(q, lds, turn, wave);
      const float dm = q[0] * inv_n;
      v = __builtin_fmaxf(__builtin_fmaf(-dm, dm, q[1] * inv_n), 0.f) + eps;
      v = q[1] < INFINITY ? v : q[1];
    };
    spread(1.f, sc.mean, p.eps);
    const bool scaled = __builtin_amdgcn_ballot_w64(out_of_range(v)) != 0;
    if (scaled) {
      const bool in = i + at.row < p.n;
      own_scale<T, LPR, W, PT>(row_at<T>(p.x, p, in ? i + at.row : 0), at, in ? n : 0, n, v, lds, turn, wave, sc);
      again(x, i + at.row);
      spread(sc.times, sc.mean, sc.eps);
    }
    const float dm = q[0] * inv_n, r = out_of_range(v) ? 1.f / sqrtf(v) : inv_root(v), k0 = -dm * r;
    const float mg = q[2] * inv_n, mgh = r * __builtin_fmaf(-dm, q[2], q[3]) * inv_n;
    if (i + at.row < p.n) {
      T* row = row_at<T>(p.dx, p, i + at.row);
#pragma unroll
      for (int k = 0; k < PT; ++k) {
        Piece<T> o;
        float o_[PW<T>];
#pragma unroll
        for (int j = 0; j < PW<T>; ++j) {
          const float y = dy[k].get(j), g = y * w[k].get(j), h = __builtin_fmaf(d[k][j], r, k0);
          dw[k][j] = __builtin_fmaf(y, h, dw[k][j]);
          db[k][j] += y;
          o_[j] = r * (g - __builtin_fmaf(h, mgh, mg));
        }
        if (scaled) {      // (r is of the scaled row; its product with the scale may leave fp32)
#pragma unroll
          for (int j = 0; j < PW<T>; ++j) o_[j] *= sc.back;
        }
#pragma unroll
        for (int j = 0; j < PW<T>; j += 2) o.set(j, o_[j], o_[j + 1]);
        o.store(row, at.channel(k), n);
      }
    }
  }
  if (!p.dw && !p.db) return;
  // the rows' lanes that hold the same channels, in their order: lanes of a wave, then waves
  float* to[2] = {p.dw ? p.dw + (int64_t)blockIdx.y * n : nullptr, p.db ? p.db + (int64_t)blockIdx.y * n : nullptr};
  if (p.blocks > 1) {
    to[0] = p.part + ((int64_t)blockIdx.y * p.blocks + blockIdx.x) * 2 * n;
    to[1] = to[0] + n;
  }
  __shared__ float sums[W == 1 ? 4 : 1][W == 1 ? PT * PW<T> * LPR : 1];
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if constexpr (W == 1) {
      __syncthreads();
#pragma unroll
      for (int k = 0; k < PT; ++k)
#pragma unroll
        for (int j = 0; j < PW<T>; ++j) {
          float v = which ? db[k][j] : dw[k][j];
#pragma unroll
          for (int o = LPR; o < 64; o <<= 1) v += __shfl_xor(v, o);
          if ((threadIdx.x & 63) < LPR) sums[wave][(k * PW<T> + j) * LPR + at.lane] = v;
        }
      __syncthreads();
      if (to[which]) {
        for (int c = threadIdx.x; c < n; c += 256) {
          const int piece = c / PW<T>, slot = (piece / LPR * PW<T> + c % PW<T>) * LPR + piece % LPR;
          to[which][c] = (sums[0][slot] + sums[1][slot]) + (sums[2][slot] + sums[3][slot]);
        }
      }
    } else if (to[which]) {
#pragma unroll
      for (int k = 0; k < PT; ++k) {
        const int c = at.channel(k);
        if (c + PW<T> <= n) {
#pragma unroll
          for (int j = 0; j < PW<T>; j += 4)
            *(float4any*)(to[which] + c + j) = which ? float4v{db[k][j], db[k][j + 1], db[k][j + 2], db[k][j + 3]} : float4v{dw[k][j], dw[k][j + 1], dw[k][j + 2], dw[k][j + 3]};
        } else {
#pragma unroll
          for (int j = 0; j < PW<T>; ++j)
            if (c + j < n) to[which][c + j] = which ? db[k][j] : dw[k][j];
        }
      }
    }
  }
}

// dw[c], db[c] = sums over the workgroups' rows; a workgroup adds 32 columns of a group's 2 * channels, 32 threads a column.
__global__ void __launch_bounds__(1024) k_norm_weights(NormParams p) {
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), row = threadIdx.x >> 5;
  const float* part = p.part + (int64_t)blockIdx.y * p.blocks * 2 * p.channels;
  float s = 0.f;
  if (c < 2 * p.channels) {
#pragma unroll 8
    for (int i = row; i < p.blocks; i += 32) s += part[(int64_t)i * 2 * p.channels + c];
  }
  __shared__ float acc[32][33];
  acc[row][threadIdx.x & 31] = s;
  __syncthreads();
  if (row == 0 && c < 2 * p.channels) {
    float r = 0.f;
    for (int i = 0; i < 32; ++i) r += acc[i][threadIdx.x & 31];
    float* to = c < p.channels ? p.dw : p.db;
    if (to) to[(int64_t)blockIdx.y * p.channels + (c < p.channels ? c : c - p.channels)] = r;
  }
}

// Waves for each compute unit.  Backward: every workgroup leaves a row of partial sums, and above 512 channels the registers (up to 256) leave place for two or three waves a SIMD: more only
// wait for it (8 / 16 waves: 131,072 x 2048 bf16 325 / 368 us, 65,536 x 1024 80 / 94, 10,007 x 999 fp32, 173 registers, 29 / 37; up to 512 channels, whose registers are fewer: 60,000 x 173
// 43 / 33, 30,000 x 336 34 / 27, 100,000 x 250 fp32 78 / 58, 200,000 x 64 23 / 22, 500,000 x 128 fp32 137 / 149).  The masks of row ends, found once, take more scalars than there are: up to
// 77 forward and 102 backward lie in lanes of vector registers.
constexpr int FWD_WAVES = 16, FWD_MOST_WAVES = 256, BWD_WAVES = 8, BWD_WAVES_NARROW = 16;

}  // namespace

int norm_backward_blocks(int64_t n, int64_t groups, int channels, int dtype, int num_cu) {
  auto of = [&](auto l, auto w, auto) {
    using At = Place<float, l.value, w.value, 1>;
    int64_t b = blocks_of(n, groups, At::STEP, At::THREADS, channels <= 512 ? BWD_WAVES_NARROW : BWD_WAVES, num_cu);
    // four rows at least for each row of partial sums, unless that leaves compute units idle
    const int64_t four = (n + 4 * At::STEP - 1) / (4 * At::STEP), all = (num_cu + groups - 1) / groups;
    if (b > four && b > all) b = four > all ? four : all;
    return (int)(b < 1 ? 1 : b);
  };
  return dtype == FREQATTN_BF16 ? for_channels<Bf16, HALF_PACKED>(channels, of) : for_channels<float, HALF_PACKED>(channels, of);
}

template <typename T>
static hipError_t forward(const NormParams& p, int num_cu, hipStream_t st) {
  return for_channels<T, sizeof(T) == 2 ? PACKED : SPREAD>(p.channels, [&](auto l, auto w, auto pt) {
    using At = Place<T, l.value, w.value, pt.value>;
    // 16 waves for each compute unit, and more where every workgroup still has four steps: rows that are dealt out as workgroups end keep memory busier than fixed shares of a long
    // tensor (16 / 4 steps: 131,072 x 2048 bf16 210 / 182 us, 2 x 65,536 x 1536 151 / 142, 20,000 x 4096 60 / 57), while the first row of a workgroup is not requested ahead (one step
    // each: 65,536 x 1024 45 / 51).  Rows of eight waves stay with 16 (8192 x 8192 45 / 48).
    int64_t blocks = blocks_of(p.n, p.groups, At::STEP, At::THREADS, FWD_WAVES, num_cu);
    if (w.value < 8) blocks = std::max(blocks, std::min(p.n / (4 * At::STEP), blocks_of(p.n, p.groups, At::STEP, At::THREADS, FWD_MOST_WAVES, num_cu)));
    hipLaunchKernelGGL((k_layer_norm<T, l.value, w.value, pt.value>), dim3((unsigned)blocks, (unsigned)p.groups), dim3(At::THREADS), 0, st, p);
    return hipGetLastError();
  });
}
template <typename T>
static hipError_t backward(const NormParams& p, hipStream_t st) {
  return for_channels<T, HALF_PACKED>(p.channels, [&](auto l, auto w, auto pt) {
    using At = Place<T, l.value, w.value, pt.value>;
    hipLaunchKernelGGL((k_layer_norm_backward<T, l.value, w.value, pt.value>), dim3((unsigned)p.blocks, (unsigned)p.groups), dim3(At::THREADS), 0, st, p);
    return hipGetLastError();
  });
}

hipError_t launch_layer_norm(NormParams p, int dtype, int num_cu, hipStream_t st) {
  return dtype == FREQATTN_BF16 ? forward<Bf16>(p, num_cu, st) : forward<float>(p, num_cu, st);
}

hipError_t launch_layer_norm_backward(NormParams p, int dtype, int num_cu, hipStream_t st) {
  p.blocks = norm_backward_blocks(p.n, p.groups, p.channels, dtype, num_cu);
  const hipError_t e = dtype == FREQATTN_BF16 ? backward<Bf16>(p, st) : backward<float>(p, st);
  if (e != hipSuccess || p.blocks == 1 || (!p.dw && !p.db)) return e;
  hipLaunchKernelGGL(k_norm_weights, dim3((unsigned)((2 * p.channels + 31) / 32), (unsigned)p.groups), dim3(1024), 0, st, p);
  return hipGetLastError();
}

}  // namespace fa
