// The join of pieces of the keys, shared by the kernels of attention that cut them.
#pragma once
#include "seq_mfma.h"

namespace fa {

namespace {

using namespace seq;

// Joins the pieces of a row: out = sum_s 2^(lse_s - top) out_s / sum_s 2^(lse_s - top).  A wave takes one row, a lane two channels; the weights are found one
// piece a lane and handed round through LDS, so that the loads of the pieces do not wait for each other.
template <typename T>
__global__ void __launch_bounds__(256) k_seq_join(SeqParams p, int piece_keys) {
  __shared__ float weights[4][MAX_PIECES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int kvh = (int)(blockIdx.x % (unsigned)p.hk);
  int seq_i, tile_i;
  seq_slot(p.q_off, p.q_rows, p.nseq, p.group, 4, (int)(blockIdx.x / (unsigned)p.hk), seq_i, tile_i);
  const SeqRange q = seq_range(p.q_off, p.q_len, p.q_rows, seq_i), k = seq_range(p.k_off, p.k_len, p.k_rows, seq_i);
  if ((int64_t)tile_i * 4 + wave >= (int64_t)q.n * p.group) return;      // (the whole wave; nothing here waits for another wave)
  const Row row = query_row(p, kvh, tile_i * 4 + wave, q.n, k.n);
  const int64_t col = (p.q_off ? (int64_t)q.base : (int64_t)seq_i * p.q_rows) + row.token, at = (int64_t)row.head * p.lse_rows + col;
  const int64_t all = (int64_t)p.hq * p.lse_rows;
  const float* lse = p.part + p.nsplit * all * p.d;
  const int n = row.last < 0 ? 0 : row.last / piece_keys + 1;    // pieces that hold keys of this row
  float w[MAX_PIECES / 64], top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int i = 0; i < MAX_PIECES / 64; ++i) {
    w[i] = i * 64 + lane < n ? lse[(i * 64 + lane) * all + at] : -INFINITY;
    top = fmaxf(top, w[i]);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int i = 0; i < MAX_PIECES / 64; ++i) {
    const float x = __builtin_amdgcn_exp2f(w[i] - ref);
    sum += x;
    weights[wave][i * 64 + lane] = x;
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // (a wave reads its own weights)
  const float inv = sum > 0.f || sum != sum ? 1.f / sum : row.last >= 0 ? __builtin_nanf("") : 0.f;
  const int c = 2 * lane;
  if (c < p.d) {
    const float* src = p.part + at * p.d + c;
    float a = 0.f, b = 0.f;
#pragma unroll 8
    for (int s = 0; s < n; ++s) {
      const float2v x = *(const float2v*)(src + s * all * p.d);
      const float y = weights[wave][s];
      a += y * x[0];     // (an infinity or NaN stays in the sum, whatever its weight)
      b += y * x[1];
    }
    T* dst = (T*)const_cast<char*>(p.o.p) + (int64_t)q.seq * p.o.bs + (int64_t)(q.base + row.token) * p.o.ts + (int64_t)row.head * p.o.hs;
    if constexpr (sizeof(T) == 4) *(float2v*)(dst + c) = float2v{a * inv, b * inv};
    else *(uint32_t*)(dst + c) = pack2(a * inv, b * inv);
  }
  if (lane == 0 && p.lse) p.lse[at] = sum > 0.f || sum != sum ? (ref + __builtin_amdgcn_logf(sum)) * LN2 : -INFINITY;
}

// piece_keys: keys of a piece.  T: float, or uint16_t for bf16.
template <typename T>
hipError_t join_pieces(const SeqParams& p, int piece_keys, hipStream_t st) {
  const int64_t slots = seq_slots(p.q_off != nullptr, p.q_rows, p.nseq, p.group, 4);
  hipLaunchKernelGGL(k_seq_join<T>, dim3((unsigned)(slots * p.hk)), dim3(256), 0, st, p, piece_keys);
  return hipGetLastError();
}

}  // namespace

}  // namespace fa
