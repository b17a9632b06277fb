// The join of pieces of the keys, shared by the kernels of attention that cut them.
#pragma once
#include "seq_mfma.h"

namespace fa {

namespace {

using namespace seq;

// How the keys of a call are cut.  resident = 0: pieces of SeqParams::split_tiles tiles.  Else, for up to 64 sequences, the length of a piece is found on the device from the
// sequences' own lengths, by every wave alike: `resident` is how many workgroups run at the same time.
//   one_round (few query rows): so short, split_tiles at least, that there are no more pieces than that and all run at once; where such pieces are long, their lengths are uneven and
//   shorter ones of up to SEQ_ROUNDS rounds end closer together (one token of 32 requests, 32 / 8 heads of 128, caches of 200 to 16,384 rows: 159 us in one round, 117 in up to four or
//   six, fp32 174 / 124 / 126; pieces of four tiles at least 115, 16 at least 129).
//   else (tiles of many rows): a third of the work that a resident workgroup has on average, in up to four pieces, where that ends sooner than tiles that are not cut.  (Chunks of 1, 512,
//   1500 and 2048 rows, 16 / 4 heads of 128: 392 us uncut, 325 so; up to eight pieces of a third 353, of half 338, of a quarter 345.)
enum { SEQ_ROUNDS = 4, SEQ_LONG_PIECE = 4 };
struct SeqCut { int resident, one_round, kt, tile_rows; };

// Key tiles of a piece.  qt, kt: the lane's sequence's tiles of queries and of keys (zero from the last sequence on).
__device__ __forceinline__ int seq_lane_sum(int x) { return __builtin_amdgcn_readlane(lane_scan(x), 63); }
__device__ __forceinline__ int seq_pieces(int kt, int piece) { return kt <= piece ? 1 : (int)(((unsigned)kt + (unsigned)piece - 1) / (unsigned)piece); }
__device__ __forceinline__ int seq_piece(const SeqParams& p, const SeqCut& cut, int qt, int kt) {
  const int most = max(lane_max(qt ? kt : 0), 1);
  if (most <= p.split_tiles) return p.split_tiles;
  const int tiles = seq_lane_sum(qt);
  float work = (float)qt * (float)kt;
#pragma unroll
  for (int o = 32; o; o >>= 1) work += __shfl_xor(work, o);
  if (cut.one_round) {     // sum of qt ceil(kt / piece) <= work / piece + tiles
    auto rounds = [&](int n) {
      const int room = n * (cut.resident / p.hk) - tiles;
      return room > 0 ? (int)(work / (float)room) + 1 : most;
    };
    int piece = rounds(1);
    if (piece > SEQ_LONG_PIECE) piece = max(SEQ_LONG_PIECE, rounds(SEQ_ROUNDS));
    return min(max(piece, p.split_tiles), most);
  }
  const float slots = (float)cut.resident / (float)p.hk, mean = work / slots;
  const int piece = max(p.split_tiles, (int)(mean * (1.f / 3.f)));
  return mean + (float)piece < 0.9f * ceilf((float)tiles / slots) * (float)most ? piece : most;
}
// For the join, behind the partial results: the piece in tiles, or 0 where it is longer than every sequence, so that nothing is to be joined.
__device__ __forceinline__ int* seq_piece_at(const SeqParams& p) { return (int*)(p.part + (int64_t)p.nsplit * p.hq * p.lse_rows * (p.d + 1)); }
__device__ __forceinline__ void seq_tell(const SeqParams& p, int piece, int kt) {
  const int most = lane_max(kt);
  if (blockIdx.x == 0 && threadIdx.x == 0) *seq_piece_at(p) = most <= piece ? 0 : piece;
}
// The lane's sequence, for seq_piece.
__device__ __forceinline__ void seq_tiles(const SeqParams& p, const SeqCut& cut, int lane, int& qt, int& kt) {
  qt = kt = 0;
  if (lane < p.nseq) {
    const SeqRange q = seq_range(p.q_off, p.q_len, p.q_rows, lane), k = seq_range(p.k_off, p.k_len, p.k_rows, lane);
    qt = (int)(((int64_t)q.n * p.group + cut.tile_rows - 1) / cut.tile_rows);
    kt = (k.n + cut.kt - 1) / cut.kt;
  }
}

// Joins the pieces of a row: out = sum_s 2^(lse_s - top) out_s / sum_s 2^(lse_s - top).  A wave takes RPW rows one after the other, a lane two channels; the weights are found one
// piece a lane and handed round through LDS, so that the loads of the pieces do not wait for each other.
template <typename T, int RPW>
__global__ void __launch_bounds__(256) k_seq_join(SeqParams p, SeqCut cut) {
  __shared__ float weights[4][MAX_PIECES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int piece = cut.resident ? *seq_piece_at(p) : p.split_tiles;
  if (piece == 0) return;
  const int kvh = (int)(blockIdx.x % (unsigned)p.hk);
  int seq_i, tile_i;
  seq_slot(p.q_off, p.q_rows, p.nseq, p.group, 4 * RPW, (int)(blockIdx.x / (unsigned)p.hk), seq_i, tile_i);
  const SeqRange q = seq_range(p.q_off, p.q_len, p.q_rows, seq_i), k = seq_range(p.k_off, p.k_len, p.k_rows, seq_i);
  const int first = (tile_i * 4 + wave) * RPW;
  if ((int64_t)tile_i * 4 * RPW + wave * RPW >= (int64_t)q.n * p.group) return;      // (the whole wave; nothing here waits for another wave)
  if (cut.resident && (k.n + cut.kt - 1) / cut.kt <= piece) return;      // (not cut: stored where it was computed)
  const int piece_keys = piece * cut.kt;
  const int64_t all = (int64_t)p.hq * p.lse_rows;
  const float* lse = p.part + p.nsplit * all * p.d;
  for (int r = first; r < min(first + RPW, q.n * p.group); ++r) {
    const Row row = query_row(p, kvh, r, q.n, k.n);
    const int64_t col = (p.q_off ? (int64_t)q.base : (int64_t)seq_i * p.q_rows) + row.token, at = (int64_t)row.head * p.lse_rows + col;
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
    if (RPW > 1) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // (the weights are read before the next row's take their place)
  }
}

// T: float, or uint16_t for bf16.
template <typename T>
hipError_t join_pieces(const SeqParams& p, const SeqCut& cut, hipStream_t st) {
  // (many rows: four a wave; 1 / 4 / 8 of them, chunks of prompts with the pieces 332 / 325 / 325 us, 1000, 300 and 1700 rows of 12 / 4 heads without a mask 135 / 133 / 139)
  const int rpw = cut.resident && !cut.one_round ? 4 : 1;
  const dim3 grid((unsigned)(seq_slots(p.q_off != nullptr, p.q_rows, p.nseq, p.group, 4 * rpw) * p.hk));
  if (rpw == 4) hipLaunchKernelGGL((k_seq_join<T, 4>), grid, dim3(256), 0, st, p, cut);
  else hipLaunchKernelGGL((k_seq_join<T, 1>), grid, dim3(256), 0, st, p, cut);
  return hipGetLastError();
}

}  // namespace

}  // namespace fa
