// Rows and tiles of attention over sequences, shared by its kernels.
//
// The G query heads of a key head are rows of one matrix: row r of a sequence and key head is token r / G, head r % G of the group, so
// that K and V are read once for the group and a single token still fills G rows.  A launch has `slots` tiles of ROWS rows per key head.
// Packed sequences: sequence i starts at slot floor(offset_i * mult / ROWS) + i, which leaves room for the tiles of all sequences
// before it (floor(a + b) + 1 >= floor(a) + ceil(b)) and is known to every workgroup without a sum over the lengths; a workgroup finds its
// sequence by bisection and ends at once where the slot is past the sequence's last tile.
#pragma once
#include <hip/hip_runtime.h>

#include "heads.h"

namespace fa {

// bf16, backward: delta = rowsum(dO O) of a row that sees up to SHORT_ROW keys is summed from the probabilities themselves, sum_j P_j (dO V^T)_j: the rounding of the
// stored out to bf16 is a share of delta, and dS is what is left of dO V^T - delta.  Over n keys of about equal probability out is smaller than v by sqrt(n), and
// its rounding with it; longer rows keep that error, whose share is larger where the values have a mean.  Relative error of dq, values of mean 0 / of mean 4:
// 64 sequences of 128 rows, 16 / 4 heads of 128, causal: 2.58e-3 / 9.9e-3 from out, 2.32e-3 / 2.35e-3 from the probabilities (about what rounding dS and dq
// leaves).  It takes both products of these keys once more: backward pass 120 -> 123 us; 256 sequences of 64 rows, 16 heads of 64, full: 129 -> 137; 512 of
// 128 rows, 16 heads of 128, full: 1024 -> 1118.
constexpr int SHORT_ROW = 128;

struct SeqRange {
  int seq;          // entry of the batch axis (0 for packed tensors)
  int base, n;      // first row and number of rows
};

__device__ __forceinline__ int seq_clamp(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

__device__ __forceinline__ SeqRange seq_range(const int32_t* off, const int32_t* len, int rows, int i) {
  SeqRange r;
  r.seq = i;
  r.base = 0;
  r.n = rows;
  if (off) {
    r.seq = 0;
    r.base = seq_clamp(off[i], 0, rows);
    r.n = seq_clamp(off[i + 1], r.base, rows) - r.base;
  }
  if (len) r.n = seq_clamp(len[i], 0, r.n);
  return r;
}

// Sequence and tile of a slot; rows are `mult` per token.  tile may lie past the sequence's last one.
__device__ __forceinline__ void seq_slot(const int32_t* off, int rows, int nseq, int mult, int tile_rows, int slot, int& seq, int& tile) {
  if (!off) {
    const int per = (int)(((int64_t)rows * mult + tile_rows - 1) / tile_rows);
    seq = slot / per;
    tile = slot - seq * per;
    return;
  }
  int lo = 0, hi = nseq - 1;   // the last sequence that starts at or before the slot
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    const int start = (int)((int64_t)seq_clamp(off[mid], 0, rows) * mult / tile_rows) + mid;
    if (start <= slot) lo = mid; else hi = mid - 1;
  }
  seq = lo;
  tile = slot - ((int)((int64_t)seq_clamp(off[lo], 0, rows) * mult / tile_rows) + lo);
  if (tile < 0) tile = 0x3fffffff / tile_rows;   // (offsets that do not ascend: past every sequence)
}

// Inclusive sum over the lanes of a wave.
__device__ __forceinline__ int lane_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // rows of 16: one, two, four, eight lanes up
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // last lane of a row to the next row, of the first half to the second
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}

// The rank-th tile of a launch in the order of descending work (the first key tiles of a sequence, or its last query tiles, under the causal mask), so that no long tile
// starts when the chip is about to run dry.  Up to 64 sequences, one a lane.  Work counts in steps of 64 rows of the other side; `count(c)` is the
// number of the lane's tiles of c steps or more, and the level of the rank is found by bisection.  Returns false past the last tile.
// (More sequences are launched in their own order; no loss was measured: 64 of 16 to 3000 rows, 46,308 in all, 16 / 4 heads of 128, causal: forward 404 us, backward
// 1245; the same and one more of one row 383 and 1267.)
template <typename F>
__device__ __forceinline__ bool seq_rank(int rank, int top, F&& count, int& seq, int& nth) {
  int lo = 0, hi = top + 1;    // level lo holds the rank, level hi does not
  int n_lo = count(0), n_hi = 0;
  if (__builtin_amdgcn_readlane(lane_scan(n_lo), 63) <= rank) return false;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1, n = count(mid);
    if (__builtin_amdgcn_readlane(lane_scan(n), 63) > rank) { lo = mid; n_lo = n; }
    else { hi = mid; n_hi = n; }
  }
  // tiles of exactly level lo, sequence by sequence, behind those above it
  const int left = rank - __builtin_amdgcn_readlane(lane_scan(n_hi), 63), upto = lane_scan(n_lo - n_hi);
  seq = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > left));
  nth = __builtin_amdgcn_readlane(n_hi, seq) + left - (seq ? __builtin_amdgcn_readlane(upto, seq - 1) : 0);   // of the sequence's tiles, by descending work
  return true;
}
__device__ __forceinline__ int lane_max(int x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x = max(x, __shfl_xor(x, o));
  return x;
}

// The workgroup's query tile (rows: tokens x heads of the group) for place `slot` of the launch's order.  False: none.
__device__ __forceinline__ bool seq_query_tile(const SeqParams& p, int tile_rows, int lane, int slot, int& seq, int& tile) {
  if (p.nseq == 1 || p.nseq > 64) {
    seq_slot(p.q_off, p.q_rows, p.nseq, p.group, tile_rows, p.slots - 1 - slot, seq, tile);
    return true;
  }
  SeqRange q = {0, 0, 0}, k = {0, 0, 0};
  if (lane < p.nseq) { q = seq_range(p.q_off, p.q_len, p.q_rows, lane); k = seq_range(p.k_off, p.k_len, p.k_rows, lane); }
  const int tiles = (int)(((int64_t)q.n * p.group + tile_rows - 1) / tile_rows), off = k.n - q.n;
  int nth;
  if (!seq_rank(slot, lane_max(tiles ? k.n : 0) >> 6, [&](int c) {
        if (c == 0 || tiles == 0) return tiles;
        if (k.n < 64 * c) return 0;
        if (!p.causal) return tiles;
        // the first tile whose last row sees 64 c keys
        const int64_t rows = (int64_t)(64 * c - off - 1) * p.group + 1;
        const int64_t first = rows <= 0 ? 0 : (rows + tile_rows - 1) / tile_rows - 1;
        return first >= tiles ? 1 : tiles - (int)first;
      }, seq, nth)) return false;
  tile = __builtin_amdgcn_readlane(tiles, seq) - 1 - nth;
  return true;
}

// The same for tiles of keys.
__device__ __forceinline__ bool seq_key_tile(const SeqParams& p, int tile_rows, int lane, int slot, int& seq, int& tile) {
  if (p.nseq == 1 || p.nseq > 64) {
    seq_slot(p.k_off, p.k_rows, p.nseq, 1, tile_rows, slot, seq, tile);
    return true;
  }
  SeqRange q = {0, 0, 0}, k = {0, 0, 0};
  if (lane < p.nseq) { q = seq_range(p.q_off, p.q_len, p.q_rows, lane); k = seq_range(p.k_off, p.k_len, p.k_rows, lane); }
  const int tiles = (k.n + tile_rows - 1) / tile_rows, off = k.n - q.n;
  return seq_rank(slot, lane_max(tiles ? q.n : 0) >> 6, [&](int c) {
    if (c == 0 || tiles == 0) return tiles;
    if (q.n < 64 * c) return 0;
    if (!p.causal) return tiles;
    const int room = q.n - 64 * c + off;     // the tile's first key is at most that
    return room < 0 ? 0 : min(tiles, room / tile_rows + 1);
  }, seq, tile);
}

// Tiles of a launch per key head (host).
inline int64_t seq_slots(bool packed, int64_t rows, int64_t nseq, int64_t mult, int64_t tile_rows) {
  return packed ? rows * mult / tile_rows + nseq : nseq * ((rows * mult + tile_rows - 1) / tile_rows);
}

}  // namespace fa
