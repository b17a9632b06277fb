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

// Tiles of a launch per key head (host).
inline int64_t seq_slots(bool packed, int64_t rows, int64_t nseq, int64_t mult, int64_t tile_rows) {
  return packed ? rows * mult / tile_rows + nseq : nseq * ((rows * mult + tile_rows - 1) / tile_rows);
}

}  // namespace fa
