// Shared by the context-free operators (rotary positions, norms of Q and K, attention over sequences): host entry points in
// heads_api.cpp, kernels in qk_norm.hip, seq_fwd.hip, seq_bwd.hip and seq_generic.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <string>

#include "freqattn.h"

namespace fa {

std::string& context_free_error();   // text of the calling thread's last failure without a context (api.cpp)

// ---- rotary positions and norms -------------------------------------------------------------------------------------
enum { ROT_MAX_PAIRS = 256 };
// Angles are kept in turns: pair i of a token at position p stands at p * turn[i] mod 2^64, a 64-bit fixed-point fraction of a turn.  The product
// is exact, so positions of any size lose nothing, and the top 32 bits are the angle to 2^-32 turns.
struct RotTable {
  uint64_t turn[ROT_MAX_PAIRS];
  uint8_t axis[ROT_MAX_PAIRS];
  int32_t axes, half;          // half: pairs that rotate (R / 2)
  int32_t interleaved;
  uint32_t grid[4];            // extents (1 where unused)
  float amplitude;
};

struct HeadsPtr { const char* p; int64_t bs, ts, hs; };   // strides in elements

struct QkParams {
  HeadsPtr in[2], dy[2], out[2];  // q, k (or one tensor); dy: gradient of the output (backward)
  const void* w[2];
  const int32_t* pos;             // nullptr: from the token index
  int64_t pos_bs;
  float* part;                    // backward: [blocks][2][d] partial weight gradients
  int32_t batch, tokens, heads[2], d;
  int32_t norm, inverse;
  float eps;
};

// A copy of x into the order of out (heads_api.cpp).
hipError_t copy_heads(int dtype, int batch, int tokens, int heads, int d, const freqattn_heads& x, const freqattn_heads& out, hipStream_t st);

hipError_t launch_qk(const QkParams& p, const RotTable& t, int dtype, int num_cu, hipStream_t st);
// most blocks of the backward launch; the workspace holds two rows of head_dim floats for each
enum { QK_BWD_BLOCKS = 1024 };
hipError_t launch_qk_backward(const QkParams& p, const RotTable& t, int dtype, float* const dw[2], int num_cu, hipStream_t st);

// ---- attention over sequences ---------------------------------------------------------------------------------------
struct SeqParams {
  HeadsPtr q, k, v, o, dout, dq, dk, dv;
  float* lse;
  float* delta;                  // backward: [q_heads][lse_rows] row sums of dout * out, or pairs (lse in units of log2, row sum)
  float* part;                   // split keys: partial results
  const int32_t *q_off, *k_off, *q_len, *k_len;
  int32_t nseq, hq, hk, group, d, q_rows, k_rows, causal;
  int64_t lse_rows, lse_k;       // columns of lse; the same count for the keys (rows of k and v over all sequences)
  float scale;
  int32_t slots;                 // tiles of the launch per key head (upper bound)
  int32_t nsplit, split_tiles;   // pieces of the keys, and key tiles of a piece
  int32_t vec;                   // all tensors and strides are 16-byte aligned and rows are whole 16-byte pieces
};

// How a forward call of the bf16 kernels is cut; depends on sizes alone.
struct SeqPlan {
  bool few;             // tiles of 32 query rows instead of 128
  int nsplit, split_tiles;
  int64_t workspace;    // bytes
  int64_t part_at;      // backward: where the partial sums start in it
};
SeqPlan seq_fwd_plan(const SeqParams& p, int num_cu);
hipError_t launch_seq_fwd(SeqParams p, const SeqPlan& s, hipStream_t st);
SeqPlan seq_bwd_plan(const SeqParams& p, int num_cu);
hipError_t launch_seq_bwd(SeqParams p, const SeqPlan& s, hipStream_t st);
hipError_t launch_seq_generic_fwd(const SeqParams& p, int dtype, hipStream_t st);
hipError_t launch_seq_generic_bwd(const SeqParams& p, int dtype, hipStream_t st);

}  // namespace fa
