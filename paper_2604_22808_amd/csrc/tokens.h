// Shared by the operators on token rows (layer norm, 8-bit codes of rows, their products, caches held in 8 bits): host entry points in tokens_api.cpp, kernels in
// layer_norm.hip, rows_i8.hip, product_i8.hip and cache8.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "freqattn.h"
#include "heads.h"

namespace fa {

// A tensor of rows: row n of `rows` of entry b at b * bs + n * rs elements, channels adjacent.
struct RowsPtr { char* p; int64_t bs, rs; };

struct NormParams {
  RowsPtr x, y, dy, dx;
  const void *w, *b;              // [channels] or [groups][channels]; nullptr: ones, zeros
  float *dw, *db;                 // [groups][channels] or nullptr
  float* part;                    // backward: [groups][blocks][2][channels]
  int64_t n;                      // rows of a group
  int32_t groups, rows, channels;
  int32_t blocks;                 // workgroups of a group
  float eps;
};
// Workgroups of a group in the backward pass; with one the sums need no workspace.
int norm_backward_blocks(int64_t n, int64_t groups, int channels, int dtype, int num_cu);
hipError_t launch_layer_norm(NormParams p, int dtype, int num_cu, hipStream_t st);
hipError_t launch_layer_norm_backward(NormParams p, int dtype, int num_cu, hipStream_t st);
enum { NORM_MOST_CHANNELS = 16384 };

struct CodeParams {
  RowsPtr x, codes;
  float* scales;                  // [batch * rows]
  int64_t n;                      // batch * rows
  int32_t rows, channels;
};
hipError_t launch_quantize_rows(const CodeParams& p, int dtype, int num_cu, hipStream_t st);

struct ProductParams {
  const char *a, *w;              // codes, rows of `channels`
  int64_t a_rs, w_rs, out_rs;     // strides in elements
  const float *a_scales, *w_scales;
  const void* bias;               // [outputs] of the output's type or nullptr
  char* out;
  int32_t rows, channels, outputs;
  int32_t vec;                    // rows of codes are aligned 16-byte pieces
};
hipError_t launch_product_i8(const ProductParams& p, int dtype, int num_cu, hipStream_t st);
enum { PRODUCT_MOST_CHANNELS = 131071 };   // 128 * 128 * 131071 < 2^31

// ---- caches held in 8 bits --------------------------------------------------------------------------------------------
// Codes are e4m3 (bias 7, NaN 0x7f and 0xff, no infinities); the rows of a block and head share a scale 2^(byte - 127).
struct Cache8Params {
  HeadsPtr k, v;                  // new rows, or where values go
  HeadsPtr ck, cv;                // codes
  uint8_t *ks, *vs;               // [sequences][blocks][heads]
  const int32_t *q_off, *q_len, *k_len;
  int32_t nseq, heads, d, q_rows, k_rows;
  int32_t shift, blocks;          // log2 of a block's rows; blocks of a cache
};
hipError_t launch_cache8_append(const Cache8Params& p, int dtype, hipStream_t st);
hipError_t launch_cache8_read(const Cache8Params& p, int dtype, hipStream_t st);

// Attention over such a cache: p.k and p.v are the codes.
struct Cache8Scales {
  const uint8_t *k, *v;
  int32_t shift, blocks;
  int32_t heads_of_row;           // heads of neighbouring channels that are read by one XCD (few rows)
};
SeqPlan cache8_plan(const SeqParams& p, int dtype, int num_cu);
hipError_t launch_cache8_attention(SeqParams p, const Cache8Scales& sc, const SeqPlan& s, int dtype, hipStream_t st);
// Few rows: waves of a workgroup; up to so many steps of all of them (128 keys each) are not cut, which saves the join: us of the device in one piece / cut, one token, 32 / 8 heads of 128: 500
// keys 8.8 / 9.4, 1000 keys 12.9 / 9.2, 2000 keys 20.9 / 9.5; 16 / 2 heads of 64: 777 keys 8.1 / 9.1, 1000 keys 8.9 / 8.2, 1500 keys 11.3 / 9.0; called one by one the second launch and its
// workspace take the host another 4.6 (capacity 1000, 16 / 2 heads of 64: 11.5 / 16.1).
enum { CACHE8_FEW_WAVES = 4, CACHE8_ONE_PIECE = 8 };
// Waves of a SIMD, by their registers: workgroups (of four waves) of a compute unit.
constexpr int cache8_few_waves(bool fp32, bool wide, int nq, bool half) {
  return nq == 1 ? (wide ? (fp32 ? 2 : 3) : fp32 ? 4 : 5) : wide ? (fp32 || half ? 1 : 2) : fp32 ? 2 : 3;
}
hipError_t launch_cache8_few(const SeqParams& p, const Cache8Scales& sc, const SeqPlan& s, int dtype, hipStream_t st);
hipError_t launch_cache8_generic(const SeqParams& p, const Cache8Scales& sc, int dtype, hipStream_t st);

}  // namespace fa
