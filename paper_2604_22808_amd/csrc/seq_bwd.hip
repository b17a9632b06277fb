// Attention over sequences, bf16, backward.
//
//   delta = rowsum(dO O) (rows of few keys: see SHORT_ROW),  P = exp(S - lse),  dS = P (dO V^T - delta),  dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
//
// Two kernels, 7 products of 2 d flops per pair instead of the 5 that one kernel would need: k_seq_dq owns query rows and sums over keys, k_seq_dkv owns
// keys and sums over query rows, each in registers and in a fixed order.  One kernel would have to add one of the two sums up through memory, by
// fp32 atomics whose order changes from run to run.
// Both keep their products transposed as the forward pass does (the owned row on the lane), so that P and dS, rounded to bf16 in the accumulator
// registers, are the second operand of the products that follow.  k_seq_dq reads K by rows (S) and by columns (dQ), V by rows (dO V^T); k_seq_dkv
// reads Q and dO both ways.  8 heads x 8192 x 128, full: k_seq_dq 390 us (1.06 PFLOP/s, matrix cores busy 58 % at 1.72 GHz: power), k_seq_dkv 550 (1.0);
// 16,384 rows x 8 heads of 64: 820 (1.0) and 1150 (0.95), where exponentials take as long as products.  k_seq_dq goes first and leaves (lse, delta) of every row, lse in units of log2, in the workspace.
#include <algorithm>

#include "seq_mfma.h"

namespace fa {

using namespace seq;

namespace {

__device__ const float no_row[2] = {INFINITY, 0.f};     // lse and delta of a row that does not exist: its probabilities are zero

// 4 bytes a lane, to LDS bytes dst + 4 lane
__device__ __forceinline__ void copy4_any(const void* addr, unsigned dst) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(addr), "s"(uniform((int)dst)) : "memory", "m0");
}

// The units of query rows that see keys from key0 on: tiles tile0 .. of each head of the group, `per_head` of them.
constexpr int UNIT = 32;
struct DkvUnits { int tile0, per_head, all; };
__device__ __forceinline__ DkvUnits dkv_units(const SeqParams& p, int nq, int nk, int key0) {
  int first = p.causal ? key0 - (nk - nq) : 0;     // the first token that sees key0
  if (first < 0) first = 0;
  DkvUnits u;
  u.tile0 = first / UNIT;
  u.per_head = nq > first ? (nq + UNIT - 1) / UNIT - u.tile0 : 0;
  u.all = u.per_head * p.group;
  return u;
}
// Units of a piece (an even number): the longest sequence's divided by the number of pieces, but not less than what leaves `split_tiles` pieces in all.
__device__ __forceinline__ int dkv_piece_units(const SeqParams& p, int lane) {
  int most = 0;
  float all = 0.f;
  for (int i = lane; i < p.nseq; i += 64) {
    const int nq = seq_range(p.q_off, p.q_len, p.q_rows, i).n, nk = seq_range(p.k_off, p.k_len, p.k_rows, i).n;
    most = max(most, nq);
    all += (float)nq * (p.causal ? fmaxf((float)nk - 0.5f * (float)nq, 0.5f * (float)nk) : (float)nk);
  }
  most = lane_max(most);
#pragma unroll
  for (int o = 32; o; o >>= 1) all += __shfl_xor(all, o);
  const int units = (most + UNIT - 1) / UNIT * p.group;
  const int least = (int)fminf(all * (float)p.hq / (64.f * (float)UNIT * (float)p.split_tiles), 1e9f);
  return max(max(2, least & ~1), ((units + p.nsplit - 1) / p.nsplit + 1) & ~1);
}

template <int D, int NW, int KT>
__global__ void __launch_bounds__(64 * NW, 2) k_seq_dq(SeqParams p) {
  constexpr int DT = D / 32, DK = D / 16, T2 = KT / 32, TILE = 32 * NW, PF = 4;
  __shared__ __attribute__((aligned(256))) uint16_t Ks[2][KT * D];
  __shared__ __attribute__((aligned(256))) uint16_t Vs[2][KT * D];
  const int lane = threadIdx.x & 63, nn = lane & 31, g = lane >> 5, wave = uniform(threadIdx.x >> 6);
  const int kvh = (int)(blockIdx.x % (unsigned)p.hk);
  int seq_i, tile_i;
  if (!seq_query_tile(p, TILE, lane, (int)(blockIdx.x / (unsigned)p.hk), seq_i, tile_i)) return;
  seq_i = uniform(seq_i);
  tile_i = uniform(tile_i);
  const SeqRange q = uniform(seq_range(p.q_off, p.q_len, p.q_rows, seq_i)), k = uniform(seq_range(p.k_off, p.k_len, p.k_rows, seq_i));
  const int rows = q.n * p.group, r_first = tile_i * TILE;
  if ((int64_t)tile_i * TILE >= rows) return;
  const Row row = query_row(p, kvh, r_first + wave * 32 + nn, q.n, k.n);
  const int rl = min(r_first + TILE, rows) - 1, w0 = r_first + wave * 32;
  const int wg_first = last_key(p.causal, r_first / p.group, q.n, k.n), wg_last = last_key(p.causal, rl / p.group, q.n, k.n);
  const bool wave_live = w0 < rows;
  const int wave_first = wave_live ? last_key(p.causal, w0 / p.group, q.n, k.n) : -1;
  const int wave_last = wave_live ? last_key(p.causal, min(w0 + 31, rows - 1) / p.group, q.n, k.n) : -1;
  const int my_last = row.live ? row.last : wave_last;
  const int tiles = (wg_last + KT) / KT, chunks = p.d >> 3;

  // the lane's share of its row of Q and dO, and delta
  bf16x8 Q[DK], G[DK];
  float delta = 0.f;
  auto at_row = [&](const HeadsPtr& v) { return (const uint16_t*)v.p + (int64_t)q.seq * v.bs + (int64_t)(q.base + row.token) * v.ts + (int64_t)row.head * v.hs; };
  {
    const uint16_t *qs = at_row(p.q), *gs = at_row(p.dout), *os = at_row(p.o);
#pragma unroll
    for (int s = 0; s < DK; ++s) {
      uint4v x = {0u, 0u, 0u, 0u}, y = x, z = x;
      if (row.live && 2 * s + g < chunks) {
        x = *(const uint4v*)(qs + s * 16 + g * 8);
        y = *(const uint4v*)(gs + s * 16 + g * 8);
        z = *(const uint4v*)(os + s * 16 + g * 8);
      }
      Q[s] = __builtin_bit_cast(bf16x8, x);
      G[s] = __builtin_bit_cast(bf16x8, y);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        delta = __builtin_fmaf(__uint_as_float(y[j] << 16), __uint_as_float(z[j] << 16), delta);
        delta = __builtin_fmaf(__uint_as_float(y[j] & 0xffff0000u), __uint_as_float(z[j] & 0xffff0000u), delta);
      }
    }
    delta += other_half(delta);
  }
  RowRead<D> rr;
  rr.template set<BOTH>(nn, g);
  ColRead<D, BOTH> cr;
  cr.set(lane);
  using Copy = TileCopy<D, NW, KT, BOTH>;
  Copy kc, vc;
  const int64_t k_bytes = p.k.ts * 2, v_bytes = p.v.ts * 2;
  kc.set(k_bytes, wave, lane);
  vc.set(v_bytes, wave, lane);
  const char* kb = p.k.p + 2 * ((int64_t)k.seq * p.k.bs + (int64_t)k.base * p.k.ts + (int64_t)kvh * p.k.hs);
  const char* vb = p.v.p + 2 * ((int64_t)k.seq * p.v.bs + (int64_t)k.base * p.v.ts + (int64_t)kvh * p.v.hs);
  const unsigned k_lds = lds_address(Ks[0]), v_lds = lds_address(Vs[0]);
  constexpr int NI = Copy::NI, TB = KT * D * 2;
  auto copy_tile = [&](int t, int buf) {
    auto kcur = kc.begin(kb + (int64_t)t * KT * k_bytes, k_bytes, wave);
    auto vcur = vc.begin(vb + (int64_t)t * KT * v_bytes, v_bytes, wave);
    if ((t + 1) * KT <= k.n && chunks == D / 8) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        kc.whole(kcur, k_bytes, k_lds + buf * TB, wave, i);
        vc.whole(vcur, v_bytes, v_lds + buf * TB, wave, i);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NI; ++i) kc.part(kcur, k_bytes, k_lds + buf * TB, wave, lane, i, k.n - t * KT, chunks);
#pragma unroll
      for (int i = 0; i < NI; ++i) vc.part(vcur, v_bytes, v_lds + buf * TB, wave, lane, i, k.n - t * KT, chunks);
    }
  };

  const int64_t col = (p.q_off ? (int64_t)q.base : (int64_t)seq_i * p.q_rows) + row.token, at = (int64_t)row.head * p.lse_rows + col;
  float lse2 = row.live ? p.lse[at] * LOG2E : 0.f;
  // A row that sees no key has no probabilities; one whose scores hold +inf, or are all -inf, has no finite ones.
  if (row.last < 0) { lse2 = INFINITY; delta = 0.f; }
  else if (!(fabsf(lse2) < INFINITY)) lse2 = __builtin_nanf("");
  const float c2 = p.scale * LOG2E;
  auto arrived = [&] {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
  };
  // scores and dO V^T of 32 keys
  auto both = [&](unsigned Kt, unsigned Vt, int t2, float16v& S, float16v& dP) {
    S = zero16();
    dP = zero16();
    products<2 * DK, PF>([&](int i) { return rr.get(i < DK ? Kt : Vt, t2, i % DK); },
                         [&](int i, const bf16x8& a) {
                           if (i < DK) S = mfma(a, Q[i], S);
                           else dP = mfma(a, G[i - DK], dP);
                         });
    in_turn<2 * DK, PF, 1>();
  };
  if (wg_first < SHORT_ROW && tiles > 0) {     // (its first row sees the fewest keys)
    static_assert(SHORT_ROW == 2 * KT, "");
    copy_tile(0, 0);
    if (tiles > 1) copy_tile(1, 1);
    arrived();
    float sum = 0.f;
#pragma nounroll
    for (int i = 0; i < min(tiles, 2) * T2; ++i) {
      const int buf = i / T2, t2 = i % T2;
      float16v S, dP;
      both(k_lds + buf * TB, v_lds + buf * TB, t2, S, dP);
      const int lim = row.last - i * 32 - 4 * g;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(S[r], c2, -lse2)) * dP[r];
        sum += 8 * (r >> 2) + (r & 3) <= lim ? x : 0.f;
      }
    }
    sum += other_half(sum);
    if (row.last < SHORT_ROW) delta = sum;
    __syncthreads();
  }
  if (row.live && g == 0) *(float2v*)(p.delta + 2 * at) = float2v{lse2, delta};

  float16v A[DT];
  auto run = [&](auto careful) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) A[dt] = zero16();
    if (tiles > 0) copy_tile(0, 0);
    arrived();
    for (int t = 0; t < tiles; ++t, arrived()) {
      const int buf = t & 1, key0 = t * KT;
      const unsigned Kt = k_lds + buf * TB, Vt = v_lds + buf * TB;
      if (t + 1 < tiles) copy_tile(t + 1, buf ^ 1);
      if (!careful.value && key0 > wave_last) continue;     // (set_aside needs every wave; all pairs of such a wave are masked below)
#pragma unroll
      for (int t2 = 0; t2 < T2; ++t2) {
        const int first = key0 + t2 * 32;
        float16v S, dP;
        both(Kt, Vt, t2, S, dP);
#pragma unroll
        for (int r = 0; r < 16; ++r) S[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[r], c2, -lse2)) * (dP[r] - delta);
        if (first + 31 > wave_first) {
          really_branch();
          const int lim = my_last - first - 4 * g;
#pragma unroll
          for (int r = 0; r < 16; ++r) S[r] = 8 * (r >> 2) + (r & 3) <= lim ? S[r] : 0.f;
        }
        bf16x8 dS[2];
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
          uint4v pk;
#pragma unroll
          for (int j = 0; j < 4; ++j) pk[j] = pack2(S[s2 * 8 + 2 * j], S[s2 * 8 + 2 * j + 1]);
          dS[s2] = __builtin_bit_cast(bf16x8, pk);
        }
        // (the scores need K as it is.  A key that is not finite has scores of +inf or NaN, and the row's sums are NaN anyway, or -inf: its dS is zero)
        if (careful.value && key0 + KT - 1 > wg_first)
          set_aside<D, BOTH>(A, Ks[buf] + t2 * 32 * D, g, ~0u, [&](int i) { return row.live && first + i <= row.last; });
        products<2 * DT, PF>([&](int i) { return cr.get(Kt, i % DT, 2 * t2 + i / DT); },
                             [&](int i, const bf16x8& a) { A[i % DT] = mfma(a, dS[i / DT], A[i % DT]); });
        in_turn<2 * DT, PF, 2>();
      }
    }
  };
  run(std::false_type{});
  if (p.causal && uniform(__syncthreads_or(row.live && any_odd(A)))) run(std::true_type{});
  uint16_t* dst = const_cast<uint16_t*>(at_row(p.dq));
  each_piece(A, p.scale, g, [&](int c, const float (&o)[8]) {
    if (row.live && c < p.d) *(uint4v*)(dst + c) = pack8(o);
  });
}

// 64 keys, over the query rows of the group's heads that see any of them, in units of 32 rows of one head.  Four waves: two for the keys (32
// each) times two for the units, which take every other one; at the end the two add their sums up through LDS.  Units come two at a time, double
// buffered; each wave copies one tensor of one unit.  (128 keys and one unit at a time: half as many, longer workgroups; 16,384 causal rows, 32 / 8 heads of
// 128: whole backward pass 10.3 ms instead of 7.9.)  Accumulators for dK and dV take half of the registers that two waves per SIMD leave a
// wave; at D = 128 V's operands stay in LDS but for the last step's (the two workgroups of a compute unit have 80 KB each).
// (D = 64 fits three waves per SIMD: 1482 -> 1359 us for 16,384 rows x 8 heads)
template <int D>
__global__ void __launch_bounds__(256, D == 64 ? 3 : 2) k_seq_dkv(SeqParams p) {
  constexpr int DT = D / 32, DK = D / 16, ROWS_U = UNIT, TILE = 64, TB = ROWS_U * D * 2, PF = 4;
  constexpr bool V_LDS = D == 128;
  constexpr int PV = V_LDS ? 2 : PF;      // (with two operands each, more do not fit)
  constexpr int VS = V_LDS ? DK - 1 : 0, VROW = 2 * (DK - 1) * 16;    // steps of V in LDS, bytes of a row there
  __shared__ __attribute__((aligned(256))) uint16_t Buf[2][2][2][TB / 2];   // [copy][unit][Q, dO]
  __shared__ __attribute__((aligned(256))) char Vs[V_LDS ? TILE * VROW : 16];
  __shared__ __attribute__((aligned(256))) float St[2][2][2 * ROWS_U];      // [copy][unit] (lse, delta) of its rows
  const int lane = threadIdx.x & 63, nn = lane & 31, g = lane >> 5, wave = uniform(threadIdx.x >> 6), kw = wave & 1, us = wave >> 1;
  // key heads fastest, then tiles, the longest first, then pieces (pieces that do not exist would leave the XCDs that they fall on idle if they were between tiles)
  unsigned id = blockIdx.x;
  const int kvh = (int)(id % (unsigned)p.hk);
  id /= (unsigned)p.hk;
  const int piece = (int)(id / (unsigned)p.slots);
  int seq_i, tile_i;
  if (!seq_key_tile(p, TILE, lane, (int)(id % (unsigned)p.slots), seq_i, tile_i)) return;
  seq_i = uniform(seq_i);
  tile_i = uniform(tile_i);
  const SeqRange q = uniform(seq_range(p.q_off, p.q_len, p.q_rows, seq_i)), k = uniform(seq_range(p.k_off, p.k_len, p.k_rows, seq_i));
  if (tile_i >= (k.n + TILE - 1) / TILE) return;
  const int key0 = tile_i * TILE, key = key0 + kw * 32 + nn, chunks = p.d >> 3;
  const bool live = key < k.n;
  const int wave_last = key0 + kw * 32 + 31;     // last key of the wave (dead ones too)
  const DkvUnits un = dkv_units(p, q.n, k.n, key0);
  const int cap = p.nsplit > 1 ? uniform(dkv_piece_units(p, lane)) : un.all, u0 = piece * cap, u1 = min(u0 + cap, un.all);
  const bool whole_sum = un.all <= cap;
  if (piece > 0 && u0 >= un.all) return;

  const uint16_t* ks = (const uint16_t*)p.k.p + (int64_t)k.seq * p.k.bs + (int64_t)(k.base + (live ? key : 0)) * p.k.ts + (int64_t)kvh * p.k.hs;
  const uint16_t* vs = (const uint16_t*)p.v.p + (int64_t)k.seq * p.v.bs + (int64_t)(k.base + (live ? key : 0)) * p.v.ts + (int64_t)kvh * p.v.hs;
  // chunk c of V's row r lies at chunk c + (r / 8) % 2 of 14: 16 rows in 16 places modulo 256 bytes
  const unsigned v_row = (unsigned)(uintptr_t)(const __attribute__((address_space(3))) char*)Vs + (kw * 32 + nn) * VROW;
  auto v_at = [&](int c) { const int at = c + ((nn >> 3) & 1); return v_row + (at == 2 * (DK - 1) ? 0 : at) * 16; };
  bf16x8 K[DK], V[DK - VS];
#pragma unroll
  for (int s = 0; s < DK; ++s) {
    uint4v x = {0u, 0u, 0u, 0u}, y = x;
    if (live && 2 * s + g < chunks) {
      x = *(const uint4v*)(ks + s * 16 + g * 8);
      y = *(const uint4v*)(vs + s * 16 + g * 8);
    }
    K[s] = __builtin_bit_cast(bf16x8, x);
    if (s < VS) *(__attribute__((address_space(3))) uint4v*)(uintptr_t)v_at(2 * s + g) = y;   // (both waves of the keys write the same)
    else V[s - VS] = __builtin_bit_cast(bf16x8, y);
  }
  const unsigned v_first = v_at(g), v_last = v_at(2 * (VS - 1) + g);   // (steps in between follow the first)

  RowRead<D> rr;
  rr.template set<BOTH>(nn, g);
  ColRead<D, BOTH> cr;
  cr.set(lane);
  // this wave copies Q (kw 0) or dO (kw 1) of its own unit
  using Copy = TileCopy<D, 1, ROWS_U, BOTH>;
  Copy cp;
  const HeadsPtr& src = kw ? p.dout : p.q;
  const int64_t src_bytes = src.ts * 2;
  cp.set(src_bytes, 0, lane);
  const char* src0 = src.p + 2 * ((int64_t)q.seq * src.bs + (int64_t)q.base * src.ts + (int64_t)kvh * p.group * src.hs);
  const unsigned buf_lds = lds_address(Buf[0][0][0]), st_lds = (unsigned)(uintptr_t)(const __attribute__((address_space(3))) float*)St[0][0];
  auto copy_unit = [&](auto careful, int head, int tile, int buf) {
    const int row0 = tile * ROWS_U;
    auto cur = cp.begin(src0 + 2 * ((int64_t)row0 * src.ts + (int64_t)head * src.hs), src_bytes, 0);
    const unsigned dst = buf_lds + ((buf * 2 + us) * 2 + kw) * TB;
    if (row0 + ROWS_U <= q.n && chunks == D / 8) {
#pragma unroll
      for (int i = 0; i < Copy::NI; ++i) cp.whole(cur, src_bytes, dst, 0, i);
    } else {
#pragma unroll
      for (int i = 0; i < Copy::NI; ++i) cp.part(cur, src_bytes, dst, 0, lane, i, q.n - row0, chunks);
    }
    if (kw == 0) {
      int i = lane;     // (two floats a row)
      if (careful.value) asm volatile("" : "+v"(i));     // (addresses made anew each time: the second pass has no registers to keep them)
      const int64_t at = (int64_t)(kvh * p.group + head) * p.lse_rows + (p.q_off ? (int64_t)q.base : (int64_t)seq_i * p.q_rows) + row0;
      copy4_any(row0 + (i >> 1) < q.n ? p.delta + 2 * at + i : no_row + (i & 1), st_lds + (buf * 2 + us) * 2 * ROWS_U * 4);
    }
  };

  const float c2 = p.scale * LOG2E;
  float16v dK[DT], dV[DT];
  auto run = [&](auto careful) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) { dK[dt] = zero16(); dV[dt] = zero16(); }
    // the wave's next unit to copy, as head and tile
    int u = u0 + us, head = un.per_head ? u / un.per_head : 0, tile = un.tile0 + u - head * un.per_head;
    auto advance = [&] {
      u += 2;
      tile += 2;
      while (tile >= un.tile0 + un.per_head) { tile -= un.per_head; ++head; }
    };
    auto next_units = [&] {
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      __syncthreads();
    };
    if (u < u1) copy_unit(careful, head, tile, 0);
    next_units();
    for (int t = u0; t < u1; t += 2, next_units()) {
      const int buf = ((t - u0) >> 1) & 1, row0 = tile * ROWS_U;
      bool idle = u >= u1;                                         // (the last unit may be the other waves' alone)
      const int shift = p.causal ? row0 + k.n - q.n : 1 << 29;     // the last key that row i of the unit sees is shift + i
      if (un.all > 0) advance();
      if (u < u1) copy_unit(careful, head, tile, buf ^ 1);
      idle = idle || shift + 31 < key0 + kw * 32;                  // (uniform) no row sees a key of the wave
      if (!careful.value && idle) continue;
      const unsigned Qt = buf_lds + (buf * 2 + us) * 2 * TB, Gt = Qt + TB;
      float16v S = zero16(), dP = zero16();
      products<DK, PF>([&](int i) { return rr.get(Qt, 0, i); }, [&](int i, const bf16x8& a) { S = mfma(a, K[i], S); });
      in_turn<DK, PF, 1>();
      struct Two { bf16x8 g, v; };
      products<DK, PV>([&](int i) {
                         Two x;
                         x.g = rr.get(Gt, 0, i);
                         if (i < VS) x.v = *(const __attribute__((address_space(3))) bf16x8*)(uintptr_t)(i == VS - 1 ? v_last : v_first + 32 * i);
                         else x.v = V[i - VS];
                         return x;
                       },
                       [&](int i, const Two& a) { dP = mfma(a.g, a.v, dP); });
      in_turn<DK, PV, V_LDS ? 2 : 1>();
      bf16x8 P[2], dS[2];
      // row 8 (r / 4) + 4 g + r % 4 of the unit sees the lane's key where that is lim or more, and exists where it is less than rows (zeros of rows that do not
      // exist times an infinity of the key would be NaN)
      const bool mask = shift < wave_last || row0 + ROWS_U > q.n;
      const int lim = key - shift - 4 * g, rows = q.n - row0 - 4 * g;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float* st = St[buf][us] + 2 * (8 * i + 4 * g);
        const float4v a = *(const float4v*)st, b = *(const float4v*)(st + 4);
        const float lse[4] = {a[0], a[2], b[0], b[2]}, del[4] = {a[1], a[3], b[1], b[3]};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = 4 * i + j;
          S[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[r], c2, -lse[j]));
          dP[r] = S[r] * (dP[r] - del[j]);
        }
      }
      if (mask) {
        really_branch();
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const bool seen = 8 * (r >> 2) + (r & 3) >= lim && 8 * (r >> 2) + (r & 3) < rows;
          S[r] = seen ? S[r] : 0.f;
          dP[r] = seen ? dP[r] : 0.f;
        }
      }
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        uint4v pp, ps;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          pp[j] = pack2(S[8 * s2 + 2 * j], S[8 * s2 + 2 * j + 1]);
          ps[j] = pack2(dP[8 * s2 + 2 * j], dP[8 * s2 + 2 * j + 1]);
        }
        P[s2] = __builtin_bit_cast(bf16x8, pp);
        dS[s2] = __builtin_bit_cast(bf16x8, ps);
      }
      if (careful.value) {     // (every wave is here, and the scores need Q and dO as they are)
        const uint32_t none = row_bits(g, [&](int r) { return !(P[r >> 3][r & 7] != (__bf16)0.f); });
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          if (t + w >= u1) continue;
          auto seen = [&](int i) { return w == us && live && row0 + i < q.n && key <= shift + i; };
          set_aside<D, BOTH>(dV, Buf[buf][w][1], g, none, seen);
          set_aside<D, BOTH>(dK, Buf[buf][w][0], g, ~0u, seen);      // (of a query that is not finite every dS is zero or NaN, as in dQ)
        }
        if (idle) continue;
      }
      products<4 * DT, PF>([&](int i) { return cr.get(i & 1 ? Qt : Gt, (i >> 1) % DT, (i >> 1) / DT); },
                           [&](int i, const bf16x8& a) {
                             const int dt = (i >> 1) % DT, s2 = (i >> 1) / DT;
                             if (i & 1) dK[dt] = mfma(a, dS[s2], dK[dt]);
                             else dV[dt] = mfma(a, P[s2], dV[dt]);
                           });
      in_turn<4 * DT, PF, 2>();
    }
  };
  run(std::false_type{});
  if (p.causal && uniform(__syncthreads_or(live && (any_odd(dK) || any_odd(dV))))) run(std::true_type{});
  // the waves of the first units take dK's sum, those of the second dV's (every wave is past its last read of the tiles: next_units)
  float* ex = (float*)Buf + wave * (DT * 16 * 64);
  const float* from = (const float*)Buf + (wave ^ 2) * (DT * 16 * 64);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) ex[(dt * 16 + r) * 64 + lane] = us ? dK[dt][r] : dV[dt][r];
  __syncthreads();
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float o = from[(dt * 16 + r) * 64 + lane];
      dK[dt][r] = us ? o + dV[dt][r] : dK[dt][r] + o;     // (units in their order in both sums)
    }
  const HeadsPtr& to = us ? p.dv : p.dk;
  uint16_t* dst = (uint16_t*)const_cast<char*>(to.p) + (int64_t)k.seq * to.bs + (int64_t)(k.base + (live ? key : 0)) * to.ts + (int64_t)kvh * to.hs;
  float* part = p.part + (((int64_t)piece * 2 + us) * p.hk * p.lse_k + (int64_t)kvh * p.lse_k + (p.k_off ? (int64_t)k.base : (int64_t)seq_i * p.k_rows) + key) * p.d;
  each_piece(dK, us ? 1.f : p.scale, g, [&](int c, const float (&o)[8]) {
    if (!live || c >= p.d) return;
    if (whole_sum) {
      *(uint4v*)(dst + c) = pack8(o);
    } else {
      *(float4v*)(part + c) = float4v{o[0], o[1], o[2], o[3]};
      *(float4v*)(part + c + 4) = float4v{o[4], o[5], o[6], o[7]};
    }
  });
}

// Adds the pieces of dK and dV up, in their order, where a tile of keys has several.  A wave takes a key, a lane two channels.
__global__ void __launch_bounds__(256) k_seq_dkv_join(SeqParams p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int kvh = (int)(blockIdx.x % (unsigned)p.hk);
  int seq_i, tile_i;
  seq_slot(p.k_off, p.k_rows, p.nseq, 1, 4, (int)(blockIdx.x / (unsigned)p.hk), seq_i, tile_i);
  const SeqRange q = seq_range(p.q_off, p.q_len, p.q_rows, seq_i), k = seq_range(p.k_off, p.k_len, p.k_rows, seq_i);
  if ((int64_t)tile_i * 4 + wave >= k.n) return;
  const int key = tile_i * 4 + wave, cap = dkv_piece_units(p, lane), all = dkv_units(p, q.n, k.n, key / 64 * 64).all;
  const int c = 2 * lane;
  if (all <= cap || c >= p.d) return;
  const int64_t rows = (int64_t)p.hk * p.lse_k, at = (int64_t)kvh * p.lse_k + (p.k_off ? (int64_t)k.base : (int64_t)seq_i * p.k_rows) + key;
  for (int w = 0; w < 2; ++w) {
    float a = 0.f, b = 0.f;
    for (int s = 0; s * cap < all; ++s) {
      const float2v x = *(const float2v*)(p.part + (((int64_t)s * 2 + w) * rows + at) * p.d + c);
      a += x[0];
      b += x[1];
    }
    const HeadsPtr& to = w ? p.dv : p.dk;
    uint16_t* dst = (uint16_t*)const_cast<char*>(to.p) + (int64_t)k.seq * to.bs + (int64_t)(k.base + key) * to.ts + (int64_t)kvh * to.hs;
    *(uint32_t*)(dst + c) = pack2(a, b);
  }
}

template <int D>
hipError_t go(SeqParams p, hipStream_t st) {
  p.slots = (int)seq_slots(p.q_off != nullptr, p.q_rows, p.nseq, p.group, 128);
  if (p.slots > 0) hipLaunchKernelGGL((k_seq_dq<D, 4, 64>), dim3((unsigned)p.slots * (unsigned)p.hk), dim3(256), 0, st, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  p.slots = (int)seq_slots(p.k_off != nullptr, p.k_rows, p.nseq, 1, 64);
  if (p.slots == 0) return hipSuccess;
  hipLaunchKernelGGL((k_seq_dkv<D>), dim3((unsigned)p.slots * (unsigned)p.nsplit * (unsigned)p.hk), dim3(256), 0, st, p);
  e = hipGetLastError();
  if (e != hipSuccess || p.nsplit == 1) return e;
  const int64_t slots = seq_slots(p.k_off != nullptr, p.k_rows, p.nseq, 1, 4);
  hipLaunchKernelGGL(k_seq_dkv_join, dim3((unsigned)(slots * p.hk)), dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace

// How a backward call is cut: pieces of the query rows that a tile of keys is summed over, where there are few tiles.
SeqPlan seq_bwd_plan(const SeqParams& p, int num_cu) {
  SeqPlan s = {};
  const int64_t blocks = seq_slots(p.k_off != nullptr, p.k_rows, p.nseq, 1, 64) * p.hk;
  const int64_t units = ((int64_t)p.q_rows + 31) / 32 * p.group;      // the most that a tile of keys can have
  s.nsplit = 1;
  // Pieces so that there are four workgroups for each compute unit, eight pieces at most.  us of the backward pass with 2 / 4 / 8 pieces (more pieces: shorter chains,
  // more partial sums): 640 tiles (16 heads x 2500 rows) 176 / 189 / 236, 290 tiles (32 / 4 heads, 4500 rows) 465 / 389 / 381, 64 tiles (8 / 1 heads of 64,
  // 4096 rows) 343 / 218 / 159.
  if (p.k_rows > 0 && units >= 32 && blocks < 4 * num_cu) s.nsplit = (int)std::min<int64_t>(8, (4 * num_cu + blocks - 1) / blocks);
  s.split_tiles = 8 * num_cu;
  const int64_t stats = ((int64_t)p.hq * p.lse_rows * 8 + 255) / 256 * 256;
  s.part_at = stats;
  s.workspace = stats + (s.nsplit > 1 ? (int64_t)s.nsplit * 2 * p.hk * p.lse_k * p.d * 4 : 0);
  return s;
}

hipError_t launch_seq_bwd(SeqParams p, const SeqPlan& s, hipStream_t st) {
  p.nsplit = s.nsplit;
  p.split_tiles = s.split_tiles;
  return p.d <= 64 ? go<64>(p, st) : go<128>(p, st);
}

}  // namespace fa
