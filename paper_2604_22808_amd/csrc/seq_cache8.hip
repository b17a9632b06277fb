// Attention over caches held in 8 bits: one pass over the keys with a running maximum and sum, as the bf16 kernel of sequences makes it, on values that are
// widened to bf16 on their way into LDS.
//
//   S = scale Q K^T,  O = softmax(S) V,   K, V: e4m3 codes times a power of two for each block of rows and head: exact in bf16
//
// A code and its block's scale become a bf16 value in one instruction for two of them, so that the tiles in LDS and everything behind them are those of
// bf16 keys and values, and memory gives half as many bytes.  Codes are loaded into registers a tile ahead, widened, and written to LDS in the order that the operand
// reads want; all rows of a wave's load lie in one block, so that a load has one scale.
//
// fp32 queries: K and V have no more than 4 significant bits, so products need fp32 only on the other side.  A query and a probability are three bf16
// numbers of 8 bits each, exactly, and their products run on the bf16 matrix instructions one after the other: 3 of those instead of fp32 products at a sixteenth of
// their rate.
//
// bf16 queries: a probability is rounded to bf16 as an operand, as the kernel of bf16 keys rounds it: the results' relative error is 2.2-2.3e-3 then, of which their own rounding to bf16 makes
// 1.7e-3; a second term would take the products with V once more.  The sum of the probabilities is of the unrounded ones.
//
// Bound by the vector unit beside the matrix cores (widening, exponentials).  4096 rows against 16,384 keys, 16 / 4 heads of 128, causal: 525 us (0.91 PFLOP/s; bf16 keys 461, fp32 queries 1343); 4 x
// 2048 rows against 8192, heads of 64: 320 (0.75).  In chunks of 1, 512, 1500 and 2048 rows against 777 to 16,000 keys (326 us with the join) compute units were busy 87 % of the time and matrix cores
// 33 %: the last pieces run on a chip that is no longer full, and the join of 24 us reads 119 MB.
#include "cache8_tile.h"
#include "seq_join.h"

namespace fa {

using namespace seq;

namespace {

// The order of N operands' products, TERMS each: PF operands up front, then one operand (READS reads) behind the products of one.
template <int N, int PF, int TERMS, int READS>
__device__ __forceinline__ void in_order() {
  __builtin_amdgcn_sched_group_barrier(0x100, PF * READS, 0);
#pragma unroll
  for (int i = 0; i < N - PF; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, TERMS, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, PF * TERMS, 0);
}

// T: type of queries and results, uint16_t for bf16.  D: channels (64, 128).
template <typename T, int D, bool HALF>
__global__ void __launch_bounds__(256, sizeof(T) == 4 ? (D == 64 ? 2 : 1) : 2) k_cache8_attention(SeqParams p, Cache8Scales sc, SeqCut cut) {
  constexpr int NW = 4, KT = SEQ_MANY_KT, DT = D / 32, DK = D / 16, T2 = KT / 32, TILE = 32 * NW, TERMS = sizeof(T) == 4 ? 3 : 1;
  __shared__ __attribute__((aligned(256))) uint16_t Ks[2][KT * D];
  __shared__ __attribute__((aligned(256))) uint16_t Vs[2][KT * D];
  const int tid = threadIdx.x, lane = tid & 63, nn = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // key heads fastest, then tiles, the longest first, then pieces of the keys
  unsigned id = blockIdx.x;
  const int kvh = (int)(id % (unsigned)p.hk);
  id /= (unsigned)p.hk;
  const int split = (int)(id / (unsigned)p.slots);
  int seq_i, tile_i, piece = p.split_tiles;
  if (cut.resident) {
    int qt, kt;
    seq_tiles(p, cut, lane, qt, kt);
    piece = uniform(seq_piece(p, cut, qt, kt));
    seq_tell(p, piece, kt);
    if (split * piece >= max(lane_max(kt), 1)) return;     // (no sequence has that piece)
  }
  if (!seq_query_tile(p, TILE, lane, (int)(id % (unsigned)p.slots), seq_i, tile_i)) return;
  seq_i = uniform(seq_i);
  tile_i = uniform(tile_i);
  const SeqRange q = uniform(seq_range(p.q_off, p.q_len, p.q_rows, seq_i)), k = uniform(seq_range(nullptr, p.k_len, p.k_rows, seq_i));
  const int rows = q.n * p.group, r_first = tile_i * TILE;
  if ((int64_t)tile_i * TILE >= rows) return;
  const Row row = query_row(p, kvh, r_first + wave * 32 + nn, q.n, k.n);
  // the last keys seen by the first and the last row of the workgroup and of the wave
  const int rl = min(r_first + TILE, rows) - 1;
  const int wg_first = last_key(p.causal, r_first / p.group, q.n, k.n), wg_last = last_key(p.causal, rl / p.group, q.n, k.n);
  const int w0 = r_first + wave * 32;
  const bool wave_live = w0 < rows;
  const int wave_first = wave_live ? last_key(p.causal, w0 / p.group, q.n, k.n) : -1;
  const int wave_last = wave_live ? last_key(p.causal, min(w0 + 31, rows - 1) / p.group, q.n, k.n) : -1;
  const int my_last = row.live ? row.last : wave_last;         // dead rows of a live wave act as its last one; nothing of them is stored

  const int t_all = (wg_last + KT) / KT;                       // tiles the workgroup's rows see (0: none)
  const bool cuts = p.nsplit > 1 && (!cut.resident || (k.n + KT - 1) / KT > piece);     // (a sequence in one piece needs no join)
  if (!cuts && split > 0) return;
  const int t0 = cuts ? split * piece : 0, t1 = cuts ? min(t0 + piece, t_all) : t_all;
  if (cuts && t0 >= t_all && split > 0) return;                // (piece 0 of a row that sees nothing stores that)

  bf16x8 Q[TERMS][DK];
  {
    const T* src = (const T*)p.q.p + (int64_t)q.seq * p.q.bs + (int64_t)(q.base + row.token) * p.q.ts + (int64_t)row.head * p.q.hs;
#pragma unroll
    for (int s = 0; s < DK; ++s) {
      const int c = s * 16 + g * 8;
      const bool in = row.live && c < p.d;
      if constexpr (TERMS == 1) {
        uint4v x = {0u, 0u, 0u, 0u};
        if (in) x = *(const uint4v*)(src + c);
        Q[0][s] = __builtin_bit_cast(bf16x8, x);
      } else {
        float x[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float4v y = {0.f, 0.f, 0.f, 0.f};
          if (in) y = *(const float4v*)(src + c + 4 * h);
#pragma unroll
          for (int j = 0; j < 4; ++j) x[4 * h + j] = y[j];
        }
        bf16x8 t[3];
        three_terms(x, t);
#pragma unroll
        for (int term = 0; term < TERMS; ++term) Q[term][s] = t[term];
      }
    }
  }
  const float c2 = p.scale * LOG2E;

  RowRead<D> kr;
  kr.template set<ROWS>(nn, g);
  ColRead<D, COLS> vr;
  vr.set(lane);
  const char* kb = p.k.p + (int64_t)k.seq * p.k.bs + (int64_t)kvh * p.k.hs;
  const char* vb = p.v.p + (int64_t)k.seq * p.v.bs + (int64_t)kvh * p.v.hs;
  const uint8_t *ks = sc.k + (int64_t)k.seq * sc.blocks * p.hk + kvh, *vs = sc.v + (int64_t)k.seq * sc.blocks * p.hk + kvh;
  const unsigned k_lds = lds_address(Ks[0]), v_lds = lds_address(Vs[0]);
  constexpr int TB = KT * D * 2;
  CodeTile<D, NW, KT, ROWS, HALF> kt;
  CodeTile<D, NW, KT, COLS, HALF> vt;
  kt.set(p.k.ts, tid);
  vt.set(p.v.ts, tid);
  auto load = [&](int t) {
    kt.load(kb, p.k.ts, ks, p.hk, sc.shift, t * KT, k.n, p.d, wave, tid);
    vt.load(vb, p.v.ts, vs, p.hk, sc.shift, t * KT, k.n, p.d, wave, tid);
  };
  auto store = [&](int buf) {
    kt.store(Ks[buf], tid);
    vt.store(Vs[buf], tid);
  };
  auto settle = [&] {      // everybody's LDS writes and reads are done
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  };

  float16v O[DT];
  float m, l;
  // careful: the second pass of a workgroup whose result was not finite, with values set aside (set_aside) and the maximum as the reference
  auto run = [&](auto careful) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) O[dt] = zero16();
    m = -INFINITY;
    l = 0.f;
    // (the second pass has other things in its registers than the tile after the next)
    if (t0 < t1) {
      load(t0);
      store(0);
      if (!careful.value && t0 + 1 < t1) load(t0 + 1);
      settle();
    }
    for (int t = t0; t < t1; ++t) {
      const int buf = (t - t0) & 1, key0 = t * KT;
      const unsigned Kt = k_lds + buf * TB, Vt = v_lds + buf * TB;
      if (t + 1 < t1) {
        if (careful.value) load(t + 1);
        store(buf ^ 1);
        if (!careful.value && t + 2 < t1) load(t + 2);
      }
      if (!careful.value && key0 > wave_last) {   // (uniform over the wave) none of its rows sees the tile (set_aside needs every wave: all masked below)
        settle();
        continue;
      }
      const bool mask = key0 + KT - 1 > wave_first;
      // ---- S^T = K Q^T
      float16v S[T2];
      __builtin_amdgcn_s_setprio(1);
      {
        constexpr int NS = T2 * DK, PF = 4;
        bf16x8 A[PF];
#pragma unroll
        for (int i = 0; i < PF; ++i) A[i] = kr.get(Kt, i / DK, i % DK);
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          const bf16x8 a = A[i % PF];
          if (i + PF < NS) A[i % PF] = kr.get(Kt, (i + PF) / DK, (i + PF) % DK);
          bf16x8 lower = a;
          if constexpr (careful.value && TERMS > 1) lower = finite8(a);
#pragma unroll
          for (int term = TERMS - 1; term >= 0; --term) S[i / DK] = mfma(term ? lower : a, Q[term][i % DK], i % DK == 0 && term == TERMS - 1 ? zero16() : S[i / DK]);
        }
        in_order<NS, PF, TERMS, 1>();
      }
      __builtin_amdgcn_s_setprio(0);
      // ---- mask, running softmax.  m (in units of log2) is a reference, not the exact maximum: it stays while a lane's probabilities of the tile add up to less than 2^40,
      // and most tiles take no maximum at all.
      if (mask) {
        really_branch();
        const int lim = my_last - key0 - 4 * g;
#pragma unroll
        for (int t2 = 0; t2 < T2; ++t2)
#pragma unroll
          for (int r = 0; r < 16; ++r) S[t2][r] = t2 * 32 + 8 * (r >> 2) + (r & 3) <= lim ? S[t2][r] : -INFINITY;
      }
      bf16x8 P[TERMS][T2][2];
      auto probabilities = [&]() -> float {
        const float nref = m == -INFINITY ? 0.f : -m;
        float ls[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t2 = 0; t2 < T2; ++t2)
#pragma unroll
          for (int s2 = 0; s2 < 2; ++s2) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              x[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[t2][s2 * 8 + j], c2, nref));
              ls[j >> 1] += x[j];
            }
            if constexpr (TERMS == 1) {
              P[0][t2][s2] = __builtin_bit_cast(bf16x8, pack8(x));
            } else {
              bf16x8 t[3];
              three_parts(x, t);
#pragma unroll
              for (int term = 0; term < TERMS; ++term) P[term][t2][s2] = t[term];
            }
          }
        return (ls[0] + ls[1]) + (ls[2] + ls[3]);
      };
      float psum = probabilities();
      if (careful.value || __builtin_amdgcn_ballot_w64(!(psum < 1.0995116e12f) || !(l > 0.f)) != 0) {   // (also where they are not numbers)
        float mc[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int t2 = 0; t2 < T2; ++t2)
#pragma unroll
          for (int r = 0; r < 16; r += 2) mc[(r >> 1) & 3] = __builtin_fmaxf(__builtin_fmaxf(mc[(r >> 1) & 3], S[t2][r]), S[t2][r + 1]);
        const float mx = max_halves(fmaxf(fmaxf(mc[0], mc[1]), fmaxf(mc[2], mc[3]))) * c2;
        const float mn = fmaxf(m, mx);
        // (a row that saw nothing before has zeros to scale, or what set_aside just added, which 0 would spoil)
        const float alpha = mn > m && m != -INFINITY ? __builtin_amdgcn_exp2f(m - mn) : 1.f;
        m = mn;
        l *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) O[dt][r] *= alpha;
        psum = probabilities();
      }
      l += psum;
      if (careful.value && (TERMS > 1 || key0 + KT - 1 > wg_first)) {      // (fp32: an infinite value must not meet a zero among a probability's terms)
#pragma unroll
        for (int t2 = 0; t2 < T2; ++t2) {
          const uint32_t none = row_bits(g, [&](int r) { return !(P[0][t2][r >> 3][r & 7] != (__bf16)0.f); });
          set_aside<D, COLS>(O, Vs[buf] + t2 * 32 * D, g, none, [&](int i) { return row.live && key0 + t2 * 32 + i <= row.last; });
        }
      }
      // ---- O^T += V^T P^T
      {
        constexpr int NS = 2 * T2 * DT, PF = 4;
        bf16x8 A[PF];
#pragma unroll
        for (int i = 0; i < PF; ++i) A[i] = vr.get(Vt, i % DT, i / DT);
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          const bf16x8 a = A[i % PF];
          if (i + PF < NS) A[i % PF] = vr.get(Vt, (i + PF) % DT, (i + PF) / DT);
#pragma unroll
          for (int term = TERMS - 1; term >= 0; --term) O[i % DT] = mfma(a, P[term][i / DT >> 1][i / DT & 1], O[i % DT]);
        }
        in_order<NS, PF, TERMS, 2>();
      }
      settle();
    }
  };
  run(std::false_type{});
  // a value that is not finite may have come from a key that its row does not see, or from large values times probabilities above one
  if (uniform(__syncthreads_or(row.live && any_odd(O)))) run(std::true_type{});

  // ---- normalise and store
  l += other_half(l);
  // (a sum of zero: the row sees nothing, or all its scores are -inf and it has no softmax; of a piece, the join tells)
  const float inv = l > 0.f || l != l ? 1.f / l : !cuts && row.last >= 0 ? __builtin_nanf("") : 0.f;
  const int64_t col = (p.q_off ? (int64_t)q.base : (int64_t)seq_i * p.q_rows) + row.token, at = (int64_t)row.head * p.lse_rows + col;
  const float lse2 = l > 0.f || l != l ? m + __builtin_amdgcn_logf(l) : -INFINITY;
  T* dst = (T*)const_cast<char*>(p.o.p) + (int64_t)q.seq * p.o.bs + (int64_t)(q.base + row.token) * p.o.ts + (int64_t)row.head * p.o.hs;
  float* part = p.part + ((int64_t)split * p.hq * p.lse_rows + at) * p.d;
  if (row.live && g == 0) {
    if (cuts) p.part[(int64_t)p.nsplit * p.hq * p.lse_rows * p.d + (int64_t)split * p.hq * p.lse_rows + at] = lse2;
    else if (p.lse) p.lse[at] = lse2 * LN2;
  }
  each_piece(O, inv, g, [&](int c, const float (&o)[8]) {
    if (!row.live || c >= p.d) return;
    if (cuts) {
      *(float4v*)(part + c) = float4v{o[0], o[1], o[2], o[3]};
      *(float4v*)(part + c + 4) = float4v{o[4], o[5], o[6], o[7]};
    } else if constexpr (TERMS == 1) {
      *(uint4v*)(dst + c) = pack8(o);
    } else {
      *(float4v*)(dst + c) = float4v{o[0], o[1], o[2], o[3]};
      *(float4v*)(dst + c + 4) = float4v{o[4], o[5], o[6], o[7]};
    }
  });
}

template <typename T, int D>
hipError_t go(const SeqParams& p, const Cache8Scales& sc, const SeqCut& cut, hipStream_t st) {
  const dim3 grid((unsigned)p.slots * (unsigned)p.nsplit * (unsigned)p.hk);
  if (p.d % 16) hipLaunchKernelGGL((k_cache8_attention<T, D, true>), grid, dim3(256), 0, st, p, sc, cut);
  else hipLaunchKernelGGL((k_cache8_attention<T, D, false>), grid, dim3(256), 0, st, p, sc, cut);
  return hipGetLastError();
}

template <typename T>
hipError_t launch(SeqParams p, const Cache8Scales& sc, const SeqPlan& s, hipStream_t st) {
  p.nsplit = s.nsplit;
  p.split_tiles = s.split_tiles;
  p.slots = (int)seq_slots(p.q_off != nullptr, p.q_rows, p.nseq, p.group, 128);
  if (p.slots == 0) return hipSuccess;
  const SeqCut cut{s.resident, 0, SEQ_MANY_KT, 128};
  const hipError_t e = p.d <= 64 ? go<T, 64>(p, sc, cut, st) : go<T, 128>(p, sc, cut, st);
  if (e != hipSuccess || s.nsplit == 1) return e;
  return join_pieces<T>(p, cut, st);
}

}  // namespace

// Few rows of an average sequence and key head, up to 32 (seq_fwd_plan), take tiles of 16 or 32 rows.  For 2 to 64 sequences the lengths decide on the device how long pieces
// are (SeqCut), and the plan says how short they may be; else it cuts by the tensors' sizes.
SeqPlan cache8_plan(const SeqParams& p, int dtype, int num_cu) {
  SeqPlan s = seq_fwd_plan(p, num_cu);
  s.tile_rows = 128;
  if (s.few) {
    const int64_t all = (int64_t)p.q_rows * p.group, mean = p.q_off ? (p.nseq ? all / p.nseq : 0) : all;
    s.tile_rows = mean <= 16 ? 16 : 32;
  }
  const bool lengths = p.nseq >= 2 && p.nseq <= 64;
  const int64_t kt = s.few ? 32 * CACHE8_FEW_WAVES : SEQ_MANY_KT, tiles = ((int64_t)p.k_rows + kt - 1) / kt;
  const int64_t groups = seq_slots(p.q_off != nullptr, p.q_rows, p.nseq, p.group, s.tile_rows) * p.hk;
  const bool fp32 = dtype == FREQATTN_F32, wide = p.d > 64;
  // workgroups that run at the same time
  const int64_t slots = (int64_t)num_cu * (s.few ? cache8_few_waves(fp32, wide, s.tile_rows / 16, p.d % 16 != 0) : fp32 && wide ? 1 : 2);
  int64_t n = 1;
  if (s.few) {
    if (groups > 0 && tiles > CACHE8_ONE_PIECE) n = lengths ? (groups <= 2 * slots ? 4 * slots / p.hk : 1) : slots / groups;
  } else if (!lengths || s.nsplit > 1) {
    return s;
  } else if (groups <= 2 * slots) {
    n = groups > slots + slots / 2 ? 2 : 4;
    if (n > tiles / 16) n = tiles / 16;
  }
  if (n > tiles) n = tiles;
  if (n > MAX_PIECES) n = MAX_PIECES;
  if (n < 1) n = 1;
  s.split_tiles = (int)(tiles > 0 ? (tiles + n - 1) / n : 1);
  s.nsplit = n > 1 ? (int)((tiles + s.split_tiles - 1) / s.split_tiles) : 1;
  s.workspace = s.nsplit > 1 ? (int64_t)s.nsplit * p.hq * p.lse_rows * (p.d + 1) * 4 : 0;
  s.resident = s.nsplit > 1 && lengths ? (int)slots : 0;
  if (s.resident) s.workspace += 16;      // (seq_piece_at)
  return s;
}

hipError_t launch_cache8_attention(SeqParams p, const Cache8Scales& sc, const SeqPlan& s, int dtype, hipStream_t st) {
  if (s.few) return launch_cache8_few(p, sc, s, dtype, st);
  return dtype == FREQATTN_BF16 ? launch<uint16_t>(p, sc, s, st) : launch<float>(p, sc, s, st);
}

}  // namespace fa
