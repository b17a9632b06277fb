// Attention over sequences, bf16, forward: one pass over the keys with a running maximum and sum.
//
// A workgroup takes 32 * NW query rows of a sequence and key head (rows: tokens x heads of the group) and walks the key tiles that its rows see.
// Scores are kept transposed, S^T = K Q^T, so that a lane owns one query: maximum and sum of a row take one exchange between the two lane
// halves, and the accumulator registers, rounded to bf16, are the second operand of O^T += V^T P^T as they stand (rows of V come in that order
// from transposing LDS reads).  K and V tiles are copied into the other half of LDS while this half is used.
// Probabilities are rounded to bf16 for the product; their sum is taken before the rounding, in fp32, as lse needs it.
//
// Few rows (a token of each of some sequences): tiles of 32 rows, one wave a workgroup, and the keys are cut into pieces of `split_tiles` tiles
// that run as workgroups of their own; their normalised results and log sums are joined by k_seq_join.
//
// Bound: long rows by the matrix cores at the clock that power leaves them (32,768 causal rows, 4 / 1 heads of 128: 1.02 ms, 1.08 PFLOP/s; in a run with counters, 1.17 ms,
// they were busy 57 % at 1.58 GHz), at head_dim 64 as much by the exponentials (16,384 rows x 8 heads: 0.66-0.69 ms, 0.8 PFLOP/s, busy 42 % at 1.91 GHz); few
// rows by memory (32 tokens against caches of 200 to 16,384 rows, 32 / 8 heads of 128: 217 us, 4.9 TB/s).
#include "seq_join.h"
#include "seq_mfma.h"

namespace fa {

using namespace seq;

namespace {

// (D = 64 fits three waves per SIMD: 720 -> 691 us for 16,384 rows x 8 heads)
template <int D, int NW, int KT>
__global__ void __launch_bounds__(64 * NW, D == 64 ? 3 : 2) k_seq_fwd(SeqParams p) {
  constexpr int DT = D / 32, DK = D / 16, T2 = KT / 32, TILE = 32 * NW;
  // One wave has one K and one V tile: the next K tile is requested when the scores are done, the next V tile when the product is, and other
  // workgroups of the compute unit (nine at D = 128) fill the wait.  More waves share two of each.
  constexpr bool ONE = NW == 1;
  constexpr int NB = ONE ? 1 : 2;
  __shared__ __attribute__((aligned(256))) uint16_t Ks[NB][KT * D];
  __shared__ __attribute__((aligned(256))) uint16_t Vs[NB][KT * D];
  const int lane = threadIdx.x & 63, nn = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // key heads fastest, then tiles, the longest first, then pieces of the keys (pieces that do not exist would leave the XCDs that they fall on idle if they
  // were between tiles)
  unsigned id = blockIdx.x;
  const int kvh = (int)(id % (unsigned)p.hk);
  id /= (unsigned)p.hk;
  const int split = (int)(id / (unsigned)p.slots), slot = (int)(id % (unsigned)p.slots);
  int seq_i, tile_i;
  if (ONE) seq_slot(p.q_off, p.q_rows, p.nseq, p.group, TILE, slot, seq_i, tile_i);
  else if (!seq_query_tile(p, TILE, lane, slot, seq_i, tile_i)) return;
  seq_i = uniform(seq_i);
  tile_i = uniform(tile_i);
  const SeqRange q = uniform(seq_range(p.q_off, p.q_len, p.q_rows, seq_i)), k = uniform(seq_range(p.k_off, p.k_len, p.k_rows, seq_i));
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
  // dead rows of a live wave act as its last one: their scores are zeros, nothing of them is stored
  const int my_last = row.live ? row.last : wave_last;

  const int t_all = (wg_last + KT) / KT;                       // tiles the workgroup's rows see (0: none)
  const int t0 = split * p.split_tiles, t1 = p.nsplit > 1 ? min(t0 + p.split_tiles, t_all) : t_all;
  if (p.nsplit > 1 && t0 >= t_all && split > 0) return;        // (piece 0 of a row that sees nothing stores that)

  const int chunks = p.d >> 3;
  bf16x8 Q[DK];
  {
    const uint16_t* src = (const uint16_t*)p.q.p + (int64_t)q.seq * p.q.bs + (int64_t)(q.base + row.token) * p.q.ts + (int64_t)row.head * p.q.hs;
#pragma unroll
    for (int s = 0; s < DK; ++s) {
      uint4v x = {0u, 0u, 0u, 0u};
      if (row.live && 2 * s + g < chunks) x = *(const uint4v*)(src + s * 16 + g * 8);
      Q[s] = __builtin_bit_cast(bf16x8, x);
    }
  }
  const float c2 = p.scale * LOG2E;

  RowRead<D> kr;
  kr.template set<ROWS>(nn, g);
  ColRead<D, COLS> vr;
  vr.set(lane);
  TileCopy<D, NW, KT, ROWS> kc;
  TileCopy<D, NW, KT, COLS> vc;
  const int64_t k_bytes = p.k.ts * 2, v_bytes = p.v.ts * 2;
  kc.set(k_bytes, wave, lane);
  vc.set(v_bytes, wave, lane);
  const char* kb = p.k.p + 2 * ((int64_t)k.seq * p.k.bs + (int64_t)k.base * p.k.ts + (int64_t)kvh * p.k.hs);
  const char* vb = p.v.p + 2 * ((int64_t)k.seq * p.v.bs + (int64_t)k.base * p.v.ts + (int64_t)kvh * p.v.hs);
  const unsigned k_lds = lds_address(Ks[0]), v_lds = lds_address(Vs[0]);
  constexpr int NI = TileCopy<D, NW, KT, ROWS>::NI, TB = KT * D * 2;
  // the copies of tile t, in order: K (even) and V (odd)
  using KC = typename TileCopy<D, NW, KT, ROWS>::Cursor;
  using VC = typename TileCopy<D, NW, KT, COLS>::Cursor;
  auto k_begin = [&](int t) { return kc.begin(kb + (int64_t)t * KT * k_bytes, k_bytes, wave); };
  auto v_begin = [&](int t) { return vc.begin(vb + (int64_t)t * KT * v_bytes, v_bytes, wave); };
  auto copy = [&](KC& kcur, VC& vcur, int buf, int i) {
    if ((i & 1) == 0) kc.whole(kcur, k_bytes, k_lds + buf * TB, wave, i >> 1);
    else vc.whole(vcur, v_bytes, v_lds + buf * TB, wave, i >> 1);
  };
  auto is_whole = [&](int t) { return (t + 1) * KT <= k.n && chunks == D / 8; };
  auto copy_k = [&](int t, int buf) {
    KC cur = k_begin(t);
    if (is_whole(t)) {
#pragma unroll
      for (int i = 0; i < NI; ++i) kc.whole(cur, k_bytes, k_lds + buf * TB, wave, i);
    } else {
#pragma unroll
      for (int i = 0; i < NI; ++i) kc.part(cur, k_bytes, k_lds + buf * TB, wave, lane, i, k.n - t * KT, chunks);
    }
  };
  auto copy_v = [&](int t, int buf) {
    VC cur = v_begin(t);
    if (is_whole(t)) {
#pragma unroll
      for (int i = 0; i < NI; ++i) vc.whole(cur, v_bytes, v_lds + buf * TB, wave, i);
    } else {
#pragma unroll
      for (int i = 0; i < NI; ++i) vc.part(cur, v_bytes, v_lds + buf * TB, wave, lane, i, k.n - t * KT, chunks);
    }
  };
  auto wait_copies = [&](bool all) {    // all but the last NI, or all; and this wave's LDS reads
    if (all) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(NI) : "memory");
  };

  float16v O[DT];
  float m, l;
  // careful: the second pass of a workgroup whose result was not finite, with values set aside (set_aside) and the maximum as the reference
  auto run = [&](auto careful) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) O[dt] = zero16();
    m = -INFINITY;
    l = 0.f;
    auto next_tile = [&] {
      if (!ONE) { wait_copies(true); __syncthreads(); }
    };
    if (t0 < t1) { copy_k(t0, 0); copy_v(t0, 0); }
    next_tile();
    for (int t = t0; t < t1; ++t, next_tile()) {
      const int buf = ONE ? 0 : (t - t0) & 1, key0 = t * KT;
      const unsigned Kt = k_lds + buf * TB, Vt = v_lds + buf * TB;
      const bool more = t + 1 < t1;
      if (!careful.value && !ONE && key0 > wave_last) {   // (uniform over the wave) none of its rows sees the tile (set_aside needs every wave: all masked below)
        if (more) { copy_k(t + 1, buf ^ 1); copy_v(t + 1, buf ^ 1); }
        continue;
      }
      if (ONE) wait_copies(false);
      const bool mask = key0 + KT - 1 > wave_first;
      // ---- S^T = K Q^T; the next tile's copies are spread over the products
      float16v S[T2];
      __builtin_amdgcn_s_setprio(1);
      auto scores = [&](auto copies) {
        constexpr int NS = T2 * DK, PF = NS < 8 ? NS : 8;
        KC kcur{nullptr};
        VC vcur{nullptr};
        if (copies.value) { kcur = k_begin(t + 1); vcur = v_begin(t + 1); }
        bf16x8 A[PF];
#pragma unroll
        for (int i = 0; i < PF; ++i) A[i] = kr.get(Kt, i / DK, i % DK);
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          const bf16x8 a = A[i % PF];
          if (i + PF < NS) A[i % PF] = kr.get(Kt, (i + PF) / DK, (i + PF) % DK);
          S[i / DK] = mfma(a, Q[i % DK], i % DK == 0 ? zero16() : S[i / DK]);
          if (copies.value) {
#pragma unroll
            for (int c = i * (2 * NI) / NS; c < (i + 1) * (2 * NI) / NS; ++c) copy(kcur, vcur, buf ^ 1, c);
          }
        }
        __builtin_amdgcn_sched_group_barrier(0x100, PF, 0);   // PF reads up front, then one read per product
#pragma unroll
        for (int i = 0; i < NS - PF; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, PF, 0);
      };
      if (!ONE && more && is_whole(t + 1)) scores(std::bool_constant<!ONE>{});
      else {
        if (!ONE && more) { copy_k(t + 1, buf ^ 1); copy_v(t + 1, buf ^ 1); }
        scores(std::false_type{});
      }
      __builtin_amdgcn_s_setprio(0);
      if (ONE && more) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        copy_k(t + 1, 0);
      }
      // ---- mask, running softmax.  m (in units of log2) is a reference, not the exact maximum.  bf16 has the range of fp32, so a probability above one
      // loses no precision: the reference stays while a lane's probabilities of the tile add up to less than 2^40 (exact relative to their sum), and most
      // tiles take no maximum at all.  Where they do not, or the row has no probabilities yet, the tile's maximum becomes the reference.  Values above some
      // 2^88 may overflow under such a reference: the second pass takes the maximum of every tile.
      if (mask) {
        really_branch();
        const int lim = my_last - key0 - 4 * g;
#pragma unroll
        for (int t2 = 0; t2 < T2; ++t2)
#pragma unroll
          for (int r = 0; r < 16; ++r) S[t2][r] = t2 * 32 + 8 * (r >> 2) + (r & 3) <= lim ? S[t2][r] : -INFINITY;
      }
      bf16x8 P[T2][2];
      auto probabilities = [&]() -> float {
        const float nref = m == -INFINITY ? 0.f : -m;
        float ls[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t2 = 0; t2 < T2; ++t2)
#pragma unroll
          for (int s2 = 0; s2 < 2; ++s2) {
            uint4v pk;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(S[t2][s2 * 8 + 2 * j], c2, nref));
              const float b = __builtin_amdgcn_exp2f(__builtin_fmaf(S[t2][s2 * 8 + 2 * j + 1], c2, nref));
              ls[j] += a;
              ls[j] += b;
              pk[j] = pack2(a, b);
            }
            P[t2][s2] = __builtin_bit_cast(bf16x8, pk);
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
      if (ONE) {
        wait_copies(!more);
      }
      if (careful.value && key0 + KT - 1 > wg_first) {
#pragma unroll
        for (int t2 = 0; t2 < T2; ++t2) {
          const uint32_t none = row_bits(g, [&](int r) { return !(P[t2][r >> 3][r & 7] != (__bf16)0.f); });
          set_aside<D, COLS>(O, Vs[buf] + t2 * 32 * D, g, none, [&](int i) { return row.live && key0 + t2 * 32 + i <= row.last; });
        }
      }
      // ---- O^T += V^T P^T
      {
        constexpr int NS = 2 * T2 * DT, PF = NS < 8 ? NS : 8;
        bf16x8 A[PF];
#pragma unroll
        for (int i = 0; i < PF; ++i) A[i] = vr.get(Vt, i % DT, i / DT);
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          const bf16x8 a = A[i % PF];
          if (i + PF < NS) A[i % PF] = vr.get(Vt, (i + PF) % DT, (i + PF) / DT);
          O[i % DT] = mfma(a, P[i / DT >> 1][i / DT & 1], O[i % DT]);
        }
        __builtin_amdgcn_sched_group_barrier(0x100, 2 * PF, 0);   // PF operands up front, then one operand (two reads) per product
#pragma unroll
        for (int i = 0; i < NS - PF; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, PF, 0);
      }
      if (ONE && more) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        copy_v(t + 1, 0);
      }
    }
  };
  run(std::false_type{});
  // a value that is not finite may have come from a key that its row does not see, or from large values times probabilities above one
  if (uniform(__syncthreads_or(row.live && any_odd(O)))) run(std::true_type{});

  // ---- normalise and store
  l += other_half(l);
  // (a sum of zero: the row sees nothing, or all its scores are -inf and it has no softmax; of a piece, the join tells)
  const float inv = l > 0.f || l != l ? 1.f / l : p.nsplit == 1 && row.last >= 0 ? __builtin_nanf("") : 0.f;
  const int64_t col = (p.q_off ? (int64_t)q.base : (int64_t)seq_i * p.q_rows) + row.token, at = (int64_t)row.head * p.lse_rows + col;
  const float lse2 = l > 0.f || l != l ? m + __builtin_amdgcn_logf(l) : -INFINITY;
  uint16_t* dst = (uint16_t*)const_cast<char*>(p.o.p) + (int64_t)q.seq * p.o.bs + (int64_t)(q.base + row.token) * p.o.ts + (int64_t)row.head * p.o.hs;
  float* part = p.part + ((int64_t)split * p.hq * p.lse_rows + at) * p.d;
  if (row.live && g == 0) {
    if (p.nsplit > 1) p.part[(int64_t)p.nsplit * p.hq * p.lse_rows * p.d + (int64_t)split * p.hq * p.lse_rows + at] = lse2;
    else if (p.lse) p.lse[at] = lse2 * LN2;
  }
  each_piece(O, inv, g, [&](int c, const float (&o)[8]) {
    if (!row.live || c >= p.d) return;
    if (p.nsplit > 1) {
      *(float4v*)(part + c) = float4v{o[0], o[1], o[2], o[3]};
      *(float4v*)(part + c + 4) = float4v{o[4], o[5], o[6], o[7]};
    } else {
      *(uint4v*)(dst + c) = pack8(o);
    }
  });
}

template <int D, int NW, int KT>
hipError_t go(const SeqParams& p, hipStream_t st) {
  hipLaunchKernelGGL((k_seq_fwd<D, NW, KT>), dim3((unsigned)p.slots * (unsigned)p.nsplit * (unsigned)p.hk), dim3(64 * NW), 0, st, p);
  return hipGetLastError();
}

constexpr int FEW_KT = SEQ_FEW_KT, MANY_KT = SEQ_MANY_KT;

}  // namespace

// How a forward call is cut.  Lengths are on the device, so the cut goes by the tensors' sizes, and suits batches whose sequences are alike.  Where they are not it costs: 64 tokens
// beside a prompt of 4096 rows (32 / 8 heads, caches of 4096) take 250 us, alone 123 and 142; packed keys count as one long sequence, so that the pieces of 32
// tokens against 32 x 4096 packed keys are longer than the sequences: 170 us, as a cache 108.
SeqPlan seq_fwd_plan(const SeqParams& p, int num_cu) {
  SeqPlan s = {};
  const bool packed = p.q_off != nullptr;
  // By the rows of an average sequence and key head: more than 32 would take several one-wave tiles, each reading all keys.
  const int64_t all = (int64_t)p.q_rows * p.group, mean = packed ? (p.nseq ? all / p.nseq : 0) : all;
  s.few = mean <= 32;
  const int tile_rows = s.few ? 32 : 128, kt = s.few ? FEW_KT : MANY_KT;
  const int64_t slots = seq_slots(packed, p.q_rows, p.nseq, p.group, tile_rows), groups = slots * p.hk, key_tiles = ((int64_t)p.k_rows + kt - 1) / kt;
  s.nsplit = 1;
  s.split_tiles = (int)(key_tiles > 0 ? key_tiles : 1);
  // Few rows: 16 one-wave workgroups for each compute unit (nine are resident); with 8 a batch whose caches are filled to an eighth of their rows is left with
  // too few (32 tokens, 2000 of 16,384 rows: 73 us instead of 47), full ones gain 2 %.  Many rows: two workgroups for each where there is less than one; with
  // four where there are less than two, joining costs more than the shorter chains give (16 heads x 2500 rows 64 us instead of 70, 4 sequences of 64
  // rows against 4096 keys 36 instead of 48).
  const int64_t target = (int64_t)num_cu * (s.few ? 16 : 2);
  if (groups > 0 && groups < target / 2 && key_tiles > 1) {
    int64_t n = target / groups;
    if (n > key_tiles) n = key_tiles;
    if (n > MAX_PIECES) n = MAX_PIECES;
    s.split_tiles = (int)((key_tiles + n - 1) / n);
    s.nsplit = (int)((key_tiles + s.split_tiles - 1) / s.split_tiles);
  }
  s.workspace = s.nsplit > 1 ? (int64_t)s.nsplit * p.hq * p.lse_rows * (p.d + 1) * 4 : 0;
  return s;
}

hipError_t launch_seq_fwd(SeqParams p, const SeqPlan& s, hipStream_t st) {
  p.nsplit = s.nsplit;
  p.split_tiles = s.split_tiles;
  p.slots = (int)seq_slots(p.q_off != nullptr, p.q_rows, p.nseq, p.group, s.few ? 32 : 128);
  if (p.slots == 0) return hipSuccess;
  hipError_t e;
  if (s.few) e = p.d <= 64 ? go<64, 1, FEW_KT>(p, st) : go<128, 1, FEW_KT>(p, st);
  else e = p.d <= 64 ? go<64, 4, MANY_KT>(p, st) : go<128, 4, MANY_KT>(p, st);
  if (e != hipSuccess || s.nsplit == 1) return e;
  return join_pieces<uint16_t>(p, SeqCut{0, 0, s.few ? FEW_KT : MANY_KT, s.few ? 32 : 128}, st);
}

}  // namespace fa
