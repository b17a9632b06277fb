// Attention over sequences, bf16, backward.
//
//   delta = rowsum(dO O),  P = exp(S - lse),  dS = P (dO V^T - delta),  dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
//
// Two kernels, 7 products of 2 d flops per pair instead of the 5 that one kernel would need: k_seq_dq owns query rows and sums over keys, k_seq_dkv owns
// keys and sums over query rows, each in registers and in a fixed order.  One kernel would have to add one of the two sums up through memory, by
// fp32 atomics whose order changes from run to run.
// Both keep their products transposed as the forward pass does (the owned row on the lane), so that P and dS, rounded to bf16 in the accumulator
// registers, are the second operand of the products that follow.  k_seq_dq reads K by rows (S) and by columns (dQ), V by rows (dO V^T); k_seq_dkv
// reads Q and dO both ways.  k_seq_dq goes first and leaves (lse, delta) of every row, lse in units of log2, in the workspace.
#include "seq_mfma.h"

namespace fa {

using namespace seq;

namespace {

__device__ const float no_row[2] = {INFINITY, 0.f};     // lse and delta of a row that does not exist: its probabilities are zero

// 4 bytes a lane, to LDS bytes dst + 4 lane
__device__ __forceinline__ void copy4_any(const void* addr, unsigned dst) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(addr), "s"(uniform((int)dst)) : "memory", "m0");
}

template <int D, int NW, int KT>
__global__ void __launch_bounds__(64 * NW, 2) k_seq_dq(SeqParams p) {
  constexpr int DT = D / 32, DK = D / 16, T2 = KT / 32, TILE = 32 * NW;
  __shared__ __attribute__((aligned(16))) uint16_t Ks[2][KT * D];
  __shared__ __attribute__((aligned(16))) uint16_t Vs[2][KT * D];
  const int lane = threadIdx.x & 63, nn = lane & 31, g = lane >> 5, wave = uniform(threadIdx.x >> 6);
  const int kvh = (int)(blockIdx.x % (unsigned)p.hk);
  int seq_i, tile_i;
  seq_slot(p.q_off, p.q_rows, p.nseq, p.group, TILE, p.slots - 1 - (int)(blockIdx.x / (unsigned)p.hk), seq_i, tile_i);
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
  const int64_t col = (p.q_off ? (int64_t)q.base : (int64_t)seq_i * p.q_rows) + row.token, at = (int64_t)row.head * p.lse_rows + col;
  float lse2 = row.live ? p.lse[at] * LOG2E : 0.f;
  // A row that sees no key (lse -inf) has no probabilities; one whose scores hold +inf has no finite ones.
  if (lse2 == -INFINITY) { lse2 = INFINITY; delta = 0.f; }
  else if (lse2 == INFINITY) lse2 = __builtin_nanf("");
  if (row.live && g == 0) *(float2v*)(p.delta + 2 * at) = float2v{lse2, delta};

  RowRead<D> rr;
  rr.template set<BOTH>(nn, g);
  ColRead<D> cr;
  cr.template set<BOTH>(lane);
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

  const float c2 = p.scale * LOG2E;
  float16v A[DT];
  auto run = [&](auto careful) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) A[dt] = zero16();
    if (tiles > 0) copy_tile(0, 0);
    auto next_tile = [&] {
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      __syncthreads();
    };
    next_tile();
    for (int t = 0; t < tiles; ++t, next_tile()) {
      const int buf = t & 1, key0 = t * KT;
      uint16_t* Kt = Ks[buf];
      const uint16_t* Vt = Vs[buf];
      if (careful.value && key0 + KT - 1 > wg_first) set_aside<D, KT, BOTH>(A, Kt, g, [&](int i) { return row.live && key0 + i <= row.last; });
      if (t + 1 < tiles) copy_tile(t + 1, buf ^ 1);
      if (key0 > wave_last) continue;
#pragma unroll
      for (int t2 = 0; t2 < T2; ++t2) {
        const int first = key0 + t2 * 32;
        float16v S = zero16(), dP = zero16();
#pragma unroll
        for (int s = 0; s < DK; ++s) S = mfma(rr.get(Kt, t2, s), Q[s], S);
#pragma unroll
        for (int s = 0; s < DK; ++s) dP = mfma(rr.get(Vt, t2, s), G[s], dP);
#pragma unroll
        for (int r = 0; r < 16; ++r) S[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[r], c2, -lse2)) * (dP[r] - delta);
        if (first + 31 > wave_first) {
          const int lim = my_last - first - 4 * g;
#pragma unroll
          for (int r = 0; r < 16; ++r) S[r] = 8 * (r >> 2) + (r & 3) <= lim ? S[r] : 0.f;
        }
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
          uint4v pk;
#pragma unroll
          for (int j = 0; j < 4; ++j) pk[j] = pack2(S[s2 * 8 + 2 * j], S[s2 * 8 + 2 * j + 1]);
          const bf16x8 dS = __builtin_bit_cast(bf16x8, pk);
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) A[dt] = mfma(cr.get(Kt, dt, 2 * t2 + s2), dS, A[dt]);
        }
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

// 32 * NW keys, over all query rows of the group's heads that see any of them, QT rows of one head at a time.
// V stays in LDS at D = 128: with it in registers too, a wave would need more than the 256 that two waves per SIMD leave it.
template <int D, int NW, int QT>
__global__ void __launch_bounds__(64 * NW, 2) k_seq_dkv(SeqParams p) {
  constexpr int DT = D / 32, DK = D / 16, T2 = QT / 32, TILE = 32 * NW;
  constexpr bool V_LDS = D == 128;
  __shared__ __attribute__((aligned(16))) uint16_t Qs[2][QT * D];
  __shared__ __attribute__((aligned(16))) uint16_t Gs[2][QT * D];
  __shared__ __attribute__((aligned(16))) uint16_t Vs[V_LDS ? TILE * D : 8];
  __shared__ __attribute__((aligned(16))) float St[2][2 * QT];     // (lse, delta) of the tile's rows
  const int lane = threadIdx.x & 63, nn = lane & 31, g = lane >> 5, wave = uniform(threadIdx.x >> 6);
  // key heads fastest; tiles from the first: under the causal mask the first keys are seen by the most rows
  const int kvh = (int)(blockIdx.x % (unsigned)p.hk);
  int seq_i, tile_i;
  seq_slot(p.k_off, p.k_rows, p.nseq, 1, TILE, (int)(blockIdx.x / (unsigned)p.hk), seq_i, tile_i);
  seq_i = uniform(seq_i);
  tile_i = uniform(tile_i);
  const SeqRange q = uniform(seq_range(p.q_off, p.q_len, p.q_rows, seq_i)), k = uniform(seq_range(p.k_off, p.k_len, p.k_rows, seq_i));
  if (tile_i >= (k.n + TILE - 1) / TILE) return;
  const int key0 = tile_i * TILE, key = key0 + wave * 32 + nn, chunks = p.d >> 3;
  const bool live = key < k.n;
  const int wave_last = key0 + wave * 32 + 31, wg_last = key0 + TILE - 1;     // last keys of the wave and of the workgroup (dead ones too)

  const uint16_t* ks = (const uint16_t*)p.k.p + (int64_t)k.seq * p.k.bs + (int64_t)(k.base + (live ? key : 0)) * p.k.ts + (int64_t)kvh * p.k.hs;
  const uint16_t* vs = (const uint16_t*)p.v.p + (int64_t)k.seq * p.v.bs + (int64_t)(k.base + (live ? key : 0)) * p.v.ts + (int64_t)kvh * p.v.hs;
  bf16x8 K[DK], V[V_LDS ? 1 : DK];
#pragma unroll
  for (int s = 0; s < DK; ++s) {
    uint4v x = {0u, 0u, 0u, 0u}, y = x;
    if (live && 2 * s + g < chunks) {
      x = *(const uint4v*)(ks + s * 16 + g * 8);
      y = *(const uint4v*)(vs + s * 16 + g * 8);
    }
    K[s] = __builtin_bit_cast(bf16x8, x);
    if constexpr (V_LDS) *(uint4v*)(Vs + (wave * 32 + nn) * D + (((2 * s + g) ^ swizzle<D, ROWS>(nn)) << 3)) = y;
    else V[s] = __builtin_bit_cast(bf16x8, y);
  }

  RowRead<D> rr, vr;
  rr.template set<BOTH>(nn, g);
  vr.template set<ROWS>(nn, g);
  ColRead<D> cr;
  cr.template set<BOTH>(lane);
  using Copy = TileCopy<D, NW, QT, BOTH>;
  Copy qc, gc;
  const int64_t q_bytes = p.q.ts * 2, g_bytes = p.dout.ts * 2;
  qc.set(q_bytes, wave, lane);
  gc.set(g_bytes, wave, lane);
  const unsigned q_lds = lds_address(Qs[0]), g_lds = lds_address(Gs[0]), s_lds = (unsigned)(uintptr_t)(const __attribute__((address_space(3))) float*)St[0];
  constexpr int NI = Copy::NI, TB = QT * D * 2;
  // query tiles: those of the first token that sees the first key and on, for one head of the group after the other
  int first = p.causal ? key0 - (k.n - q.n) : 0;
  if (first < 0) first = 0;
  const int tile0 = first / QT, per_head = q.n > first ? (q.n + QT - 1) / QT - tile0 : 0, all = per_head * p.group;
  auto copy_tile = [&](int head, int tile, int buf) {
    const int row0 = tile * QT, h = kvh * p.group + head;
    auto qcur = qc.begin(p.q.p + 2 * ((int64_t)q.seq * p.q.bs + (int64_t)(q.base + row0) * p.q.ts + (int64_t)h * p.q.hs), q_bytes, wave);
    auto gcur = gc.begin(p.dout.p + 2 * ((int64_t)q.seq * p.dout.bs + (int64_t)(q.base + row0) * p.dout.ts + (int64_t)h * p.dout.hs), g_bytes, wave);
    if (row0 + QT <= q.n && chunks == D / 8) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        qc.whole(qcur, q_bytes, q_lds + buf * TB, wave, i);
        gc.whole(gcur, g_bytes, g_lds + buf * TB, wave, i);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NI; ++i) qc.part(qcur, q_bytes, q_lds + buf * TB, wave, lane, i, q.n - row0, chunks);
#pragma unroll
      for (int i = 0; i < NI; ++i) gc.part(gcur, g_bytes, g_lds + buf * TB, wave, lane, i, q.n - row0, chunks);
    }
    if (wave < 2 * QT / 64) {
      const int i = wave * 64 + lane;     // (two floats a row)
      const int64_t at = (int64_t)h * p.lse_rows + (p.q_off ? (int64_t)q.base : (int64_t)seq_i * p.q_rows) + row0;
      copy4_any(row0 + (i >> 1) < q.n ? p.delta + 2 * at + i : no_row + (i & 1), s_lds + buf * (2 * QT * 4) + wave * 256);
    }
  };

  const float c2 = p.scale * LOG2E;
  float16v dK[DT], dV[DT];
  auto run = [&](auto careful) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) { dK[dt] = zero16(); dV[dt] = zero16(); }
    int head = 0, tile = tile0;
    if (all > 0) copy_tile(0, tile0, 0);
    auto next_tile = [&] {
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      __syncthreads();
    };
    next_tile();
    for (int t = 0; t < all; ++t, next_tile()) {
      const int buf = t & 1, row0 = tile * QT;
      uint16_t* Qt = Qs[buf];
      uint16_t* Gt = Gs[buf];
      // the last key that row i of the tile sees is shift + i
      const int shift = p.causal ? row0 + k.n - q.n : 1 << 29;
      if (careful.value && (shift < wg_last || row0 + QT > q.n)) {
        auto seen = [&](int i) { return live && row0 + i < q.n && key <= shift + i; };
        set_aside<D, QT, BOTH>(dV, Gt, g, seen);
        set_aside<D, QT, BOTH>(dK, Qt, g, seen);
      }
      if (++tile == tile0 + per_head) { tile = tile0; ++head; }
      if (t + 1 < all) copy_tile(head, tile, buf ^ 1);
#pragma unroll
      for (int t2 = 0; t2 < T2; ++t2) {
        if (shift + t2 * 32 + 31 < key0 + wave * 32) continue;    // (uniform) no row of the half sees a key of the wave
        float16v S = zero16(), dP = zero16();
#pragma unroll
        for (int s = 0; s < DK; ++s) S = mfma(rr.get(Qt, t2, s), K[s], S);
#pragma unroll
        for (int s = 0; s < DK; ++s) {
          if constexpr (V_LDS) dP = mfma(rr.get(Gt, t2, s), vr.get(Vs, wave, s), dP);
          else dP = mfma(rr.get(Gt, t2, s), V[s], dP);
        }
        const bool mask = shift + t2 * 32 < wave_last;
        const int lim = key - shift - t2 * 32 - 4 * g;     // row 8 (r / 4) + 4 g + r % 4 sees the lane's key where that is lim or more
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
          uint4v pp, ps;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float* st = St[buf] + 2 * (t2 * 32 + 8 * (2 * s2 + i) + 4 * g);
            const float4v a = *(const float4v*)st, b = *(const float4v*)(st + 4);
            const float lse[4] = {a[0], a[2], b[0], b[2]}, del[4] = {a[1], a[3], b[1], b[3]};
            float x[4], y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int r = 8 * s2 + 4 * i + j;
              x[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[r], c2, -lse[j]));
              y[j] = x[j] * (dP[r] - del[j]);
              if (mask) {
                const bool seen = 8 * (r >> 2) + (r & 3) >= lim;
                x[j] = seen ? x[j] : 0.f;
                y[j] = seen ? y[j] : 0.f;
              }
            }
            pp[2 * i] = pack2(x[0], x[1]); pp[2 * i + 1] = pack2(x[2], x[3]);
            ps[2 * i] = pack2(y[0], y[1]); ps[2 * i + 1] = pack2(y[2], y[3]);
          }
          const bf16x8 P = __builtin_bit_cast(bf16x8, pp), dS = __builtin_bit_cast(bf16x8, ps);
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            dV[dt] = mfma(cr.get(Gt, dt, 2 * t2 + s2), P, dV[dt]);
            dK[dt] = mfma(cr.get(Qt, dt, 2 * t2 + s2), dS, dK[dt]);
          }
        }
      }
    }
  };
  run(std::false_type{});
  if (p.causal && uniform(__syncthreads_or(live && (any_odd(dK) || any_odd(dV))))) run(std::true_type{});
  auto out = [&](const HeadsPtr& v) { return (uint16_t*)const_cast<char*>(v.p) + (int64_t)k.seq * v.bs + (int64_t)(k.base + (live ? key : 0)) * v.ts + (int64_t)kvh * v.hs; };
  uint16_t *dk = out(p.dk), *dv = out(p.dv);
  each_piece(dK, p.scale, g, [&](int c, const float (&o)[8]) {
    if (live && c < p.d) *(uint4v*)(dk + c) = pack8(o);
  });
  each_piece(dV, 1.f, g, [&](int c, const float (&o)[8]) {
    if (live && c < p.d) *(uint4v*)(dv + c) = pack8(o);
  });
}

template <int D, int QT>
hipError_t go(SeqParams p, hipStream_t st) {
  p.slots = (int)seq_slots(p.q_off != nullptr, p.q_rows, p.nseq, p.group, 128);
  if (p.slots > 0) hipLaunchKernelGGL((k_seq_dq<D, 4, 64>), dim3((unsigned)p.slots * (unsigned)p.hk), dim3(256), 0, st, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  p.slots = (int)seq_slots(p.k_off != nullptr, p.k_rows, p.nseq, 1, 128);
  if (p.slots > 0) hipLaunchKernelGGL((k_seq_dkv<D, 4, QT>), dim3((unsigned)p.slots * (unsigned)p.hk), dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_seq_bwd(const SeqParams& p, hipStream_t st) { return p.d <= 64 ? go<64, 64>(p, st) : go<128, 32>(p, st); }

}  // namespace fa
