// Attention over caches held in 8 bits for few query rows: single tokens, a few of them.  Same mathematics as the kernel of many rows (seq_cache8.hip); what counts here is
// how many bytes of the cache are on their way at any time.
//
// A workgroup takes 16 NQ query rows of a sequence and key head (tokens x heads of the group) and a piece of the keys; its NW waves take 32 keys each of every
// 32 NW, by themselves, and their results meet in LDS at the end.  Products are 16 x 16 x 32, so that 16 rows waste little.
//   S^T = K Q^T    a lane holds the codes of one key: they are widened in registers and multiplied as they stand.  The channels of a step are those that the lane's 16-byte
//                  pieces hold (64 (s / 2) + 16 g + 8 (s % 2) for lane group g), which the queries follow
//   O^T += V^T P^T a lane of S^T holds keys 4 g + r and 16 + 4 g + r of one query, which is the order in which V's rows come from transposing LDS reads
// With bf16 queries a probability is rounded to bf16 as an operand (see there).
// Few registers (O takes D / 4 a lane and 16 rows) let many waves run at once, each with its next 32 keys under way.
//
// Bound by memory once the caches are long: one token of 32 requests against 16,384 rows, 32 / 8 heads of 128: 211 us, 5.1 TB/s (bf16 cache 380; fp32 queries 220); 128 against 1024: 48, 5.6; heads of 64,
// 8 / 8: 114, 4.7; caches of 200 to 16,384 rows 115, of which the join 7.  Short ones by latency: one token of one request against 777 rows 8.1, against 16,384 in two launches 15.5.
//
// A value that is not finite and that not every row of the tile sees must not reach the others as 0 x NaN, nor an infinite one meet a zero among the three terms of an fp32 number: where a
// wave's result is not finite, it runs again, with the tiles that have masked pairs (fp32: or such values) multiplied pair by pair, and such keys by the first term alone.
#include "cache8_tile.h"
#include "seq_join.h"

namespace fa {

using namespace seq;

namespace {

__device__ __forceinline__ float4v mfma16(const bf16x8& a, const bf16x8& b, const float4v& c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Over the four lanes that hold a query's keys.
template <typename F>
__device__ __forceinline__ float over_groups(float x, F&& f) {
  uint32_t b = __float_as_uint(x);
  const auto s = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  x = f(__uint_as_float(s[0]), __uint_as_float(s[1]));
  b = __float_as_uint(x);
  const auto u = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return f(__uint_as_float(u[0]), __uint_as_float(u[1]));
}

template <typename T, int D, int NQ, int NW, bool HALF>
__global__ void __launch_bounds__(64 * NW, cache8_few_waves(sizeof(T) == 4, D > 64, NQ, HALF)) k_cache8_few(SeqParams p, Cache8Scales sc, SeqCut cut) {
  constexpr int DT = D / 16, ST = D / 32, PP = D / 64, TILE = 16 * NQ, TERMS = sizeof(T) == 4 ? 3 : 1, WT = 32 * NW;
  __shared__ __attribute__((aligned(256))) uint16_t tiles[NW][32 * D];
  __shared__ float ms[NW][TILE], ls[NW][TILE];
  const int lane = threadIdx.x & 63, ql = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // Up to 8 heads whose channels lie behind each other go to one XCD (workgroups are dealt to the 8 of them in turn) at about the same time: it fetches whole rows of the cache, and
  // a line that two heads share once.
  unsigned id = blockIdx.x;
  {
    const unsigned f = (unsigned)sc.heads_of_row;
    id = (id / (8 * f) * 8 + id % 8) * f + id / 8 % f;
  }
  // key heads fastest, then, cut by lengths, a sequence's tiles and their pieces behind each other; else tiles, then pieces
  const int kvh = (int)(id % (unsigned)p.hk);
  id /= (unsigned)p.hk;
  int seq_i, tile_i, split, piece = p.split_tiles;
  if (cut.resident) {
    int qt, kt;
    seq_tiles(p, cut, lane, qt, kt);
    piece = uniform(seq_piece(p, cut, qt, kt));
    seq_tell(p, piece, kt);
    const int each = seq_pieces(kt, piece), upto = lane_scan(qt * each);
    if ((int)id >= __builtin_amdgcn_readlane(upto, 63)) return;
    seq_i = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > (int)id));
    const int at = (int)id - (seq_i ? __builtin_amdgcn_readlane(upto, seq_i - 1) : 0), n = __builtin_amdgcn_readlane(each, seq_i);
    tile_i = at / n;
    split = at - tile_i * n;
  } else {
    split = (int)(id / (unsigned)p.slots);
    if (split >= p.nsplit) return;
    seq_slot(p.q_off, p.q_rows, p.nseq, p.group, TILE, (int)(id % (unsigned)p.slots), seq_i, tile_i);
  }
  seq_i = uniform(seq_i);
  tile_i = uniform(tile_i);
  split = uniform(split);
  const SeqRange q = uniform(seq_range(p.q_off, p.q_len, p.q_rows, seq_i)), k = uniform(seq_range(nullptr, p.k_len, p.k_rows, seq_i));
  const int rows = q.n * p.group, r_first = tile_i * TILE;
  if ((int64_t)tile_i * TILE >= rows) return;
  Row row[NQ];
#pragma unroll
  for (int i = 0; i < NQ; ++i) row[i] = query_row(p, kvh, r_first + 16 * i + ql, q.n, k.n);
  const int first = last_key(p.causal, r_first / p.group, q.n, k.n), last = last_key(p.causal, (min(r_first + TILE, rows) - 1) / p.group, q.n, k.n);
  int my_last[NQ];     // (dead rows act as the last one; nothing of them is stored)
#pragma unroll
  for (int i = 0; i < NQ; ++i) my_last[i] = row[i].live ? row[i].last : last;

  const int t_all = (last + WT) / WT;                          // steps of all waves that the rows see (0: none)
  const bool cuts = p.nsplit > 1 && (!cut.resident || (k.n + WT - 1) / WT > piece);     // (a sequence in one piece needs no join)
  if (!cuts && split > 0) return;
  const int t0 = cuts ? split * piece : 0, t1 = cuts ? min(t0 + piece, t_all) : t_all;
  if (cuts && t0 >= t_all && split > 0) return;                // (piece 0 of a row that sees nothing stores that)

  bf16x8 Q[NQ][TERMS][ST];
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const T* src = (const T*)p.q.p + (int64_t)q.seq * p.q.bs + (int64_t)(q.base + row[i].token) * p.q.ts + (int64_t)row[i].head * p.q.hs;
#pragma unroll
    for (int s = 0; s < ST; ++s) {
      const int c = 64 * (s >> 1) + 16 * g + 8 * (s & 1);
      const bool in = row[i].live && c < p.d;
      if constexpr (TERMS == 1) {
        uint4v x = {0u, 0u, 0u, 0u};
        if (in) x = *(const uint4v*)(src + c);
        Q[i][0][s] = __builtin_bit_cast(bf16x8, x);
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
        for (int term = 0; term < TERMS; ++term) Q[i][term][s] = t[term];
      }
    }
  }
  const float c2 = p.scale * LOG2E;

  const int n = min(k.n, last + 1);                            // keys that some row sees; the others count as zeros
  const char* kb = p.k.p + (int64_t)k.seq * p.k.bs + (int64_t)kvh * p.k.hs;
  const char* vb = p.v.p + (int64_t)k.seq * p.v.bs + (int64_t)kvh * p.v.hs;
  const uint8_t *ks = sc.k + (int64_t)k.seq * sc.blocks * p.hk + kvh, *vs = sc.v + (int64_t)k.seq * sc.blocks * p.hk + kvh;
  uint16_t* const tile = tiles[wave];
  CodeTile<D, 1, 32, COLS, HALF> vt;
  vt.set(p.v.ts, lane);
  uint4v kx[2][PP];
  int ke[2];
  const int64_t k_off = (int64_t)ql * p.k.ts + 16 * g;
  auto load = [&](int t) {
    const int key0 = t * WT + wave * 32;
    if (key0 >= n) return;       // (uniform over the wave)
    const char* from = kb + (int64_t)key0 * p.k.ts;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      ke[h] = ks[(int64_t)(min(key0 + 16 * h, n - 1) >> sc.shift) * p.hk];
#pragma unroll
      for (int i = 0; i < PP; ++i)
        kx[h][i] = load_piece<HALF>(from + (int64_t)(16 * h) * p.k.ts + k_off + 64 * i, key0 + 16 * h + ql < n, 64 * i + 16 * g, p.d);
    }
    vt.load(vb, p.v.ts, vs, p.hk, sc.shift, key0, n, p.d, 0, lane);
  };
  // LDS byte of the lane's first transposing read: rows 16 h + 4 g + 0..3, channels 16 dt + ql
  unsigned v_at;
  {
    const int r = 4 * g + (ql >> 2);
    v_at = lds_address(tile) + r * D * 2 + (ql & 1) * 8 + ((((ql & 3) >> 1) ^ swizzle<D, COLS>(r)) << 4);
  }
  auto value = [&](int dt) {
    uint4v r;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const unsigned at = (v_at ^ (unsigned)(dt << 5)) + h * 16 * D * 2;
      const uint2v u = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4v __attribute__((address_space(3)))*)(uintptr_t)at));
      r[2 * h] = u[0];
      r[2 * h + 1] = u[1];
    }
    return __builtin_bit_cast(bf16x8, r);
  };

  float4v O[NQ][DT];
  float m[NQ], l[NQ];
  // careful: the second pass of a wave whose result was not finite
  auto run = [&](auto careful) {
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) O[i][dt] = float4v{0.f, 0.f, 0.f, 0.f};
      m[i] = -INFINITY;
      l[i] = 0.f;
    }
    if (!careful.value && t0 < t1) load(t0);
    for (int t = t0; t < t1; ++t) {
      const int key0 = t * WT + wave * 32;
      if (key0 > last) break;    // (uniform over the wave)
      if (careful.value) load(t);
      // ---- S^T = K Q^T
      float4v S[NQ][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int st = 0; st < ST; ++st) {
          const bf16x8 a = __builtin_bit_cast(bf16x8, widen8(kx[h][st >> 1][2 * (st & 1)], kx[h][st >> 1][2 * (st & 1) + 1], ke[h]));
          bf16x8 lower = a;
          if constexpr (careful.value && TERMS > 1) lower = finite8(a);
#pragma unroll
          for (int i = 0; i < NQ; ++i)
#pragma unroll
            for (int term = TERMS - 1; term >= 0; --term)
              S[i][h] = mfma16(term ? lower : a, Q[i][term][st], st == 0 && term == TERMS - 1 ? float4v{0.f, 0.f, 0.f, 0.f} : S[i][h]);
        }
      }
      vt.store(tile, lane);
      if (!careful.value && t + 1 < t1) load(t + 1);
      // ---- mask, running softmax: m (in units of log2) is a reference, not the exact maximum: it stays while a lane's probabilities of the step add up to less than 2^40
      bf16x8 P[NQ][TERMS];
      float pf[NQ][8];
      const bool mask = key0 + 31 > first;
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        if (mask) {
          really_branch();
          const int lim = my_last[i] - key0 - 4 * g;
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[i][h][r] = 16 * h + r <= lim ? S[i][h][r] : -INFINITY;
        }
        auto probabilities = [&]() -> float {
          const float nref = m[i] == -INFINITY ? 0.f : -m[i];
          float sum[2] = {0.f, 0.f};
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            pf[i][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[i][j >> 2][j & 3], c2, nref));
            sum[j & 1] += pf[i][j];
          }
          return sum[0] + sum[1];
        };
        float psum = probabilities();
        if (careful.value || __builtin_amdgcn_ballot_w64(!(psum < 1.0995116e12f) || !(l[i] > 0.f)) != 0) {   // (also where they are not numbers)
          float mx = -INFINITY;
#pragma unroll
          for (int j = 0; j < 8; ++j) mx = __builtin_fmaxf(mx, S[i][j >> 2][j & 3]);
          mx = over_groups(mx, [](float a, float b) { return __builtin_fmaxf(a, b); }) * c2;
          const float mn = fmaxf(m[i], mx);
          const float alpha = mn > m[i] && m[i] != -INFINITY ? __builtin_amdgcn_exp2f(m[i] - mn) : 1.f;
          m[i] = mn;
          l[i] *= alpha;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 4; ++r) O[i][dt][r] *= alpha;
          psum = probabilities();
        }
        l[i] += psum;
        if constexpr (TERMS == 1) {
          uint4v w;
#pragma unroll
          for (int j = 0; j < 4; ++j) w[j] = pack2(pf[i][2 * j], pf[i][2 * j + 1]);
          P[i][0] = __builtin_bit_cast(bf16x8, w);
        } else {
          three_parts(pf[i], P[i]);
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      bool by_pairs = careful.value && mask;
      if constexpr (careful.value && TERMS > 1) {      // (also where a value is not finite: a term of a probability may be zero)
        bool odd = false;
        for (int c = lane; c < 32 * D / 2; c += 64) {
          const uint32_t x = ((const uint32_t*)tile)[c];
          odd = odd || (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u;
        }
        by_pairs = by_pairs || __builtin_amdgcn_ballot_w64(odd) != 0;
      }
      if (by_pairs) {
        // pair by pair: key 16 h + 4 gg + r's probability is on lane group gg
#pragma nounroll
        for (int gg = 0; gg < 4; ++gg)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int key = 16 * (j >> 2) + 4 * gg + (j & 3);
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
              const float mine = TERMS == 1 ? (float)P[i][0][j] : pf[i][j], x = __shfl(mine, 16 * gg + ql);
              const bool seen = row[i].live && key0 + key <= row[i].last;
#pragma unroll
              for (int dt = 0; dt < DT; ++dt) {
                const uint2v v = *(const uint2v*)(tile + key * D + (((2 * dt + (g >> 1)) ^ swizzle<D, COLS>(key)) << 3) + 4 * (g & 1));
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                  const float y = __uint_as_float((r & 1) ? (v[r >> 1] & 0xffff0000u) : (v[r >> 1] << 16));
                  if (seen) O[i][dt][r] = __builtin_fmaf(x, y, O[i][dt][r]);
                }
              }
            }
          }
      } else {
        // ---- O^T += V^T P^T
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const bf16x8 a = value(dt);
#pragma unroll
          for (int i = 0; i < NQ; ++i)
#pragma unroll
            for (int term = TERMS - 1; term >= 0; --term) O[i][dt] = mfma16(a, P[i][term], O[i][dt]);
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // (the tile is read before the next one takes its place)
    }
  };
  run(std::false_type{});
  // a value that is not finite may have come from a key that its row does not see, or from large values times probabilities above one
  {
    float probe = 0.f;
#pragma unroll
    for (int i = 0; i < NQ; ++i)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 4; ++r) probe = row[i].live ? __builtin_fmaf(O[i][dt][r], 0.f, probe) : probe;
    if (__builtin_amdgcn_ballot_w64(probe != 0.f) != 0) run(std::true_type{});
  }

  // ---- the waves' results together: out = sum_w 2^(m_w - top) O_w / sum_w 2^(m_w - top) l_w; each wave a share of the channels
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    l[i] = over_groups(l[i], [](float a, float b) { return a + b; });
    if (g == 0) {
      ms[wave][16 * i + ql] = m[i];
      ls[wave][16 * i + ql] = l[i];
    }
  }
  const int64_t all = (int64_t)p.hq * p.lse_rows;
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    float* mine = (float*)tile;
    if (i > 0) __syncthreads();
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *(float4v*)(mine + (dt * 64 + lane) * 4) = O[i][dt];
    __syncthreads();
    float top = -INFINITY, sum = 0.f, w[NW];
#pragma unroll
    for (int x = 0; x < NW; ++x) top = fmaxf(top, ms[x][16 * i + ql]);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int x = 0; x < NW; ++x) {
      w[x] = __builtin_amdgcn_exp2f(ms[x][16 * i + ql] - ref);
      sum += w[x] * ls[x][16 * i + ql];
    }
    // (a sum of zero: the row sees nothing, or all its scores are -inf and it has no softmax; of a piece, the join tells)
    const float inv = sum > 0.f || sum != sum ? 1.f / sum : !cuts && row[i].last >= 0 ? __builtin_nanf("") : 0.f;
    const float lse2 = sum > 0.f || sum != sum ? ref + __builtin_amdgcn_logf(sum) : -INFINITY;
    const int64_t col = (p.q_off ? (int64_t)q.base : (int64_t)seq_i * p.q_rows) + row[i].token, at = (int64_t)row[i].head * p.lse_rows + col;
    if (row[i].live && g == 0 && wave == 0) {
      if (cuts) p.part[(int64_t)p.nsplit * all * p.d + (int64_t)split * all + at] = lse2;
      else if (p.lse) p.lse[at] = lse2 * LN2;
    }
    T* dst = (T*)const_cast<char*>(p.o.p) + (int64_t)q.seq * p.o.bs + (int64_t)(q.base + row[i].token) * p.o.ts + (int64_t)row[i].head * p.o.hs;
    for (int dt = wave; dt < DT; dt += NW) {
      float4v o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < NW; ++x) {
        const float4v y = *(const float4v*)((const float*)tiles[x] + (dt * 64 + lane) * 4);
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r] += w[x] * y[r];     // (an infinity or NaN stays in the sum, whatever its weight)
      }
      const int c = 16 * dt + 4 * g;
      if (!row[i].live || c >= p.d) continue;
#pragma unroll
      for (int r = 0; r < 4; ++r) o[r] *= inv;
      if (cuts) *(float4v*)(p.part + ((int64_t)split * all + at) * p.d + c) = o;
      else if constexpr (TERMS == 1) *(uint2v*)(dst + c) = uint2v{pack2(o[0], o[1]), pack2(o[2], o[3])};
      else *(float4v*)(dst + c) = o;
    }
  }
}

template <typename T, int D, int NQ>
hipError_t go(const SeqParams& p, Cache8Scales sc, const SeqCut& cut, hipStream_t st) {
  constexpr int NW = CACHE8_FEW_WAVES;
  int64_t blocks = (int64_t)p.slots * p.nsplit * p.hk;
  if (cut.resident && blocks > SEQ_ROUNDS * (int64_t)cut.resident) blocks = SEQ_ROUNDS * (int64_t)cut.resident;
  if (sc.heads_of_row > 1 && blocks < 32 * sc.heads_of_row) sc.heads_of_row = p.d > 64 ? 1 : sc.heads_of_row > 2 && p.d <= 32 ? 4 : 2;   // (too few for every XCD: lines)
  const int64_t f = 8 * sc.heads_of_row;
  const dim3 grid((unsigned)((blocks + f - 1) / f * f));
  if (p.d % 16) hipLaunchKernelGGL((k_cache8_few<T, D, NQ, NW, true>), grid, dim3(64 * NW), 0, st, p, sc, cut);
  else hipLaunchKernelGGL((k_cache8_few<T, D, NQ, NW, false>), grid, dim3(64 * NW), 0, st, p, sc, cut);
  return hipGetLastError();
}

template <typename T>
hipError_t launch(SeqParams p, Cache8Scales sc, const SeqPlan& s, hipStream_t st) {
  sc.heads_of_row = p.k.hs != p.d || p.hk < 2 ? 1 : p.hk < 4 ? 2 : p.hk < 8 ? 4 : 8;
  p.nsplit = s.nsplit;
  p.split_tiles = s.split_tiles;
  p.slots = (int)seq_slots(p.q_off != nullptr, p.q_rows, p.nseq, p.group, s.tile_rows);
  if (p.slots == 0) return hipSuccess;
  const SeqCut cut{s.resident, 1, 32 * CACHE8_FEW_WAVES, s.tile_rows};
  hipError_t e;
  if (s.tile_rows == 16) e = p.d <= 64 ? go<T, 64, 1>(p, sc, cut, st) : go<T, 128, 1>(p, sc, cut, st);
  else e = p.d <= 64 ? go<T, 64, 2>(p, sc, cut, st) : go<T, 128, 2>(p, sc, cut, st);
  if (e != hipSuccess || s.nsplit == 1) return e;
  return join_pieces<T>(p, cut, st);
}

}  // namespace

hipError_t launch_cache8_few(const SeqParams& p, const Cache8Scales& sc, const SeqPlan& s, int dtype, hipStream_t st) {
  return dtype == FREQATTN_BF16 ? launch<uint16_t>(p, sc, s, st) : launch<float>(p, sc, s, st);
}

}  // namespace fa
