// Attention of up to 32 rows of a chunk over a paged cache, by a workgroup of 256 threads (see cache_chunk_kernel.hip for the mathematics): for chunks of so few rows,
// and for tiles of longer ones that have no more.
#pragma once

#include <type_traits>

#include "cache_chunk.h"

namespace s2 {

// Up to 32 queries of one (sequence, head), one split of what they attend: nothing of the cache is shared between the wavefronts of a workgroup.  Two of them take a unit, 32 tokens
// each, against all queries: K comes from memory straight into the layout of the first operand, V through a piece of LDS of the wavefront's own (as in
// cache_attn_kernel.hip; one wavefront's queries against units that all fetch leave three of four idle: 64 sequences of 1 to 12 rows over e4m3 244 us,
// so 222, 5.3 TB/s).
template <int D, int NQ, bool SMALL>
struct ChunkFewShared {
  static constexpr int W = 4, FT = D / 16;
  alignas(16) uint16_t v[W][32 * ChunkTile<D>::kStride];
  u32x2 pieces[W][ChunkWalk<SMALL>::kRing];
  ChunkScope scope;
  float m[W][16 * NQ], l[W][16 * NQ];
  uint32_t odd[NQ * FT / 4 * 64];  // (count_odd)
  uint32_t any_odd;
};
// (p: the kernel's parameters; x, r: its tile, of 1 to 16 * NQ rows)
template <int D, int FMT, int NQ, bool SMALL>
__device__ __forceinline__ void chunk_few(const CacheChunkParams& p, const ChunkTileAt& x, const ChunkRows& r, int h, int split, ChunkFewShared<D, NQ, SMALL>& sh) {
  using Rows = CacheRows<D, FMT>;
  using Tile = ChunkTile<D>;
  using Pieces = ChunkWalk<SMALL>;
  constexpr int W = 4, KK = D / 32, FT = D / 16;
  constexpr int RS = D + 4;  // floats to a row where wavefronts are summed
  static_assert(16 * RS * 4 <= 32 * Tile::RB, "a tile of sums fits where V was");

  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const float cl = p.scale_log2e;

  ChunkQuery q[NQ];
  bf16x8 qf[NQ][KK];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    q[n] = chunk_query(p, x, r, 16 * n + c);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
      qf[n][kk] = q[n].there ? *reinterpret_cast<const bf16x8*>(p.q + (x.row + 16 * n + c) * p.q_sr + h * p.q_sh + Rows::feature(kk, g)) : bf16x8{};
  }
  for (int i = tid; i < NQ * FT / 4 * 64; i += 64 * W) sh.odd[i] = 0;
  if (tid == 0) {
    sh.any_odd = 0;
    sh.scope.init(p, x, r, h, split);
  }
  __syncthreads();

  f32x4 acc[NQ][FT];
  float m_run[NQ], l_run[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m_run[n] = kNegInf;
    l_run[n] = 0.f;
#pragma unroll
    for (int ft = 0; ft < FT; ++ft) acc[n][ft] = f32x4{};
  }

  uint16_t* const my_v = sh.v[wave];
  const uint32_t v_write = lds_addr(my_v) + c * Tile::RB, v_read = lds_addr(my_v) + Tile::tr_lane(lane);
  const int half = wave & 1;
  Pieces walk(sh.scope, r.n_rows, wave, sh.pieces[wave], q[0], q[NQ - 1], wave >> 1, W / 2);

  typename Rows::Part kr[2], vr[2];
  auto load = [&](auto is_v, const ChunkUnit (&w)[2], typename Rows::Part (&to)[2]) __attribute__((always_inline)) {
    constexpr bool V = decltype(is_v)::value;
#pragma unroll
    for (int t = 0; t < 2; ++t)
      Rows::load(to[t], (V ? p.c.v : p.c.k) + w[t].off, Rows::kScaled ? (V ? p.c.vs : p.c.ks) + w[t].scale_off : nullptr, w[t].rows, p.c.tok, p.c.scale_tok,
                 (SMALL ? 0 : 32 * half + 16 * t) + c, g);
  };
  constexpr std::false_type kK{};
  constexpr std::true_type kV{};
  f32x4 s[NQ][2];
  uint32_t seen[NQ];
  auto scores = [&](bool some, int unit) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      u32x4 k[KK];
      Rows::operands(kr[t], g, k);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
#pragma unroll
        for (int n = 0; n < NQ; ++n) s[n][t] = mfma16(__builtin_bit_cast(bf16x8, k[kk]), qf[n][kk], kk ? s[n][t] : f32x4{});
    }
    if (some) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        seen[n] = (uint32_t)(chunk_seen<SMALL>(walk, unit, q[n].rel, q[n].pos) >> (32 * half));
#pragma unroll
        for (int t = 0; t < 2; ++t) mask_scores(s[n][t], seen[n], t, g);
      }
    }
  };
  auto sums = [&](bool some) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      float mx = kNegInf;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[n][t][e]);
      mx = max_halves(max_rows(mx));
      const float m_new = fmaxf(m_run[n], mx);
      const float mc = m_new == kNegInf ? 0.f : m_new * cl;
      if (__any(m_new > m_run[n])) {
        const float alpha = m_new > m_run[n] ? fast_exp2(m_run[n] * cl - mc) : 1.f;  // (see cache_attn_kernel.hip)
        l_run[n] *= alpha;
        m_run[n] = m_new;
#pragma unroll
        for (int ft = 0; ft < FT; ++ft) acc[n][ft] *= alpha;
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[n][t][e] = fast_exp2(__builtin_fmaf(s[n][t][e], cl, -mc));
          l_run[n] += s[n][t][e];
        }
    }
    u32x4 v[2][KK];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      Rows::operands(vr[i], g, v[i]);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
        *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(v_write + 16 * i * Tile::RB + 2 * Rows::feature(kk, g)) = v[i][kk];
    }
    wait_lds();
    bool odd = false;
    if (some) {
      asm volatile("");  // (else looked for in every unit)
      odd = __any((odd_bits(v[0]) | odd_bits(v[1])) != 0);
    }
    if (odd) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) count_odd<D>(v_read, seen[n], sh.odd + n * FT / 4 * 64, &sh.any_odd, lane);
      wait_lds();
      clean_words(reinterpret_cast<uint32_t*>(my_v), 32 * Tile::RB / 4, lane);
      wait_lds();
    }
    bf16x8 pf[NQ], pr[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) two_terms(s[n][0], s[n][1], pf[n], pr[n]);
#pragma unroll
    for (int ft = 0; ft < FT; ++ft) {
      const bf16x8 vf = __builtin_bit_cast(bf16x8, lds_read_tr2(v_read, v_read, Tile::tr_off(0, ft), Tile::tr_off(0, ft) + 16 * Tile::RB));
#pragma unroll
      for (int n = 0; n < NQ; ++n) acc[n][ft] = mfma16(vf, pf[n], mfma16(vf, pr[n], acc[n][ft]));
    }
    asm volatile("" ::: "memory");
  };
  if (walk.find()) {
    ChunkUnit w[2];
    walk.template take<2>(0, 2 * half, w);
    load(kK, w, kr);
    load(kV, w, vr);
    for (int n = 0;; ++n) {
      ChunkUnit next[2] = {};
      const bool more = walk.find();
      if (more) walk.template take<2>(n + 1, 2 * half, next);
      // the next unit's K goes into the registers that the scores have freed, its V into those that the sums free
      scores(w[0].some(), n);
      __builtin_amdgcn_sched_barrier(0);
      load(kK, next, kr);
      __builtin_amdgcn_sched_barrier(0);
      sums(w[0].some());
      __builtin_amdgcn_sched_barrier(0);
      load(kV, next, vr);
      if (!more) break;
      w[0] = next[0];
      w[1] = next[1];
    }
  }
  const CacheChunkParams& pe = chunk_params();
  // (both halves have walked the same units)
  if (pe.missing && lane == 0 && half == 0 && walk.n_missing > 0) atomicAdd(pe.missing, walk.n_missing);

  // the wavefronts' sums, a tile of queries at a time, through where V was
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    l_run[n] = sum_groups(l_run[n]);
    if (g == 0) {
      sh.m[wave][16 * n + c] = q[n].there ? m_run[n] : kNegInf;
      sh.l[wave][16 * n + c] = q[n].there ? l_run[n] : 0.f;
    }
  }
  constexpr int TPR = D / 8;  // threads to a query, eight features each
  const int i = tid / TPR, d = 8 * (tid % TPR);
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    __syncthreads();
    float m = kNegInf;
#pragma unroll
    for (int w = 0; w < W; ++w) m = fmaxf(m, sh.m[w][16 * n + c]);
    // (no maximum and no sum: no token; scores that are all NaN leave a sum of NaN)
    const float weight = sh.l[wave][16 * n + c] == 0.f ? 0.f : fast_exp2((m_run[n] - m) * cl);
#pragma unroll
    for (int ft = 0; ft < FT; ++ft) acc[n][ft] *= weight;
    float* const mine = reinterpret_cast<float*>(my_v) + c * RS + 4 * g;
#pragma unroll
    for (int ft = 0; ft < FT; ++ft) *reinterpret_cast<f32x4*>(mine + 16 * ft) = q[n].there ? acc[n][ft] : f32x4{};
    // (not before the weight: it may be another wavefront that the query has its tokens of)
    if (sh.any_odd && wave == 0 && q[n].there) add_odd<D>(mine, sh.odd + n * FT / 4 * 64, lane);
    __syncthreads();
    const int row = 16 * n + i;
    if (i >= 16 || row >= x.rows) continue;
    float mt = kNegInf, l = 0.f, o[8];
#pragma unroll
    for (int w = 0; w < W; ++w) mt = fmaxf(mt, sh.m[w][row]);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      if (sh.l[w][row] != 0.f) l += sh.l[w][row] * fast_exp2((sh.m[w][row] - mt) * cl);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] += reinterpret_cast<const float*>(sh.v[w])[i * RS + d + e];
    }
    put_chunk_row<D>(pe, x, h, row, split, d, o, mt, l);
  }
}

}  // namespace s2
