// Attention of a tree of drafted tokens to each sequence over a paged cache in bf16, 8 or 4 bits (section 4.1).
//
// o_i = sum_j p_ij v_j / sum_j p_ij, p_ij = exp(scale q_i k_j - max), over the cached tokens that the node's block row of the mask keeps
// and over the node itself and those above it.  All nodes of a sequence share what they read: 4 D T flops to a
// cached token's 2 rows, so that bytes bound it as long as products are matrix instructions and a row is brought to bf16 once.
//
// This kernel is for up to 32 queries, one or two tiles of the 16x16x32 MFMA.  A wavefront takes 32 cached tokens at a time for all queries of a
// (sequence, head), and nothing of the cache is shared between wavefronts: no barrier, four streams to a workgroup.  Scores are
// formed as keys x queries: K comes from memory straight into the layout of the first operand (16 rows, four lanes to a row: CacheRows), a
// lane of the result holds one query, and the probabilities are the second operand of the product with V as they stand.  V needs its tokens along the
// contraction: its rows go through a piece of LDS that is the wavefront's own, written as they come and read by the transpose read.  (With K and V
// shared by a workgroup in LDS, as for more queries, 24 nodes of 64 sequences over e4m3 took 251 us instead of 242, 20 of 8 sequences 27.4 instead of 23.1, P in one term.)
//
// A tree's nodes lie in up to five block rows (64 nodes, blocks of 16).  The blocks that any of them keeps are walked once: row by row,
// each block in the first row that keeps it, with one bit to a row that does.
//
// The units of 64 tokens of a (sequence, head) are shared by num_splits workgroups of four wavefronts, two of them to a unit; wavefronts merge through
// LDS, splits through a second launch.
//
// The cache's bytes bound it: 4 nodes of 64 sequences over bf16 (32 heads of 31 to 47 blocks of 64 tokens, D = 128) 403 us, 5.7 TB/s; 24 nodes over e4m3
// 246 us, 4.9 TB/s; 12 over e2m1 136 us, 4.6 TB/s.  8 nodes of one sequence of 32768 tokens take 16 us, of which the bytes are 8.  Loads two units ahead
// instead of one gain nothing (the registers that they take cost 2 to 10 %), nor does V in LDS before the softmax.
#include <hip/hip_runtime.h>

#include "cache_attn.h"
#include "config.h"

namespace s2 {

namespace {

// Wavefronts to a SIMD that the registers are limited for: as many as fit without spilling (D = 128: 140 over
// e2m1, 151 over e4m3, 176 over bf16, and with two tiles 206, 217 and 238).
constexpr int waves_for(int D, int FMT, int NQ) { return NQ == 2 ? (D == 64 ? 3 : 2) : D == 64 ? 4 : FMT == S2_KV_BF16 ? 2 : 3; }

// SMALL: blocks of 16 or 32 tokens, so that a unit of 64 is gathered from four or two of the list's blocks; else it is a piece of one block.
template <int D, int FMT, int NQ, bool SMALL>
__global__ __launch_bounds__(256, waves_for(D, FMT, NQ)) void cache_attn_kernel(const CacheAttnParams p) {
  using Rows = CacheRows<D, FMT>;
  using Tile = ChunkTile<D>;
  constexpr int W = 4, KK = D / 32, FT = D / 16;
  constexpr int RS = D + 4;  // floats to a row where wavefronts are summed
  static_assert(16 * RS * 4 <= 32 * Tile::RB, "a tile of sums fits where V was");

  __shared__ __align__(16) uint16_t sh_v[W][32 * Tile::kStride];
  __shared__ float sh_m[W][16 * NQ], sh_l[W][16 * NQ];
  __shared__ uint32_t sh_odd[NQ * FT / 4 * 64];  // (count_odd)
  __shared__ uint32_t sh_any_odd;

  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int item = blockIdx.x;
  const int bh = item / p.by_splits, split = item - bh * p.num_splits;
  const int b = bh / p.by_heads, h = bh - b * p.heads;
  const float cl = p.scale_log2e;

  int L = load_const<int32_t>(p.seq_lens + b);
  L = min(max(L, 0), p.max_len);
  const Nodes nodes = nodes_of(p, b, L, lane);
  // the queries of my column
  int rel_q[NQ];
  bool there_q[NQ];
  bf16x8 qf[NQ][KK];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int node = 16 * n + c;
    rel_q[n] = __shfl(nodes.rel, node, 64);
    there_q[n] = nodes.all >> node & 1;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
      qf[n][kk] = there_q[n] ? *reinterpret_cast<const bf16x8*>(p.q + b * p.q_ss + h * p.q_sh + node * p.q_sn + Rows::feature(kk, g)) : bf16x8{};
  }

  for (int i = tid; i < NQ * FT / 4 * 64; i += 64 * W) sh_odd[i] = 0;
  if (tid == 0) sh_any_odd = 0;
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

  uint16_t* const my_v = sh_v[wave];
  const uint32_t v_write = lds_addr(my_v) + c * Tile::RB, v_read = lds_addr(my_v) + Tile::tr_lane(lane);
  // two wavefronts to a unit of 64 tokens, half of it each
  const int half = wave & 1;
  Walk<SMALL> walk(b, h, L, nodes, split, wave >> 1, W / 2, 2 * half);

  typename Rows::Part kr[2], vr[2];
  auto load = [&](auto is_v, const Unit<SMALL>& w, typename Rows::Part (&x)[2]) __attribute__((always_inline)) {
    constexpr bool V = decltype(is_v)::value;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int page = w.my_page[t], skip = Unit<SMALL>::skip(w.my_info[t]);
      const uint8_t* const at = (V ? p.c.v : p.c.k) + page * p.c.page + skip * p.c.tok;
      const uint8_t* const scale_at = Rows::kScaled ? (V ? p.c.vs : p.c.ks) + page * p.c.scale_page + skip * p.c.scale_tok : nullptr;
      Rows::load(x[t], at, scale_at, Unit<SMALL>::rows(w.my_info[t]), p.c.tok, p.c.scale_tok, (SMALL ? 0 : 32 * half + 16 * t) + c, g);
    }
  };
  constexpr std::false_type kK{};
  constexpr std::true_type kV{};
  constexpr std::false_type kCached{};
  constexpr std::true_type kDrafts{};
  // (DRAFTS: the unit of drafted tokens, fetched where it is used)
  auto operands = [&](auto is_v, auto drafts, int t, const typename Rows::Part& x, u32x4 (&out)[KK]) __attribute__((always_inline)) {
    if constexpr (decltype(drafts)::value)
      draft_rows<Rows, decltype(is_v)::value>(nodes.all, b, h, t, c, g, out);
    else
      Rows::operands(x, g, out);
  };

  f32x4 s[NQ][2];
  uint32_t seen[NQ];
  auto scores = [&](auto drafts, bool some, auto see) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      u32x4 k[KK];
      operands(kK, drafts, t, kr[t], k);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
#pragma unroll
        for (int n = 0; n < NQ; ++n) s[n][t] = mfma16(__builtin_bit_cast(bf16x8, k[kk]), qf[n][kk], kk ? s[n][t] : f32x4{});
    }
    if (some) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        seen[n] = (uint32_t)(see(n) >> (32 * half));
#pragma unroll
        for (int t = 0; t < 2; ++t) mask_scores(s[n][t], seen[n], t, g);
      }
    }
  };
  auto sums = [&](auto drafts, bool mixed) __attribute__((always_inline)) {
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
        // (0 before the first token; where the maximum stays exactly 1, which the difference of the two roundings does not give: a query's result
        // is not to depend on whether another one's maximum has moved)
        const float alpha = m_new > m_run[n] ? fast_exp2(m_run[n] * cl - mc) : 1.f;
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
      operands(kV, drafts, i, vr[i], v[i]);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
        *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(v_write + 16 * i * Tile::RB + 2 * Rows::feature(kk, g)) = v[i][kk];
    }
    wait_lds();
    bool odd = false;
    if (mixed) {
      asm volatile("");  // (else looked for in every unit)
      odd = __any((odd_bits(v[0]) | odd_bits(v[1])) != 0);
    }
    if (odd) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) count_odd<D>(v_read, seen[n], sh_odd + n * FT / 4 * 64, &sh_any_odd, lane);
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
  {
    Unit<SMALL> w;
    if (walk.template next<false>(p, w)) {
      load(kK, w, kr);
      load(kV, w, vr);
      for (bool more = true; more;) {
        Unit<SMALL> next;
        more = walk.template next<true>(p, next);
        // the next unit's K goes into the registers that the scores have freed, its V into those that the sums free
        scores(kCached, w.some, [&](int n) { return unit_seen(w, rel_q[n]); });
        __builtin_amdgcn_sched_barrier(0);
        load(kK, next, kr);
        __builtin_amdgcn_sched_barrier(0);
        sums(kCached, w.mixed);
        __builtin_amdgcn_sched_barrier(0);
        load(kV, next, vr);
        w = next;
      }
    }
  }
  // the drafted tokens, 32 at most: the first half of a unit of their own
  if (split == p.num_splits - 1 && wave == 0 && nodes.all) {
    scores(kDrafts, true, [&](int n) { return drafts_seen(nodes, h, 16 * n + c, rel_q[n]); });
    sums(kDrafts, true);
  }
  const CacheAttnParams& pe = params_in_memory();
  // (both halves have walked the same units)
  if (pe.missing && lane == 0 && half == 0 && walk.n_missing > 0) atomicAdd(pe.missing, walk.n_missing);

  // the wavefronts' sums, a tile of queries at a time, through where V was
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    l_run[n] = sum_groups(l_run[n]);
    if (g == 0) {
      sh_m[wave][16 * n + c] = there_q[n] ? m_run[n] : kNegInf;
      sh_l[wave][16 * n + c] = there_q[n] ? l_run[n] : 0.f;
    }
  }
  constexpr int TPR = D / 8;  // threads to a query, eight features each
  const int i = tid / TPR, d = 8 * (tid % TPR);
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    __syncthreads();
    float m = kNegInf;
#pragma unroll
    for (int w = 0; w < W; ++w) m = fmaxf(m, sh_m[w][16 * n + c]);
    // (no maximum and no sum: no token; scores that are all NaN leave a sum of NaN)
    const float weight = sh_l[wave][16 * n + c] == 0.f ? 0.f : fast_exp2((m_run[n] - m) * cl);
#pragma unroll
    for (int ft = 0; ft < FT; ++ft) acc[n][ft] *= weight;
    float* const mine = reinterpret_cast<float*>(my_v) + c * RS + 4 * g;
#pragma unroll
    for (int ft = 0; ft < FT; ++ft) *reinterpret_cast<f32x4*>(mine + 16 * ft) = there_q[n] ? acc[n][ft] : f32x4{};
    // (not before the weight: it may be another wavefront that the query has its tokens of)
    if (sh_any_odd && wave == 0 && there_q[n]) add_odd<D>(mine, sh_odd + n * FT / 4 * 64, lane);
    __syncthreads();
    const int node = 16 * n + i;
    if (i >= 16 || node >= pe.nodes) continue;
    float mt = kNegInf, l = 0.f, o[8];
#pragma unroll
    for (int w = 0; w < W; ++w) mt = fmaxf(mt, sh_m[w][node]);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      if (sh_l[w][node] != 0.f) l += sh_l[w][node] * fast_exp2((sh_m[w][node] - mt) * cl);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] += reinterpret_cast<const float*>(sh_v[w])[i * RS + d + e];
    }
    put_result<D>(pe, b, h, node, split, d, o, mt, l);
  }
}

// Merges the splits, a wavefront to a row of the result: lane i holds the weight of split i, groups of D/4 lanes add up the splits of their own, four
// of them requested at a time together with the (max, sum) pairs.
template <int D>
__global__ __launch_bounds__(256) void cache_attn_merge_kernel(const CacheAttnParams p) {
  constexpr int LPR = D / 4, NG = 64 / LPR, NP = 4;
  const int lane = threadIdx.x & 63, g = lane / LPR, c = lane % LPR, n = p.num_splits;
  const int64_t row = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= (int64_t)p.nseq * p.heads * p.nodes) return;
  const float* const ml = p.part_ml + row * n * 2;
  const f32x4* const part = reinterpret_cast<const f32x4*>(p.part_acc) + row * n * LPR + c;
  f32x4 x[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) x[i] = part[(int64_t)min(g + NG * i, n - 1) * LPR];
  const float ms = lane < n ? ml[2 * lane] : kNegInf, ls = lane < n ? ml[2 * lane + 1] : 0.f;
  float m = ms;
  m = fmaxf(m, of_neighbour<1>(m));
  m = fmaxf(m, of_neighbour<2>(m));
  m = fmaxf(m, of_neighbour<4>(m));
  m = max_halves(max_rows(fmaxf(m, of_neighbour<8>(m))));
  const float weight = ls == 0.f ? 0.f : fast_exp2((ms - m) * p.scale_log2e);  // (no sum: no token)
  float l = ls * weight;
  l += of_neighbour<1>(l);
  l += of_neighbour<2>(l);
  l += of_neighbour<4>(l);
  l += of_neighbour<8>(l);
  l = sum_halves(sum_rows(l));
  f32x4 a = f32x4{};
  for (int s0 = 0;;) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int s = s0 + g + NG * i;
      const float of = __shfl(weight, s & 63, 64);
      if (s < n) a += x[i] * of;
    }
    s0 += NG * NP;
    if (s0 >= n) break;
#pragma unroll
    for (int i = 0; i < NP; ++i) x[i] = part[(int64_t)min(s0 + g + NG * i, n - 1) * LPR];
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float y = a[e];
    if (LPR == 16) y = sum_rows(y);
    a[e] = sum_halves(y);
  }
  if (lane >= LPR) return;
  const int64_t bh = row / p.nodes;
  const int node = (int)(row - bh * p.nodes);
  const int64_t b = bh / p.heads, h = bh - b * p.heads;
  bf16x4 out;
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = (__bf16)(l == 0.f ? 0.f : a[e] / l);
  *reinterpret_cast<bf16x4*>(p.o + b * p.q_ss + h * p.q_sh + node * p.q_sn + 4 * c) = out;
  if (lane == 0 && p.lse) p.lse[row] = l == 0.f ? kNegInf : m * p.scale + __logf(l);
}

template <int D, int FMT, int NQ>
void launch_blocks(const CacheAttnParams& p, hipStream_t stream) {
  const dim3 grid(p.nseq * p.heads * p.num_splits), block(256);
  if (p.block_size < 64)
    hipLaunchKernelGGL((cache_attn_kernel<D, FMT, NQ, true>), grid, block, 0, stream, p);
  else
    hipLaunchKernelGGL((cache_attn_kernel<D, FMT, NQ, false>), grid, block, 0, stream, p);
}

template <int D, int FMT>
void launch_tiles(const CacheAttnParams& p, hipStream_t stream) {
  if (p.nodes <= 16)
    launch_blocks<D, FMT, 1>(p, stream);
  else
    launch_blocks<D, FMT, 2>(p, stream);
}

template <int D>
hipError_t launch_dim(const CacheAttnParams& p, hipStream_t stream) {
  hipError_t e;
  if (!p.parents) {
    e = launch_cache_decode(p, stream);
  } else if (p.nodes > 32) {
    e = launch_cache_attn_shared(p, stream);
  } else {
    switch (p.c.format) {
      case S2_KV_BF16: launch_tiles<D, S2_KV_BF16>(p, stream); break;
      case S2_KV_MXFP8: launch_tiles<D, S2_KV_MXFP8>(p, stream); break;
      default: launch_tiles<D, S2_KV_MXFP4>(p, stream); break;
    }
    e = hipGetLastError();
  }
  if (e != hipSuccess || p.num_splits == 1) return e;
  const int64_t rows = (int64_t)p.nseq * p.heads * p.nodes;
  hipLaunchKernelGGL((cache_attn_merge_kernel<D>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_attn(const CacheAttnParams& params, hipStream_t stream) {
  CacheAttnParams p = params;
  p.by_heads = fast_div(p.heads);
  p.by_splits = fast_div(p.num_splits);
  p.by_stride = fast_div(p.stride > 0 ? p.stride : 1);
  return p.c.head_dim == 128 ? launch_dim<128>(p, stream) : launch_dim<64>(p, stream);
}

}  // namespace s2
