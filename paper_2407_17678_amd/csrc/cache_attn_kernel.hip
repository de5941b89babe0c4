// Attention over a paged cache in bf16, 8 or 4 bits (section 4.1): a decode step, or a tree of drafted tokens to each sequence.
//
// o_i = sum_j p_ij v_j / sum_j p_ij, p_ij = exp(scale q_i k_j - max), over the cached tokens that the node's block row of the mask keeps
// and, in a tree, over the node itself and those above it.  All nodes of a sequence share what they read: 4 D T flops to a
// cached token's 2 rows, so that bytes bound it up to T = 64 nodes as long as products are matrix instructions and a row is brought to
// bf16 once.  Hence: a wavefront takes 64 cached tokens at a time for ALL queries of a (sequence, head); nothing of the cache is
// shared between wavefronts.  Scores are formed as keys x queries (16x16x32 MFMA): K comes from memory straight into the layout of the
// first operand (16 rows, four lanes to a row: CacheRows), a lane of the result holds one query, and the probabilities are the second
// operand of the product with V as they stand.  V needs its tokens along the contraction: its rows go through a piece of LDS that is
// the wavefront's own, written as they come and read by the transpose read.
//
// A tree's nodes lie in up to five block rows (64 nodes, blocks of 16).  The blocks that any of them keeps are walked once: row by row,
// each block in the first row that keeps it, with one bit to a row that does.
//
// The units of 64 tokens of a (sequence, head) are shared by num_splits workgroups of four wavefronts; wavefronts merge through LDS,
// splits through a second launch.
#include <hip/hip_runtime.h>

#include "config.h"
#include "kernels.h"
#include "kv_cache.h"
#include "row_blocks.h"
#include "sched_util.h"

namespace s2 {

namespace {

constexpr float kNegInf = -__builtin_inff();
constexpr int kMaxRows = 5;  // block rows that 64 positions can lie in, blocks of 16 tokens

// Wavefronts to a SIMD that the registers are for: accumulators, queries, K and V of a unit on their way, scores.
constexpr int waves_for(int D, int dwords, int NQ) { return NQ * (D / 4 + D / 8 + 16) + 8 * dwords + 48 <= 256 ? 2 : 1; }

template <int D, int FMT, int NQ>
__global__ __launch_bounds__(256, waves_for(D, CacheRows<D, FMT>::kDwords, NQ)) void cache_attn_kernel(const CacheAttnParams p) {
  using Rows = CacheRows<D, FMT>;
  using Tile = ChunkTile<D>;
  constexpr int W = 4, KK = D / 32, FT = D / 16, Q = 16 * NQ;
  constexpr int RS = D + 4;  // floats to a row where wavefronts are summed
  static_assert(16 * RS * 4 <= 32 * Tile::RB, "a tile of sums fits where V was");

  __shared__ __align__(16) uint16_t sh_v[W][32 * Tile::kStride];
  __shared__ float sh_p[W][16][Q];  // probabilities of 16 tokens, where V is taken token by token
  __shared__ float sh_m[W][Q], sh_l[W][Q];

  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int item = blockIdx.x;
  const int bh = item / p.by_splits, split = item - bh * p.num_splits;
  const int b = bh / p.by_heads, h = bh - b * p.heads;
  const int S = p.block_size, sh = p.c.block_shift, T = p.nodes;
  const bool tree = p.parents != nullptr;
  const float cl = p.scale_log2e;

  int L = load_const<int32_t>(p.seq_lens + b);
  L = min(max(L, tree ? 0 : 1), p.max_len);

  // Node `lane`: the nodes above it (bits), its depth, the block row it is in, counted from the first one.
  uint64_t above = 1;
  int depth = 0;
  bool there = lane == 0;
  if (tree) {
    int up = lane < T ? p.parents[(int64_t)b * T + lane] : -2;
    if (up < -1 || up >= lane) up = -2;
    above = (uint64_t)1 << lane;
#pragma unroll
    for (int i = 0; i < 6; ++i) {  // (the chain above a node doubles each time)
      const int from = max(up, 0);
      const uint32_t lo = __shfl((uint32_t)above, from, 64), hi = __shfl((uint32_t)(above >> 32), from, 64);
      const int next = __shfl(up, from, 64);
      if (up >= 0) {
        above |= (uint64_t)hi << 32 | lo;
        up = next;
      }
    }
    depth = __popcll(above) - 1;
    there = up == -1 && L + depth < p.max_len;
  }
  const int row0 = (tree ? L : L - 1) >> sh;
  const int rel = there && tree ? ((L + depth) >> sh) - row0 : 0;
  const uint64_t nodes_there = __ballot(there);
  int n_rows = nodes_there ? 1 : 0;
#pragma unroll
  for (int r = 1; r < kMaxRows; ++r) n_rows += __ballot(rel >= r) != 0;

  // The queries of my column in each tile.
  int rel_q[NQ];
  bool there_q[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    rel_q[n] = __shfl(rel, 16 * n + c, 64);
    there_q[n] = nodes_there >> (16 * n + c) & 1;
  }
  bf16x8 qf[NQ][KK];
  auto load_queries = [&](auto feature) {
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
        qf[n][kk] = there_q[n] ? *reinterpret_cast<const bf16x8*>(p.q + b * p.q_ss + h * p.q_sh + (16 * n + c) * p.q_sn + feature(kk)) : bf16x8{};
  };
  load_queries([&](int kk) { return Rows::feature(kk, g); });

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

  f32x4 s[NQ][4];
  // Scores of 16 tokens.
  auto score = [&](int t, const u32x4 (&k)[KK]) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      s[n][t] = f32x4{};
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) s[n][t] = mfma16(__builtin_bit_cast(bf16x8, k[kk]), qf[n][kk], s[n][t]);
    }
  };
  // Scores (masked ones -inf) to probabilities; the accumulators go along with the maximum.
  auto softmax = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      float mx = kNegInf;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[n][t][e]);
      mx = max_halves(max_rows(mx));
      const float m_new = fmaxf(m_run[n], mx);
      const float mc = m_new == kNegInf ? 0.f : m_new * cl;
      const float alpha = fast_exp2(m_run[n] * cl - mc);  // (-inf before the first token: 0)
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[n][t][e] = fast_exp2(__builtin_fmaf(s[n][t][e], cl, -mc));
          sum += s[n][t][e];
        }
      l_run[n] = l_run[n] * alpha + sum;
      m_run[n] = m_new;
#pragma unroll
      for (int ft = 0; ft < FT; ++ft) acc[n][ft] *= alpha;
    }
  };
  // 32 tokens' V (two pieces) into LDS, and their products.  seen(n, t, e): whether the column's query attends token 4 * g + e of piece t; asked only
  // where `mixed`: then a token that some query does not attend may hold anything, and 0 times that need not be 0.
  auto values = [&](int half, const u32x4 (&v0)[KK], const u32x4 (&v1)[KK], auto feature, bool mixed, auto seen) __attribute__((always_inline)) {
    uint32_t odd = 0;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(v_write + 2 * feature(kk)) = v0[kk];
      *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(v_write + 16 * Tile::RB + 2 * feature(kk)) = v1[kk];
      if (mixed) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          odd |= (v0[kk][e] & 0x7f80u) == 0x7f80u || (v0[kk][e] & 0x7f800000u) == 0x7f800000u || (v1[kk][e] & 0x7f80u) == 0x7f80u ||
                 (v1[kk][e] & 0x7f800000u) == 0x7f800000u;
      }
    }
    wait_lds();
    if (mixed && __any(odd)) {
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            // (as the product takes it; -1: not attended)
            const float x = (float)(__bf16)(t ? s[n][2 * half + 1][e] : s[n][2 * half][e]);
            sh_p[wave][4 * g + e][16 * n + c] = seen(n, 2 * half + t, e) ? x : -1.f;
          }
        wait_lds();
        for (int j = 0; j < 16; ++j)
#pragma unroll
          for (int n = 0; n < NQ; ++n) {
            const float x = sh_p[wave][j][16 * n + c];
#pragma unroll
            for (int ft = 0; ft < FT; ++ft)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint16_t bits = my_v[(16 * t + j) * Tile::kStride + 16 * ft + 4 * g + e];
                const float v = __builtin_bit_cast(float, (uint32_t)bits << 16);
                acc[n][ft][e] = x < 0.f ? acc[n][ft][e] : __builtin_fmaf(x, v, acc[n][ft][e]);
              }
          }
        wait_lds();
      }
      return;
    }
    bf16x8 pf[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const f32x4 a = s[n][2 * half], z = s[n][2 * half + 1];
      pf[n] = __builtin_bit_cast(bf16x8, u32x4{pack2(a[0], a[1]), pack2(a[2], a[3]), pack2(z[0], z[1]), pack2(z[2], z[3])});
    }
#pragma unroll
    for (int ft = 0; ft < FT; ++ft) {
      const bf16x8 vf = __builtin_bit_cast(bf16x8, lds_read_tr2(v_read, v_read, Tile::tr_off(0, ft), Tile::tr_off(0, ft) + 16 * Tile::RB));
#pragma unroll
      for (int n = 0; n < NQ; ++n) acc[n][ft] = mfma16(vf, pf[n], acc[n][ft]);
    }
    asm volatile("" ::: "memory");
  };

  // ---- the cached tokens
  const int32_t* const table = p.c.table + ((int64_t)b * p.heads + h) * p.c.max_blocks;
  int n_missing = 0;
  const int all_rows = (1 << n_rows) - 1;

  // Four pieces of 16 tokens of the list's blocks.
  struct Unit {
    int page[4], skip[4], rows[4], bits[4];
  };
  int r_now = -1, u_now = 0, u_end = 0;
  RowBlocks rb{};
  // The wavefront's next unit with a token to read.
  auto next_unit = [&](Unit& w) {
    for (;;) {
      u_now += W;
      while (u_now >= u_end) {
        if (++r_now >= n_rows) return false;
        rb = row_blocks(p, h, row0 + r_now);
        const int units = ((rb.count << sh) + 63) >> 6;
        const int even = units / p.by_splits, rest = units - even * p.num_splits;
        u_now = even * split + rest * split / p.by_splits + wave;
        u_end = even * (split + 1) + rest * (split + 1) / p.by_splits;
      }
      int any = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int l = 64 * u_now + 16 * i, n = l >> sh, skip = l & (S - 1);
        const bool inside = n < rb.count;
        const int blk = rb.block(inside ? n : 0);
        int rows = inside ? min(max(L - (blk * S + skip), 0), 16) : 0, bits = 1 << r_now;
        if (n_rows > 1 && rows > 0) {
          for (int r = 0; r < n_rows; ++r) {
            if (r == r_now || !row_keeps(p, row_blocks(p, h, row0 + r), h, row0 + r, blk, n)) continue;
            if (r < r_now) rows = 0;  // (read in that row's turn)
            bits |= 1 << r;
          }
        }
        int page = 0;
        if (rows > 0) {
          page = load_const<int32_t>(table + blk);
          if (page < 0 || page >= p.c.num_pages) {
            n_missing += skip == 0;
            rows = 0;
          }
        }
        w.page[i] = page;
        w.skip[i] = skip;
        w.rows[i] = rows;
        w.bits[i] = bits;
        any |= rows;
      }
      if (any) return true;
    }
  };

  typename Rows::Part kr[4], vr[4];
  auto load = [&](const Unit& w, const uint8_t* pool, const uint8_t* scales, typename Rows::Part (&x)[4]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint8_t* const at = pool + w.page[i] * p.c.page + w.skip[i] * p.c.tok;
      const uint8_t* const scale_at = Rows::kScaled ? scales + w.page[i] * p.c.scale_page + w.skip[i] * p.c.scale_tok : nullptr;
      Rows::load(x[i], at, scale_at, w.rows[i], p.c.tok, p.c.scale_tok, c, g);
    }
  };
  auto compute = [&](const Unit& w) __attribute__((always_inline)) {
    bool mixed = false;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      u32x4 k[KK];
      Rows::operands(kr[t], g, k);
      score(t, k);
      mixed |= w.rows[t] > 0 && w.bits[t] != all_rows;
      if (w.rows[t] < 16 || w.bits[t] != all_rows) {
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (4 * g + e >= w.rows[t] || !(w.bits[t] >> rel_q[n] & 1)) s[n][t][e] = kNegInf;
      }
    }
    softmax();
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      u32x4 v0[KK], v1[KK];
      Rows::operands(vr[2 * half], g, v0);
      Rows::operands(vr[2 * half + 1], g, v1);
      values(half, v0, v1, [&](int kk) { return Rows::feature(kk, g); }, mixed,
             [&](int n, int t, int e) { return 4 * g + e < w.rows[t] && (w.bits[t] >> rel_q[n] & 1); });
    }
  };
  {
    Unit w;
    u_now = -W;
    while (next_unit(w)) {
      load(w, p.c.k, p.c.ks, kr);
      load(w, p.c.v, p.c.vs, vr);
      compute(w);
    }
  }
  if (p.missing && lane == 0 && n_missing > 0) atomicAdd(p.missing, n_missing);

  // ---- the drafted ones: one unit, taken by one wavefront of the last split
  if (tree && split == p.num_splits - 1 && wave == W - 1 && nodes_there) {
    uint64_t in_row[kMaxRows];
#pragma unroll
    for (int r = 0; r < kMaxRows; ++r) in_row[r] = __ballot(there && rel == r);
    uint64_t sees[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const uint32_t lo = __shfl((uint32_t)above, 16 * n + c, 64), hi = __shfl((uint32_t)(above >> 32), 16 * n + c, 64);
      sees[n] = (uint64_t)hi << 32 | lo;
    }
    for (int r = 0; r < n_rows; ++r) {
      const RowBlocks row = row_blocks(p, h, row0 + r);
      uint64_t kept = 0;
#pragma unroll
      for (int a = 0; a < kMaxRows; ++a)
        if (a <= r && row_keeps(p, row, h, row0 + r, row0 + a, row.count - 1)) kept |= in_row[a];
#pragma unroll
      for (int n = 0; n < NQ; ++n)
        if (rel_q[n] == r) sees[n] &= kept;
    }
    const uint16_t* const from = p.k_draft + b * p.kv_ss + h * p.kv_sh;
    const int64_t to_v = p.v_draft - p.k_draft;
    auto fetch = [&](int t, int64_t off, u32x4 (&x)[KK]) __attribute__((always_inline)) {
      const bool here = nodes_there >> (16 * t + c) & 1;  // (nobody attends a node that is not there, and it may hold anything)
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
        x[kk] = here ? *reinterpret_cast<const u32x4*>(from + off + (16 * t + c) * p.kv_sn + Rows::feature(kk, g)) : u32x4{};
    };
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      u32x4 k[KK];
      fetch(t, 0, k);
      score(t, k);
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (!(sees[n] >> (16 * t + 4 * g + e) & 1)) s[n][t][e] = kNegInf;
    }
    softmax();
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      u32x4 v0[KK], v1[KK];
      fetch(2 * half, to_v, v0);
      fetch(2 * half + 1, to_v, v1);
      values(half, v0, v1, [&](int kk) { return Rows::feature(kk, g); }, true,
             [&](int n, int t, int e) { return (sees[n] >> (16 * t + 4 * g + e) & 1) != 0; });
    }
  }

  // ---- the wavefronts' sums, 16 queries at a time through where V was
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const float l = sum_groups(l_run[n]);
    if (g == 0) {
      sh_m[wave][16 * n + c] = there_q[n] ? m_run[n] : kNegInf;
      sh_l[wave][16 * n + c] = there_q[n] ? l : 0.f;
    }
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    float m = kNegInf;
#pragma unroll
    for (int w = 0; w < W; ++w) m = fmaxf(m, sh_m[w][16 * n + c]);
    // (no maximum and no sum: no token; scores that are all NaN leave a sum of NaN)
    const float weight = sh_l[wave][16 * n + c] == 0.f ? 0.f : fast_exp2((m_run[n] - m) * cl);
    float* const mine = reinterpret_cast<float*>(my_v) + c * RS + 4 * g;
#pragma unroll
    for (int ft = 0; ft < FT; ++ft)
#pragma unroll
      for (int e = 0; e < 4; ++e) mine[16 * ft + e] = there_q[n] ? acc[n][ft][e] * weight : 0.f;
    __syncthreads();
    constexpr int TPR = D / 8;  // threads to a query, eight features each
    const int i = tid / TPR, d = 8 * (tid % TPR), node = 16 * n + i;
    if (i < 16 && node < T) {
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
      const int64_t row = (int64_t)bh * T + node;
      if (p.num_splits == 1) {
        bf16x8 out;
#pragma unroll
        for (int e = 0; e < 8; ++e) out[e] = (__bf16)(l == 0.f ? 0.f : o[e] / l);
        *reinterpret_cast<bf16x8*>(p.o + b * p.q_ss + h * p.q_sh + node * p.q_sn + d) = out;
        if (d == 0 && p.lse) p.lse[row] = l == 0.f ? kNegInf : mt * p.scale + __logf(l);
      } else {
        float* const to = p.part_acc + (row * p.num_splits + split) * D + d;
#pragma unroll
        for (int e = 0; e < 8; ++e) to[e] = o[e];
        if (d == 0) {
          p.part_ml[(row * p.num_splits + split) * 2] = mt;
          p.part_ml[(row * p.num_splits + split) * 2 + 1] = l;
        }
      }
    }
    __syncthreads();
  }
}

// Merges the splits: D/8 lanes to a row of the result.
template <int D>
__global__ __launch_bounds__(256) void cache_attn_merge_kernel(const CacheAttnParams p) {
  constexpr int TPR = D / 8;
  const int64_t row = (int64_t)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
  const int d = 8 * (threadIdx.x % TPR);
  if (row >= (int64_t)p.nseq * p.heads * p.nodes) return;
  const float* const ml = p.part_ml + row * p.num_splits * 2;
  const float* const part = p.part_acc + row * p.num_splits * D + d;
  float m = kNegInf;
  for (int i = 0; i < p.num_splits; ++i) m = fmaxf(m, ml[2 * i]);
  float l = 0.f, o[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = 0.f;
  for (int i = 0; i < p.num_splits; ++i) {
    if (ml[2 * i + 1] == 0.f) continue;  // no token
    const float weight = fast_exp2((ml[2 * i] - m) * p.scale_log2e);
    l += ml[2 * i + 1] * weight;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] += part[(int64_t)i * D + e] * weight;
  }
  const int64_t bh = row / p.nodes;
  const int node = (int)(row - bh * p.nodes);
  const int64_t b = bh / p.heads, h = bh - b * p.heads;
  bf16x8 out;
#pragma unroll
  for (int e = 0; e < 8; ++e) out[e] = (__bf16)(l == 0.f ? 0.f : o[e] / l);
  *reinterpret_cast<bf16x8*>(p.o + b * p.q_ss + h * p.q_sh + node * p.q_sn + d) = out;
  if (d == 0 && p.lse) p.lse[row] = l == 0.f ? kNegInf : m * p.scale + __logf(l);
}

template <int D, int FMT>
hipError_t launch_nodes(const CacheAttnParams& p, hipStream_t stream) {
  const dim3 grid(p.nseq * p.heads * p.num_splits), block(256);
  if (p.nodes <= 16)
    hipLaunchKernelGGL((cache_attn_kernel<D, FMT, 1>), grid, block, 0, stream, p);
  else if (p.nodes <= 32)
    hipLaunchKernelGGL((cache_attn_kernel<D, FMT, 2>), grid, block, 0, stream, p);
  else
    hipLaunchKernelGGL((cache_attn_kernel<D, FMT, 4>), grid, block, 0, stream, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.num_splits == 1) return e;
  const int64_t rows = (int64_t)p.nseq * p.heads * p.nodes, per = 256 / (D / 8);
  hipLaunchKernelGGL((cache_attn_merge_kernel<D>), dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, stream, p);
  return hipGetLastError();
}

template <int D>
hipError_t launch_format(const CacheAttnParams& p, hipStream_t stream) {
  switch (p.c.format) {
    case S2_KV_BF16: return launch_nodes<D, S2_KV_BF16>(p, stream);
    case S2_KV_MXFP8: return launch_nodes<D, S2_KV_MXFP8>(p, stream);
    default: return launch_nodes<D, S2_KV_MXFP4>(p, stream);
  }
}

}  // namespace

hipError_t launch_cache_attn(const CacheAttnParams& params, hipStream_t stream) {
  CacheAttnParams p = params;
  p.by_heads = fast_div(p.heads);
  p.by_splits = fast_div(p.num_splits);
  p.by_stride = fast_div(p.stride > 0 ? p.stride : 1);
  return p.c.head_dim == 128 ? launch_format<128>(p, stream) : launch_format<64>(p, stream);
}

}  // namespace s2
