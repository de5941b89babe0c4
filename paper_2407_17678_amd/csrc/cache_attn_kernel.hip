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

// Wavefronts to a SIMD: two while accumulators, scores, queries and a unit of K and of V on their way fit 256 registers.
constexpr int waves_for(int D, int NQ) { return NQ == 1 || (NQ == 2 && D == 64) ? 2 : 1; }

// SMALL: blocks of 16 or 32 tokens, so that a unit of 64 is gathered from four or two of the list's blocks; else it is a piece of one block.
template <int D, int FMT, int NQ, bool SMALL>
__global__ __launch_bounds__(256, waves_for(D, NQ)) void cache_attn_kernel(const CacheAttnParams p) {
  using Rows = CacheRows<D, FMT>;
  using Tile = ChunkTile<D>;
  constexpr int W = 4, KK = D / 32, FT = D / 16, Q = 16 * NQ;
  constexpr int RS = D + 4;  // floats to a row where wavefronts are summed
  // With 64 queries their operands are read from LDS, one by one for a whole unit's K; with fewer they stay in registers.
  constexpr bool kQueriesInLds = NQ == 4;
  constexpr int kGroup = kQueriesInLds ? 4 : 1;  // pieces of K that are operands at the same time
  static_assert(16 * RS * 4 <= 32 * Tile::RB, "a tile of sums fits where V was");

  __shared__ __align__(16) uint16_t sh_v[W][32 * Tile::kStride];
  __shared__ u32x4 sh_q[kQueriesInLds ? NQ * KK * 64 : 1];
  __shared__ float sh_m[W][Q], sh_l[W][Q];
  // Infinities and NaN of V that were taken out of the products (values(), below): bits of [query tile][feature tile][lane], a byte to a feature.
  __shared__ uint32_t sh_odd[NQ * FT * 64];
  __shared__ uint32_t sh_any_odd;

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
  for (int i = tid; i < NQ * FT * 64; i += 64 * W) sh_odd[i] = 0;
  if (tid == 0) sh_any_odd = 0;
  bf16x8 qf[kQueriesInLds ? 1 : NQ][KK];
#pragma unroll
  for (int n = 0; n < NQ; ++n)
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      if (kQueriesInLds && (n * KK + kk) % W != wave) continue;
      const bf16x8 x = there_q[n] ? *reinterpret_cast<const bf16x8*>(p.q + b * p.q_ss + h * p.q_sh + (16 * n + c) * p.q_sn + Rows::feature(kk, g)) : bf16x8{};
      if constexpr (kQueriesInLds)
        sh_q[(n * KK + kk) * 64 + lane] = __builtin_bit_cast(u32x4, x);
      else
        qf[n][kk] = x;
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

  uint16_t* const my_v = sh_v[wave];
  const uint32_t v_write = lds_addr(my_v) + c * Tile::RB, v_read = lds_addr(my_v) + Tile::tr_lane(lane);

  f32x4 s[NQ][4];
  // Scores of the pieces t0 .. t0 + kGroup - 1.
  auto score = [&](int t0, const u32x4 (&k)[kGroup][KK]) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        bf16x8 q;
        if constexpr (kQueriesInLds)
          q = __builtin_bit_cast(bf16x8, sh_q[(n * KK + kk) * 64 + lane]);
        else
          q = qf[n][kk];
#pragma unroll
        for (int i = 0; i < kGroup; ++i) s[n][t0 + i] = mfma16(__builtin_bit_cast(bf16x8, k[i][kk]), q, kk ? s[n][t0 + i] : f32x4{});
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
      if (__any(m_new > m_run[n])) {
        const float alpha = fast_exp2(m_run[n] * cl - mc);  // (-inf before the first token: 0)
        l_run[n] *= alpha;
        m_run[n] = m_new;
#pragma unroll
        for (int ft = 0; ft < FT; ++ft) acc[n][ft] *= alpha;
      }
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[n][t][e] = fast_exp2(__builtin_fmaf(s[n][t][e], cl, -mc));
          sum += s[n][t][e];
        }
      l_run[n] += sum;
    }
  };
  auto write_v = [&](int piece, const u32x4 (&v)[KK]) __attribute__((always_inline)) {
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
      *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(v_write + 16 * piece * Tile::RB + 2 * Rows::feature(kk, g)) = v[kk];
  };
  // 32 tokens' V (two pieces) into LDS, and their products.  odd: there are infinities or NaN among them (asked only where some query does not attend some
  // token: that may hold anything, and 0 times it need not be 0).  They are then taken out, and which of them a query attends is found by products of ones
  // and zeros and kept until the end.
  auto values = [&](int half, const u32x4 (&v)[2][KK], bool odd, const uint64_t (&seen)[NQ]) __attribute__((always_inline)) {
    write_v(0, v[0]);
    write_v(1, v[1]);
    wait_lds();
    if (odd) {
      uint32_t* const words = reinterpret_cast<uint32_t*>(my_v);
#pragma unroll 1
      for (int kind = 0; kind < 3; ++kind) {  // infinity, minus infinity, NaN
        auto ones = [&](uint32_t x) { return (kind == 0 ? x == 0x7f80u : kind == 1 ? x == 0xff80u : (x & 0x7fffu) > 0x7f80u) ? 0x3f80u : 0u; };
#pragma unroll 1
        for (int ft = 0; ft < FT; ++ft) {
          u32x4 vf = lds_read_tr2(v_read + 32 * ft, v_read + 32 * ft, 0, 16 * Tile::RB);
#pragma unroll
          for (int e = 0; e < 4; ++e) vf[e] = ones(vf[e] & 0xffffu) | ones(vf[e] >> 16) << 16;
#pragma unroll
          for (int n = 0; n < NQ; ++n) {
            const uint32_t mine = (uint32_t)(seen[n] >> (32 * half)) >> (4 * g);  // tokens 4 g .. and 16 + 4 g ..
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = ((mine >> (16 * (e / 2) + 2 * (e % 2))) & 1) * 0x3f80u + ((mine >> (16 * (e / 2) + 2 * (e % 2) + 1)) & 1) * 0x3f800000u;
            const f32x4 count = mfma16(__builtin_bit_cast(bf16x8, vf), __builtin_bit_cast(bf16x8, w), f32x4{});
            uint32_t found = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) found |= (count[e] > 0.f ? 1u : 0u) << (8 * e + kind);
            if (found) {
              atomicOr(&sh_odd[(n * FT + ft) * 64 + lane], found);
              sh_any_odd = 1;
            }
          }
        }
      }
      wait_lds();
#pragma unroll 1
      for (int i = lane; i < 32 * Tile::RB / 4; i += 64) {
        const uint32_t x = words[i];
        words[i] = ((x & 0x7f80u) == 0x7f80u ? 0u : x & 0xffffu) | ((x & 0x7f800000u) == 0x7f800000u ? 0u : x & 0xffff0000u);
      }
      wait_lds();
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

  // 64 tokens: of one block, or (SMALL) four pieces of 16 of the list's blocks; or the drafted ones.
  constexpr int NB = SMALL ? 4 : 1, kTokens = 64 / NB;
  struct Unit {
    int page[NB], skip[NB], rows[NB], bits[NB];
    bool drafts;
  };
  int r_now = -1, u_now = -W, u_end = 0;
  RowBlocks rb{};
  bool drafts_left = tree && split == p.num_splits - 1 && wave == W - 1 && nodes_there;
  // The wavefront's next unit with a token to read.
  auto next_unit = [&](Unit& w) __attribute__((always_inline)) {
    w.drafts = false;
    for (;;) {
      u_now += W;
      while (u_now >= u_end) {
        if (r_now + 1 >= n_rows) {
          if (!drafts_left) return false;
          drafts_left = false;
          w.drafts = true;
          return true;
        }
        ++r_now;
        rb = row_blocks(p, h, row0 + r_now);
        const int units = ((rb.count << sh) + 63) >> 6;
        const int even = units / p.by_splits, rest = units - even * p.num_splits;
        u_now = even * split + rest * split / p.by_splits + wave;
        u_end = even * (split + 1) + rest * (split + 1) / p.by_splits;
      }
      int any = 0;
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int l = 64 * u_now + 16 * i, n = l >> sh, skip = l & (S - 1);
        const bool inside = !SMALL || n < rb.count;
        const int blk = rb.block(inside ? n : 0);
        int rows = inside ? min(max(L - (blk * S + skip), 0), kTokens) : 0, bits = 1 << r_now;
        if (n_rows > 1 && rows > 0) {
#pragma unroll 1
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

  // What a node's row i keeps of the nodes above it and itself, for the query of my column.
  auto drafts_seen = [&](uint64_t (&seen)[NQ]) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const uint32_t lo = __shfl((uint32_t)above, 16 * n + c, 64), hi = __shfl((uint32_t)(above >> 32), 16 * n + c, 64);
      seen[n] = (uint64_t)hi << 32 | lo;
    }
    if (n_rows == 1) return;
#pragma unroll 1
    for (int r = 0; r < n_rows; ++r) {
      const RowBlocks row = row_blocks(p, h, row0 + r);
      uint64_t kept = 0;
#pragma unroll 1
      for (int a = 0; a <= r; ++a)
        if (row_keeps(p, row, h, row0 + r, row0 + a, row.count - 1)) kept |= __ballot(there && rel == a);
#pragma unroll
      for (int n = 0; n < NQ; ++n)
        if (rel_q[n] == r) seen[n] &= kept;
    }
  };
  // (a node that is not there may hold anything: nobody attends it, and it is not fetched)
  auto draft_rows = [&](int t, const uint16_t* of, auto& x) __attribute__((always_inline)) {
    const bool here = nodes_there >> (16 * t + c) & 1;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const u32x4 row = here ? *reinterpret_cast<const u32x4*>(of + b * p.kv_ss + h * p.kv_sh + (16 * t + c) * p.kv_sn + Rows::feature(kk, g)) : u32x4{};
      if constexpr (Rows::kScaled) {
        x[kk] = row;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * kk + e] = row[e];
      }
    }
  };

  typename Rows::Part kr[4], vr[4];
  auto load = [&](const Unit& w, const uint8_t* pool, const uint8_t* scales, const uint16_t* drafted, typename Rows::Part (&x)[4]) __attribute__((always_inline)) {
    if (w.drafts) {
      if constexpr (!Rows::kScaled) {
#pragma unroll
        for (int t = 0; t < 4; ++t) draft_rows(t, drafted, x[t].x);
      }
      return;  // (else fetched where they are used)
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const uint8_t* const at = pool + w.page[i] * p.c.page + w.skip[i] * p.c.tok;
      const uint8_t* const scale_at = Rows::kScaled ? scales + w.page[i] * p.c.scale_page + w.skip[i] * p.c.scale_tok : nullptr;
#pragma unroll
      for (int t = 0; t < 4 / NB; ++t) Rows::load(x[i + t], at, scale_at, w.rows[i], p.c.tok, p.c.scale_tok, 16 * t + c, g);
    }
  };
  // Tokens that the query of my column attends, where they are not all of the unit.
  uint64_t seen[NQ];
  bool some, mixed;  // not all queries attend all tokens; some query does not attend a token that is there
  auto scores = [&](const Unit& w) __attribute__((always_inline)) {
#pragma unroll
    for (int t0 = 0; t0 < 4; t0 += kGroup) {
      u32x4 k[kGroup][KK];
      if (Rows::kScaled && w.drafts) {
        if constexpr (Rows::kScaled) {
#pragma unroll
          for (int i = 0; i < kGroup; ++i) draft_rows(t0 + i, p.k_draft, k[i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < kGroup; ++i) Rows::operands(kr[t0 + i], g, k[i]);
      }
      score(t0, k);
    }
    some = mixed = w.drafts;
    if (w.drafts) {
      drafts_seen(seen);
    } else {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        some |= w.rows[i] < kTokens || w.bits[i] != all_rows;
        mixed |= w.rows[i] > 0 && w.bits[i] != all_rows;
      }
      if (some) {
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          seen[n] = 0;
#pragma unroll
          for (int i = 0; i < NB; ++i)
            if (w.bits[i] >> rel_q[n] & 1) seen[n] |= (w.rows[i] >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << w.rows[i]) - 1) << (16 * i);
        }
      }
    }
    if (some) {
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const uint32_t mine = (uint32_t)(seen[n] >> (32 * (t / 2))) >> (16 * (t % 2) + 4 * g);
#pragma unroll
          for (int e = 0; e < 4; ++e) s[n][t][e] = mine >> e & 1 ? s[n][t][e] : kNegInf;
        }
    }
  };
  auto sums = [&](const Unit& w) __attribute__((always_inline)) {
    softmax();
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      u32x4 v[2][KK];
      if (Rows::kScaled && w.drafts) {
        if constexpr (Rows::kScaled) {
#pragma unroll
          for (int i = 0; i < 2; ++i) draft_rows(2 * half + i, p.v_draft, v[i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) Rows::operands(vr[2 * half + i], g, v[i]);
      }
      bool odd = false;
      if (mixed) {
        uint32_t top = 0;  // (an exponent field of ones carries into its value's sign)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int kk = 0; kk < KK; ++kk)
#pragma unroll
            for (int e = 0; e < 4; ++e) top |= (v[i][kk][e] & 0x7fff7fffu) + 0x00800080u;
        odd = __any((top & 0x80008000u) != 0);
      }
      values(half, v, odd, seen);
    }
  };
  {
    Unit w;
    if (next_unit(w)) {
      load(w, p.c.k, p.c.ks, p.k_draft, kr);
      load(w, p.c.v, p.c.vs, p.v_draft, vr);
      for (;;) {
        Unit next;
        const bool more = next_unit(next);
        // the next unit's K goes into the registers that the scores have freed, its V into those that the sums free
        scores(w);
        __builtin_amdgcn_sched_barrier(0);
        if (more) load(next, p.c.k, p.c.ks, p.k_draft, kr);
        __builtin_amdgcn_sched_barrier(0);
        sums(w);
        __builtin_amdgcn_sched_barrier(0);
        if (!more) break;
        load(next, p.c.v, p.c.vs, p.v_draft, vr);
        w = next;
      }
    }
  }
  if (p.missing && lane == 0 && n_missing > 0) atomicAdd(p.missing, n_missing);

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
    if (sh_any_odd) {
#pragma unroll
      for (int ft = 0; ft < FT; ++ft) {
        const uint32_t found = wave == 0 ? sh_odd[(n * FT + ft) * 64 + lane] : 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t x = found >> (8 * e) & 7;
          if (x) acc[n][ft][e] = x == 1 ? -kNegInf : x == 2 ? kNegInf : __builtin_nanf("");
        }
      }
    }
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

template <int D, int FMT, bool SMALL>
void launch_split(const CacheAttnParams& p, hipStream_t stream) {
  const dim3 grid(p.nseq * p.heads * p.num_splits), block(256);
  if (p.nodes <= 16)
    hipLaunchKernelGGL((cache_attn_kernel<D, FMT, 1, SMALL>), grid, block, 0, stream, p);
  else if (p.nodes <= 32)
    hipLaunchKernelGGL((cache_attn_kernel<D, FMT, 2, SMALL>), grid, block, 0, stream, p);
  else
    hipLaunchKernelGGL((cache_attn_kernel<D, FMT, 4, SMALL>), grid, block, 0, stream, p);
}

template <int D, int FMT>
hipError_t launch_nodes(const CacheAttnParams& p, hipStream_t stream) {
  if (p.block_size < 64)
    launch_split<D, FMT, true>(p, stream);
  else
    launch_split<D, FMT, false>(p, stream);
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
