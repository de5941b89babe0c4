// Attention of a chunk of new tokens to each sequence over a paged cache in bf16, 8 or 4 bits that holds their keys and values already (section 4.1's cache,
// section 5.3's prefill in chunks).
//
// o_i = sum_j p_ij v_j / sum_j p_ij, p_ij = exp(scale q_i k_j - max), over the cached tokens j <= i that the block row of i keeps.  Queries of a tile share
// what they read: a tile of 16 rows makes 64 D flops of a token's K and V, so that a tile of a few rows is bound by the cache's bytes and one of 128 by
// matrix instructions.
//
// The four wavefronts of a workgroup share a unit of 64 tokens: each fetches a piece of 16 of them, brings it to bf16 once and writes its K and V rows into LDS
// (ChunkTile); then each takes its 16 or 32 queries against the whole unit.  Scores are formed as keys x queries, so that a lane holds one query and the
// probabilities are the second operand of the product with V as they stand.
#include <hip/hip_runtime.h>

#include "cache_attn.h"
#include "config.h"

namespace s2 {

namespace {

// A tile of a launch: `rows` (0: there is no such tile) new tokens of sequence b from its row `row` on, which is the token at position `pos`; the first new
// token is at position `start`.
struct ChunkTileAt {
  int b, row, rows;
  int skipped;          // queries of the tile before its first row
  int64_t pos, start;
};
// Tiles of up to kChunkFew rows begin at a sequence's first new token, larger ones at multiples of their rows in its positions, so that a tile lies in as few
// block rows as it can.  Either every sequence has as many as the longest may need, or (packed) there are those of the rows that there are: sequence
// b, whose rows begin at lo, has the tiles from lo / rows + 2 b on, as many at least as it needs, and the last one that begins at or before a tile is found 64
// sequences at a time.
// (a sequence's rows in the tensors)
__device__ __forceinline__ int chunk_rows(const CacheChunkParams& p, int lo, int hi) {
  const int from = min(max(lo, 0), p.num_rows);
  return (int)min((int64_t)(min(max(hi, from), p.num_rows) - from), max(p.max_new - (from - (int64_t)lo), (int64_t)0));
}
__device__ __forceinline__ ChunkTileAt chunk_tile_at(const CacheChunkParams& p, int t) {
  ChunkTileAt x;
  int tile, lo, hi, start;
  if (!p.packed) {
    x.b = t / p.by_tiles;
    tile = t - x.b * p.seq_tiles;
    lo = load_const<int32_t>(p.cu + x.b);
    hi = load_const<int32_t>(p.cu + x.b + 1);
    start = load_const<int32_t>(p.start + x.b);
  } else {
    const int lane = threadIdx.x & 63;
    int first = 0, count = p.nseq;
    for (;;) {
      const int step = (count + 63) >> 6;
      const bool is = lane * step < count;
      const int b = first + (is ? lane * step : 0);
      const int from = p.cu[b], to = p.cu[b + 1], at = p.start[b];
      const int begins = (min(max(from, 0), p.num_rows) >> p.tile_shift) + 2 * b;
      const int last = max(__popcll(__ballot(is && begins <= t)) - 1, 0);
      if (step == 1) {
        x.b = first + last;
        lo = __builtin_amdgcn_readlane(from, last);
        hi = __builtin_amdgcn_readlane(to, last);
        start = __builtin_amdgcn_readlane(at, last);
        tile = t - __builtin_amdgcn_readlane(begins, last);
        break;
      }
      first += last * step;
      count = min(step, count - last * step);
    }
  }
  // rows of the tensors, whatever the arrays hold
  const int from = min(max(lo, 0), p.num_rows);
  const int n = chunk_rows(p, lo, hi);
  x.start = (int64_t)start + (from - (int64_t)lo);
  const int BM = 1 << p.tile_shift;
  const int head = p.tile_shift > 6 ? (int)(x.start & (BM - 1)) : 0;
  const int r0 = (int)min(max((int64_t)tile * BM - head, (int64_t)0), (int64_t)n), r1 = (int)min((int64_t)(tile + 1) * BM - head, (int64_t)n);
  x.rows = max(r1 - r0, 0);
  x.skipped = tile == 0 ? head : 0;
  x.pos = x.start + r0;
  x.row = from + r0;
  return x;
}

// Positions [lo, hi) of a tile that the table has room for, and the block rows they lie in.
struct Rows8 {
  int lo, hi, row0, n_rows;
};

// 64 tokens: of one block, or (SMALL) four pieces of 16 of the list's blocks.
template <bool SMALL>
struct ChunkUnit {
  static constexpr int NB = SMALL ? 4 : 1, kTokens = 64 / NB;
  int info[NB];          // tokens to read | block rows that keep them << 8
  int at[NB];            // position of the first
  int my_page, my_info, my_at;  // of this wavefront's piece
  bool some;             // some query may not attend some token
};

// The units of a split.  In closed form the blocks that any row of the tile keeps are those of its first row and the blocks after them up to the last; lists are
// walked row by row, each block in the turn of the first row that keeps it.  Lanes look units up 64 at a time (SMALL: 16, a lane to a piece).
template <bool SMALL>
struct ChunkWalk {
  static constexpr int NB = ChunkUnit<SMALL>::NB, kTokens = ChunkUnit<SMALL>::kTokens, kUnits = 64 / NB;
  int b, h, piece, split;
  Rows8 r;
  int first_row;                     // block row of the chunk's first token, for what is counted
  bool first_tile;
  int n_missing = 0;
  int turn = -1, u_now = 0, u_end = 0;
  int page = 0, info = 0, at = 0;    // of this lane's unit (piece)
  uint64_t live = 0, some = 0;

  __device__ static uint64_t of_units(uint64_t pieces) {
    if (!SMALL) return pieces;
    pieces |= pieces >> 1;
    return (pieces | pieces >> 2) & 0x1111111111111111ull;
  }

  __device__ __forceinline__ RowBlocks blocks_of(const CacheChunkParams& p, int turn_) const {
    RowBlocks rb = row_blocks(p, h, r.row0 + turn_);
    if (!p.row_ptr) rb.count = rb.n_stripe + (r.row0 + r.n_rows - rb.local_lo);
    return rb;
  }

  __device__ __forceinline__ void look_up(const CacheChunkParams& p) {
    const int sh = p.c.block_shift, S = 1 << sh, turns = p.row_ptr ? r.n_rows : 1;
    RowBlocks rb;
    if (u_now < u_end) rb = blocks_of(p, turn);
    while (u_now >= u_end) {
      if (turn + 1 >= turns) return;
      ++turn;
      rb = blocks_of(p, turn);
      const int units = (int)((((int64_t)rb.count << sh) + 63) >> 6);
      const int even = units / p.by_splits, rest = units - even * p.num_splits;
      u_now = even * split + rest * split / p.by_splits;
      u_end = even * (split + 1) + rest * (split + 1) / p.by_splits;
    }
    const int lane = lane_now();
    const int u = u_now + lane / NB, l = 64 * u + 16 * (lane % NB), n = l >> sh, skip = l & (S - 1);
    u_now += kUnits;
    const bool inside = u < u_end && n < rb.count;
    const int blk = inside ? rb.block_of_lane(n) : 0;
    at = blk * S + skip;
    int rows = inside ? min(max(r.hi - at, 0), kTokens) : 0, bits = 0;
#pragma unroll 1
    for (int i = 0; i < r.n_rows; ++i) {
      const RowBlocks other = p.row_ptr ? row_blocks(p, h, r.row0 + i) : RowBlocks{};
      if (rows > 0 && row_keeps(p, other, h, r.row0 + i, blk, n)) {
        if (i < turn) rows = 0;  // (read in that row's turn)
        bits |= 1 << i;
      }
    }
    if (bits == 0) rows = 0;
    page = rows > 0 ? p.c.table[((int64_t)b * p.heads + h) * p.c.max_blocks + blk] : 0;
    const bool held = page >= 0 && page < p.c.num_pages;
    if (__any(rows > 0 && !held) && p.missing) {
      // a block counts once: in the tile of the first of the chunk's rows that keeps it (in closed form no row drops a block and keeps it later)
      bool counts = rows > 0 && !held && skip == 0;
      if (!first_tile) {
        if (p.row_ptr) {
#pragma unroll 1
          for (int i = first_row; i < r.row0; ++i) {
            const RowBlocks other = row_blocks(p, h, i);
            if (counts && row_keeps(p, other, h, i, blk, n)) counts = false;
          }
        } else {
          counts = counts && blk * S >= r.lo;
        }
      }
      n_missing += __popcll(__ballot(counts));
    }
    if (!held) page = rows = 0;
    info = rows | bits << 8;
    const int all = (1 << r.n_rows) - 1;
    live = of_units(__ballot(rows > 0));
    some = of_units(__ballot(rows < kTokens || bits != all || at + rows - 1 > r.lo));
  }

  __device__ __forceinline__ bool next(const CacheChunkParams& p, ChunkUnit<SMALL>& w) {
    while (live == 0) {
      if (u_now >= u_end && turn + 1 >= (p.row_ptr ? r.n_rows : 1)) {
#pragma unroll
        for (int t = 0; t < NB; ++t) w.info[t] = w.at[t] = 0;
        w.my_page = w.my_info = w.my_at = 0;  // (no rows: loading it fetches nothing)
        w.some = false;
        return false;
      }
      look_up(p);
    }
    const int i = __builtin_ctzll(live);
    live &= live - 1;
    w.some = some >> i & 1;
#pragma unroll
    for (int t = 0; t < NB; ++t) {
      w.info[t] = __builtin_amdgcn_readlane(info, i + t);
      w.at[t] = __builtin_amdgcn_readlane(at, i + t);
    }
    const int mine = SMALL ? i + piece : i;
    w.my_page = __builtin_amdgcn_readlane(page, mine);
    w.my_info = SMALL ? __builtin_amdgcn_readlane(info, mine) : w.info[0];
    w.my_at = SMALL ? __builtin_amdgcn_readlane(at, mine) : w.at[0];
    return true;
  }
};

// Tokens of a unit that the query at position `pos`, in the tile's block row `rel`, attends, bits.
template <bool SMALL>
__device__ __forceinline__ uint64_t chunk_seen(const ChunkUnit<SMALL>& w, int rel, int pos) {
  uint64_t seen = 0;
#pragma unroll
  for (int i = 0; i < ChunkUnit<SMALL>::NB; ++i) {
    const int rows = min(w.info[i] & 255, pos - w.at[i] + 1);
    if ((w.info[i] >> 8 >> rel & 1) && rows > 0) seen |= (rows >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << rows) - 1) << (16 * i);
  }
  return seen;
}

constexpr int chunk_waves_for(int D, int NQ) { return NQ == 2 ? (D == 64 ? 3 : 2) : D == 64 ? 4 : 3; }

// A workgroup: 64 * NQ queries of one (sequence, head), one split of what they attend.
template <int D, int FMT, int NQ, bool SMALL>
__global__ __launch_bounds__(256, chunk_waves_for(D, NQ)) void cache_chunk_kernel(const CacheChunkParams p) {
  using Rows = CacheRows<D, FMT>;
  using Tile = ChunkTile<D>;
  constexpr int W = 4, KK = D / 32, FT = D / 16, kOdd = NQ * FT / 4 * 64;
  constexpr int RS = D + 4;           // floats to a row where results are turned
  static_assert(W * 16 * RS * 4 <= 2 * Tile::kBytes, "the wavefronts' sums, a tile of 16 queries each, fit where K and V were");

  __shared__ __align__(16) uint16_t sh_kv[2][Tile::kElems];
  __shared__ float sh_m[W][16], sh_l[W][16];
  __shared__ uint32_t sh_odd[W * kOdd];  // (count_odd)
  __shared__ uint32_t sh_any_odd, sh_unit_odd[2];

  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int th = blockIdx.x / p.by_splits, split = blockIdx.x - th * p.num_splits;
  const int tile = th / p.by_heads, h = th - tile * p.heads;
  const float cl = p.scale_log2e;

  const ChunkTileAt x = chunk_tile_at(p, tile);
  if (x.rows <= 0) return;
  const int b = x.b;
  Rows8 r;
  r.lo = (int)min(max(x.pos, (int64_t)0), (int64_t)p.max_len);
  r.hi = (int)min(max(x.pos + x.rows, (int64_t)0), (int64_t)p.max_len);
  const bool any = r.lo < r.hi;
  r.row0 = r.lo >> p.c.block_shift;
  r.n_rows = any ? ((r.hi - 1) >> p.c.block_shift) - r.row0 + 1 : 0;

  // the queries of my column: a wavefront's are 16 * NQ that lie side by side, counted from the tile's beginning
  int row_q[NQ], pos_q[NQ], rel_q[NQ];
  bool there_q[NQ];
  bf16x8 qf[NQ][KK];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    row_q[n] = 16 * NQ * wave + 16 * n + c - x.skipped;
    const int64_t pos = x.pos + row_q[n];
    there_q[n] = row_q[n] >= 0 && row_q[n] < x.rows && pos >= r.lo && pos < r.hi;
    pos_q[n] = there_q[n] ? (int)pos : -1;
    rel_q[n] = there_q[n] ? (pos_q[n] >> p.c.block_shift) - r.row0 : 0;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
      qf[n][kk] = there_q[n] ? *reinterpret_cast<const bf16x8*>(p.q + (x.row + row_q[n]) * p.q_sr + h * p.q_sh + 32 * kk + 8 * g) : bf16x8{};
  }
  bool any_q = false;
#pragma unroll
  for (int n = 0; n < NQ; ++n) any_q = any_q || __any(there_q[n]);

  for (int i = tid; i < W * kOdd; i += 64 * W) sh_odd[i] = 0;
  if (tid == 0) sh_any_odd = sh_unit_odd[0] = sh_unit_odd[1] = 0;

  f32x4 acc[NQ][FT];
  float m_run[NQ], l_run[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m_run[n] = kNegInf;
    l_run[n] = 0.f;
#pragma unroll
    for (int ft = 0; ft < FT; ++ft) acc[n][ft] = f32x4{};
  }

  const uint32_t at_k = lds_addr(sh_kv[0]), at_v = lds_addr(sh_kv[1]);
  // (writes without bank conflicts: see cache_attn_shared_kernel.hip)
  const bool turned = ((c >> 3 ^ c >> 2) & 1) != 0;
  const int gw = FMT == S2_KV_BF16 && turned ? g ^ 1 : g;
  const uint32_t write = (16 * wave + c) * Tile::RB;
  const uint32_t k_read = at_k + Tile::row_lane(lane), v_read = at_v + Tile::tr_lane(lane);
  ChunkWalk<SMALL> walk;
  walk.b = b;
  walk.h = h;
  walk.piece = wave;
  walk.split = split;
  walk.r = r;
  walk.first_row = (int)min(max(x.start, (int64_t)0), (int64_t)p.max_len - 1) >> p.c.block_shift;
  walk.first_tile = x.pos == x.start || x.pos <= 0;
  if (!any) walk.turn = 1 << 20;  // (nothing to look up)

  typename Rows::Part kr, vr;
  auto load = [&](auto is_v, const ChunkUnit<SMALL>& w, typename Rows::Part& to) __attribute__((always_inline)) {
    constexpr bool V = decltype(is_v)::value;
    const int skip = w.my_at & (p.block_size - 1);
    const uint8_t* const at = (V ? p.c.v : p.c.k) + w.my_page * p.c.page + skip * p.c.tok;
    const uint8_t* const scale_at = Rows::kScaled ? (V ? p.c.vs : p.c.ks) + w.my_page * p.c.scale_page + skip * p.c.scale_tok : nullptr;
    Rows::load(to, at, scale_at, w.my_info & 255, p.c.tok, p.c.scale_tok, (SMALL ? 0 : 16 * wave) + c, gw);
  };
  constexpr std::false_type kK{};
  constexpr std::true_type kV{};
  auto put_part = [&](auto is_v, typename Rows::Part& part, uint32_t to, bool some, int turn) __attribute__((always_inline)) {
    u32x4 rows[KK];
    if constexpr (Rows::kScaled) Rows::turn(part, turned);
    Rows::operands(part, g, rows);
    const int turn_of = Rows::kScaled && turned ? 16 : 0;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
      *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(to + write + (kk % 2 ? -turn_of : turn_of) + 2 * Rows::feature(kk, gw)) = rows[kk];
    if (decltype(is_v)::value && some) {
      asm volatile("");  // (else looked for in every unit)
      if (odd_bits(rows)) sh_unit_odd[turn] = 1;
    }
  };
  // (what it has asked of the LDS is done before a wavefront is past it; loads from memory stay on their way)
  auto barrier = [&]() __attribute__((always_inline)) {
    wait_lds();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  auto attend = [&](const ChunkUnit<SMALL>& w, int turn) __attribute__((always_inline)) {
    const bool odd = w.some && sh_unit_odd[turn];  // (the same for all wavefronts)
    f32x4 s[NQ][4];
    if (any_q) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          const bf16x8 k = __builtin_bit_cast(bf16x8, lds_read16(k_read, Tile::row_off(t, kk)));
#pragma unroll
          for (int n = 0; n < NQ; ++n) s[n][t] = mfma16(k, qf[n][kk], kk ? s[n][t] : f32x4{});
        }
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        uint64_t seen = 0;
        if (w.some) {
          seen = chunk_seen<SMALL>(w, rel_q[n], pos_q[n]);
#pragma unroll
          for (int t = 0; t < 4; ++t) mask_scores(s[n][t], seen, t, g);
        }
        float mx = kNegInf;
#pragma unroll
        for (int t = 0; t < 4; ++t)
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
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[n][t][e] = fast_exp2(__builtin_fmaf(s[n][t][e], cl, -mc));
            l_run[n] += s[n][t][e];
          }
        if (odd) {
#pragma unroll 1
          for (int u = 0; u < 2; ++u)
            count_odd<D>(v_read + 32 * u * Tile::RB, (uint32_t)(seen >> (32 * u)), sh_odd + wave * kOdd + n * FT / 4 * 64, &sh_any_odd, lane);
        }
      }
    }
    if (odd) {
      barrier();
      clean_words(reinterpret_cast<uint32_t*>(sh_kv[1]) + 16 * wave * Tile::RB / 4, 16 * Tile::RB / 4, lane);
      barrier();
    }
    if (!any_q) return;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      bf16x8 pf[NQ], pr[NQ];
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        if constexpr (NQ == 1) {
          two_terms(s[n][2 * u], s[n][2 * u + 1], pf[n], pr[n]);
        } else {
          // rounded to bf16, as in the forward of a whole sequence: off by up to 2^-8 of a probability, about what rounding the result is
          pf[n] = __builtin_bit_cast(bf16x8, u32x4{pack2(s[n][2 * u][0], s[n][2 * u][1]), pack2(s[n][2 * u][2], s[n][2 * u][3]),
                                                   pack2(s[n][2 * u + 1][0], s[n][2 * u + 1][1]), pack2(s[n][2 * u + 1][2], s[n][2 * u + 1][3])});
        }
      }
#pragma unroll
      for (int ft = 0; ft < FT; ++ft) {
        const bf16x8 vf = __builtin_bit_cast(bf16x8, lds_read_tr2(v_read, v_read, Tile::tr_off(u, ft), Tile::tr_off(u, ft) + 16 * Tile::RB));
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          if constexpr (NQ == 1) acc[n][ft] = mfma16(vf, pr[n], acc[n][ft]);
          acc[n][ft] = mfma16(vf, pf[n], acc[n][ft]);
        }
      }
    }
  };

  {
    int turn = 0;
    ChunkUnit<SMALL> w;
    bool more = walk.next(p, w);
    load(kK, w, kr);
    load(kV, w, vr);
    for (; more; turn ^= 1) {
      ChunkUnit<SMALL> next;
      more = walk.next(p, next);
      barrier();  // nobody reads the unit before any more
      put_part(kK, kr, at_k, false, turn);
      put_part(kV, vr, at_v, w.some, turn);
      if (tid == 0) sh_unit_odd[turn ^ 1] = 0;
      load(kK, next, kr);
      load(kV, next, vr);
      barrier();
      attend(w, turn);
      w = next;
    }
  }
  if (p.missing && tid == 0 && walk.n_missing > 0) atomicAdd(p.missing, walk.n_missing);

  // results from query-on-lane to rows, a tile of 16 queries of every wavefront at a time, through where K and V were
  float* const sums = reinterpret_cast<float*>(sh_kv[0]);
  float* const mine = sums + (16 * wave + c) * RS + 4 * g;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const float l = sum_groups(l_run[n]);
    __syncthreads();
    if (g == 0) {
      sh_m[wave][c] = there_q[n] ? m_run[n] : kNegInf;
      sh_l[wave][c] = there_q[n] ? l : 0.f;
    }
#pragma unroll
    for (int ft = 0; ft < FT; ++ft) *reinterpret_cast<f32x4*>(mine + 16 * ft) = there_q[n] ? acc[n][ft] : f32x4{};
    if (sh_any_odd && there_q[n]) add_odd<D>(mine, sh_odd + wave * kOdd + n * FT / 4 * 64, lane);
    __syncthreads();
    constexpr int TPR = D / 8;  // threads to a query, eight features each
    for (int i = tid / TPR; i < 16 * W; i += 64 * W / TPR) {
      const int row = 16 * NQ * (i / 16) + 16 * n + i % 16 - x.skipped, d = 8 * (tid % TPR);
      if (row < 0 || row >= x.rows) continue;
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = sums[i * RS + d + e];
      const float m = sh_m[i / 16][i % 16], ls = sh_l[i / 16][i % 16];
      if (p.num_splits == 1) {
        bf16x8 out;
#pragma unroll
        for (int e = 0; e < 8; ++e) out[e] = (__bf16)(ls == 0.f ? 0.f : o[e] / ls);
        *reinterpret_cast<bf16x8*>(p.o + (x.row + row) * p.q_sr + h * p.q_sh + d) = out;
        if (d == 0 && p.lse) p.lse[(int64_t)h * p.num_rows + x.row + row] = ls == 0.f ? kNegInf : m * p.scale + __logf(ls);
      } else {
        // (rows of a sequence are counted from its first one in the tensors)
        const int64_t at = (((int64_t)b * p.heads + h) * p.max_new + (x.pos - x.start) + row) * p.num_splits + split;
        f32x4* const to = reinterpret_cast<f32x4*>(p.part_acc + at * D + d);
        to[0] = f32x4{o[0], o[1], o[2], o[3]};
        to[1] = f32x4{o[4], o[5], o[6], o[7]};
        if (d == 0) {
          p.part_ml[at * 2] = m;
          p.part_ml[at * 2 + 1] = ls;
        }
      }
    }
  }
}

// Merges the splits, a wavefront to a row (see cache_attn_kernel.hip).
template <int D>
__global__ __launch_bounds__(256) void cache_chunk_merge_kernel(const CacheChunkParams p) {
  constexpr int LPR = D / 4, NG = 64 / LPR;
  const int lane = threadIdx.x & 63, g = lane / LPR, c = lane % LPR, n = p.num_splits;
  const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t bh = item / p.max_new;
  const int i = (int)(item - bh * p.max_new);
  if (bh >= (int64_t)p.nseq * p.heads) return;
  const int b = (int)bh / p.by_heads, h = (int)bh - b * p.heads;
  const int lo = load_const<int32_t>(p.cu + b), hi = load_const<int32_t>(p.cu + b + 1);
  const int from = min(max(lo, 0), p.num_rows);
  if (i >= chunk_rows(p, lo, hi)) return;
  const float* const ml = p.part_ml + item * n * 2;
  const f32x4* const part = reinterpret_cast<const f32x4*>(p.part_acc) + item * n * LPR + c;
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
  for (int s0 = 0; s0 < n; s0 += NG) {
    const int s = s0 + g;
    const float of = __shfl(weight, s & 63, 64);
    if (s < n) a += part[(int64_t)s * LPR] * of;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float y = a[e];
    if (LPR == 16) y = sum_rows(y);
    a[e] = sum_halves(y);
  }
  if (lane >= LPR) return;
  bf16x4 out;
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = (__bf16)(l == 0.f ? 0.f : a[e] / l);
  const int64_t row = from + i;
  *reinterpret_cast<bf16x4*>(p.o + row * p.q_sr + h * p.q_sh + 4 * c) = out;
  if (lane == 0 && p.lse) p.lse[(int64_t)h * p.num_rows + row] = l == 0.f ? kNegInf : m * p.scale + __logf(l);
}

template <int D, int FMT, int NQ>
void launch_blocks(const CacheChunkParams& p, hipStream_t stream) {
  const dim3 grid(p.num_tiles * p.heads * p.num_splits), block(256);
  if (p.block_size < 64)
    hipLaunchKernelGGL((cache_chunk_kernel<D, FMT, NQ, true>), grid, block, 0, stream, p);
  else
    hipLaunchKernelGGL((cache_chunk_kernel<D, FMT, NQ, false>), grid, block, 0, stream, p);
}

template <int D, int FMT>
void launch_tiles(const CacheChunkParams& p, hipStream_t stream) {
  if (p.tile_shift <= 6)
    launch_blocks<D, FMT, 1>(p, stream);
  else
    launch_blocks<D, FMT, 2>(p, stream);
}

template <int D>
hipError_t launch_dim(const CacheChunkParams& p, hipStream_t stream) {
  switch (p.c.format) {
    case S2_KV_BF16: launch_tiles<D, S2_KV_BF16>(p, stream); break;
    case S2_KV_MXFP8: launch_tiles<D, S2_KV_MXFP8>(p, stream); break;
    default: launch_tiles<D, S2_KV_MXFP4>(p, stream); break;
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.num_splits == 1) return e;
  const int64_t rows = (int64_t)p.nseq * p.heads * p.max_new;
  hipLaunchKernelGGL((cache_chunk_merge_kernel<D>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

int64_t chunk_tiles(CacheChunkParams& p) {
  p.tile_shift = p.max_new <= kChunkFew ? 6 : 7;
  const int64_t BM = 1 << p.tile_shift;
  const int64_t each = p.max_new <= kChunkFew ? 1 : (p.max_new + 2 * BM - 2) / BM;
  const int64_t of_rows = p.num_rows / BM + 2 * (int64_t)p.nseq;
  p.packed = of_rows < each * p.nseq;
  const int64_t tiles = p.packed ? of_rows : each * p.nseq;
  p.seq_tiles = (int)each;
  p.num_tiles = (int)std::min<int64_t>(tiles, kMostGroups + 1);
  return tiles;
}

hipError_t launch_cache_chunk(const CacheChunkParams& params, hipStream_t stream) {
  CacheChunkParams p = params;
  p.by_heads = fast_div(p.heads);
  p.by_splits = fast_div(p.num_splits);
  p.by_stride = fast_div(p.stride > 0 ? p.stride : 1);
  p.by_tiles = fast_div(p.seq_tiles);
  return p.c.head_dim == 128 ? launch_dim<128>(p, stream) : launch_dim<64>(p, stream);
}

}  // namespace s2
