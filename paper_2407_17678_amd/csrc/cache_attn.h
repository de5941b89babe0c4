// Internal: what the kernels of attention over a paged cache (cache_attn_kernel.hip, cache_attn_shared_kernel.hip, cache_decode_kernel.hip) have in common: the
// nodes of a tree, the walk over the blocks that their rows keep, masks, and what is done about values of V that are not numbers.
#pragma once
#include <hip/hip_runtime.h>

#include "kernels.h"
#include "kv_cache.h"
#include "row_blocks.h"
#include "sched_util.h"

namespace s2 {

constexpr float kNegInf = -__builtin_inff();
constexpr int kMaxNodeRows = 5;  // block rows that 64 positions can lie in, blocks of 16 tokens

// Node `lane` of a sequence's tree.
struct Nodes {
  uint64_t above;    // it and the nodes above it, bits
  bool there;
  int rel;           // its block row, counted from row0
  int row0, n_rows;  // block rows of the nodes that are there
  uint64_t all;      // the nodes that are there
};
__device__ __forceinline__ Nodes nodes_of(const CacheAttnParams& p, int b, int L, int lane) {
  Nodes x;
  const int sh = p.c.block_shift;
  int up = lane < p.nodes ? p.parents[(int64_t)b * p.nodes + lane] : -2;
  if (up < -1 || up >= lane) up = -2;
  x.above = (uint64_t)1 << lane;
#pragma unroll
  for (int i = 0; i < 6; ++i) {  // (the chain above a node doubles each time)
    if (!__any(up >= 0)) break;
    const int from = max(up, 0);
    const uint32_t lo = __shfl((uint32_t)x.above, from, 64), hi = __shfl((uint32_t)(x.above >> 32), from, 64);
    const int next = __shfl(up, from, 64);
    if (up >= 0) {
      x.above |= (uint64_t)hi << 32 | lo;
      up = next;
    }
  }
  const int depth = __popcll(x.above) - 1;
  x.there = up == -1 && L + depth < p.max_len;
  x.row0 = L >> sh;
  x.rel = x.there ? ((L + depth) >> sh) - x.row0 : 0;
  x.all = __ballot(x.there);
  x.n_rows = x.all ? 1 : 0;
#pragma unroll
  for (int r = 1; r < kMaxNodeRows; ++r) x.n_rows += __ballot(x.rel >= r) != 0;
  return x;
}

// The kernel's parameters as they lie in memory, for what is done once or rarely: read there they do not occupy scalar registers in between (which the
// loops of these kernels have none to spare of: spilled to lanes, about 100 to a unit of 64 tokens, they took a third of its time).
__device__ __forceinline__ const CacheAttnParams& params_in_memory() {
  auto at = (const __attribute__((address_space(4))) CacheAttnParams*)(uintptr_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  return *(const CacheAttnParams*)at;
}

// 64 tokens: of one block, or (SMALL: blocks of 16 or 32) four pieces of 16 of the list's blocks.
template <bool SMALL>
struct Unit {
  static constexpr int NB = SMALL ? 4 : 1, kTokens = 64 / NB;
  int page[NB];
  int info[NB];          // tokens to read | block rows that keep it << 8 | tokens of the block before them << 16
  int my_page[2], my_info[2];  // SMALL: of the walk's own piece and the one after it
  bool some;   // some query may not attend some token
  bool mixed;  // some query does not attend a token that is there
  __device__ static int rows(int info) { return info & 255; }
  __device__ static int bits(int info) { return info >> 8 & 255; }
  __device__ static int skip(int info) { return info >> 16; }
};

// The units of a split, block row by block row: each block in the turn of the first row that keeps it.  Lanes look them up 64 at a time (SMALL: 16, a
// lane to a piece), so that a unit costs a few lane reads where it is used: looked up one by one by scalar instructions it is about 150 of them and two
// trips to the L2, in each wavefront.
template <bool SMALL>
struct Walk {
  static constexpr int NB = Unit<SMALL>::NB, kTokens = Unit<SMALL>::kTokens, kUnits = 64 / NB;
  int b, h, L, row0, n_rows, split, first, step, piece;  // unit `first` of the split, and every step-th
  int n_missing = 0;
  int r_now = -1, u_now = 0, u_end = 0;
  int page = 0, info = 0;            // of this lane's unit (piece)
  uint64_t live = 0, some = 0, mixed = 0;

  __device__ __forceinline__ Walk(int b_, int h_, int L_, const Nodes& x, int split_, int first_, int step_, int piece_)
      : b(b_), h(h_), L(L_), row0(x.row0), n_rows(x.n_rows), split(split_), first(first_), step(step_), piece(piece_) {}

  // bit NB * i: whether any of the NB bits from there on is set
  __device__ static uint64_t of_units(uint64_t pieces) {
    if (!SMALL) return pieces;
    pieces |= pieces >> 1;
    return (pieces | pieces >> 2) & 0x1111111111111111ull;
  }

  __device__ __forceinline__ void look_up(const CacheAttnParams& p) {
    const int S = p.block_size, sh = p.c.block_shift;
    RowBlocks rb;
    if (u_now < u_end) rb = row_blocks(p, h, row0 + r_now);
    while (u_now >= u_end) {
      if (r_now + 1 >= n_rows) return;
      ++r_now;
      rb = row_blocks(p, h, row0 + r_now);
      const int units = ((rb.count << sh) + 63) >> 6;
      const int even = units / p.by_splits, rest = units - even * p.num_splits;
      u_now = even * split + rest * split / p.by_splits + first;
      u_end = even * (split + 1) + rest * (split + 1) / p.by_splits;
    }
    const int lane = lane_now();
    const int u = u_now + step * (lane / NB), l = 64 * u + 16 * (lane % NB), n = l >> sh, skip = l & (S - 1);
    u_now += step * kUnits;
    const bool inside = u < u_end && n < rb.count;
    const int blk = inside ? rb.block_of_lane(n) : 0;
    int rows = inside ? min(max(L - (blk * S + skip), 0), kTokens) : 0, bits = 1 << r_now;
    if (n_rows > 1) {
#pragma unroll 1
      for (int r = 0; r < n_rows; ++r) {
        if (r == r_now) continue;
        const RowBlocks other = row_blocks(p, h, row0 + r);
        if (rows > 0 && row_keeps(p, other, h, row0 + r, blk, n)) {
          if (r < r_now) rows = 0;  // (read in that row's turn)
          bits |= 1 << r;
        }
      }
    }
    page = rows > 0 ? p.c.table[((int64_t)b * p.heads + h) * p.c.max_blocks + blk] : 0;
    const bool held = page >= 0 && page < p.c.num_pages;
    n_missing += __popcll(__ballot(rows > 0 && !held && skip == 0));
    if (!held) page = rows = 0;
    info = rows | bits << 8 | skip << 16;
    const int all = (1 << n_rows) - 1;
    live = of_units(__ballot(rows > 0));
    some = of_units(__ballot(rows < kTokens || bits != all));
    mixed = of_units(__ballot(rows > 0 && bits != all));
  }

  // The next unit with a token to read (AGAIN: the parameters are read from memory).
  template <bool AGAIN>
  __device__ __forceinline__ bool next(const CacheAttnParams& p, Unit<SMALL>& w) {
    while (live == 0) {
      if (u_now >= u_end && r_now + 1 >= n_rows) {
        // (no rows, so that loading it fetches nothing: the loads are issued in any case, for where a load might not have been issued
        // the compiler waits as if it had not, that is for what was issued after it)
#pragma unroll
        for (int t = 0; t < NB; ++t) w.page[t] = w.info[t] = 0;
        w.my_page[0] = w.my_page[1] = w.my_info[0] = w.my_info[1] = 0;
        w.some = w.mixed = false;
        return false;
      }
      look_up(AGAIN ? params_in_memory() : p);
    }
    const int i = __builtin_ctzll(live);
    live &= live - 1;
    w.some = some >> i & 1;
    w.mixed = mixed >> i & 1;
#pragma unroll
    for (int t = 0; t < NB; ++t) {
      w.page[t] = __builtin_amdgcn_readlane(page, i + t);
      w.info[t] = __builtin_amdgcn_readlane(info, i + t);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {  // (of the last piece there is none after it, and it is not used)
      w.my_page[t] = SMALL ? __builtin_amdgcn_readlane(page, i + ((piece + t) & 3)) : w.page[0];
      w.my_info[t] = SMALL ? __builtin_amdgcn_readlane(info, i + ((piece + t) & 3)) : w.info[0];
    }
    return true;
  }
};

// Tokens of a unit that a query in block row `rel` attends, bits.
template <bool SMALL>
__device__ __forceinline__ uint64_t unit_seen(const Unit<SMALL>& w, int rel) {
  uint64_t seen = 0;
#pragma unroll
  for (int i = 0; i < Unit<SMALL>::NB; ++i) {
    const int rows = Unit<SMALL>::rows(w.info[i]);
    if (Unit<SMALL>::bits(w.info[i]) >> rel & 1) seen |= (rows >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << rows) - 1) << (16 * i);
  }
  return seen;
}
// Drafted nodes that the query of node `node` attends: it and those above it, in blocks that its row keeps.
__device__ __forceinline__ uint64_t drafts_seen(const Nodes& x, int h, int node, int rel) {
  const uint32_t lo = __shfl((uint32_t)x.above, node, 64), hi = __shfl((uint32_t)(x.above >> 32), node, 64);
  uint64_t seen = (uint64_t)hi << 32 | lo;
  if (x.n_rows == 1) return seen;
  const CacheAttnParams& p = params_in_memory();
#pragma unroll 1
  for (int r = 0; r < x.n_rows; ++r) {
    const RowBlocks row = row_blocks(p, h, x.row0 + r);
    uint64_t kept = 0;
#pragma unroll 1
    for (int a = 0; a <= r; ++a)
      if (row_keeps(p, row, h, x.row0 + r, x.row0 + a, row.count - 1)) kept |= __ballot(x.there && x.rel == a);
    if (rel == r) seen &= kept;
  }
  return seen;
}
// A score tile of 16 tokens (the piece of index t) without those that are not attended.
__device__ __forceinline__ void mask_scores(f32x4& s, uint64_t seen, int t, int g) {
  const uint32_t mine = (uint32_t)(seen >> (32 * (t / 2))) >> (16 * (t % 2) + 4 * g);
#pragma unroll
  for (int e = 0; e < 4; ++e) s[e] = mine >> e & 1 ? s[e] : kNegInf;
}

// Probabilities on their way to V: the second operand of a matrix product holds bf16, so each goes as two terms, its first eight bits and what is left of it,
// 16 bits together.  (One rounded term is off by up to 2^-8, which a decode step, whose probabilities stay in 32 bits, is not; it would take one product of the two:
// us with one and with two terms, 64 x 32 heads of 31 to 47 blocks of 64 tokens, bf16 24 nodes 428 and 429, e4m3 24 nodes 243 and 246, 64 nodes 303 and 340, e2m1 12
// nodes 132 and 136, 24 nodes 165 and 185, 64 nodes 255 and 293.)  The first is cut, not rounded, and what is left counted 2^-23 too large, so that both are above 0
// wherever the probability is above 2^-100: twice an infinity of V is that infinity, and not NaN.
__device__ __forceinline__ void two_terms(float a, float b, uint32_t& first, uint32_t& rest) {
  const uint32_t x = __builtin_bit_cast(uint32_t, a), y = __builtin_bit_cast(uint32_t, b);
  first = __builtin_amdgcn_perm(y, x, 0x07060302);
  constexpr float kUp = 1.f + 0x1p-23f;
  rest = pack2(__builtin_fmaf(a, kUp, -__builtin_bit_cast(float, x & 0xffff0000u)), __builtin_fmaf(b, kUp, -__builtin_bit_cast(float, y & 0xffff0000u)));
}
// those of two tiles of scores, as an operand each
__device__ __forceinline__ void two_terms(const f32x4& lo, const f32x4& hi, bf16x8& first, bf16x8& rest) {
  uint32_t a[4], b[4];
  two_terms(lo[0], lo[1], a[0], b[0]);
  two_terms(lo[2], lo[3], a[1], b[1]);
  two_terms(hi[0], hi[1], a[2], b[2]);
  two_terms(hi[2], hi[3], a[3], b[3]);
  first = __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], a[2], a[3]});
  rest = __builtin_bit_cast(bf16x8, u32x4{b[0], b[1], b[2], b[3]});
}

// What a query does not attend stays out of its result whatever it holds; but its probability of 0 times an infinity or NaN in V is none.  Where
// some query does not attend some token of a unit and V holds such values, they are taken out of V, and which of them a query attends is found by
// products of ones and zeros and kept until the end, when they are added to its sums: those of units that all queries attend are in them already, and an
// infinity beside a NaN or the other infinity is a NaN.
//
// any_odd: whether one of these bf16 pairs is not finite (an exponent field of ones carries into its value's sign)
template <int KK>
__device__ __forceinline__ uint32_t odd_bits(const u32x4 (&v)[KK]) {
  uint32_t top = 0;
#pragma unroll
  for (int kk = 0; kk < KK; ++kk)
#pragma unroll
    for (int e = 0; e < 4; ++e) top |= (v[kk][e] & 0x7fff7fffu) + 0x00800080u;
  return top & 0x80008000u;
}
// For a tile of 16 queries and 32 tokens of V in LDS (transposed reads at v_read; seen: bits of the 32): ors two bits to each of the lane's four features of
// feature tile ft into byte ft % 4 of found[ft / 4 * 64 + lane]: 1 infinity, 2 minus infinity, 3 NaN (or both).
template <int D>
__device__ __forceinline__ void count_odd(uint32_t v_read, uint32_t seen, uint32_t* found, uint32_t* any, int lane) {
  const uint32_t mine = seen >> (4 * (lane >> 4));  // tokens 4 g .. and 16 + 4 g ..
  u32x4 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = ((mine >> (16 * (e / 2) + 2 * (e % 2))) & 1) * 0x3f80u + ((mine >> (16 * (e / 2) + 2 * (e % 2) + 1)) & 1) * 0x3f800000u;
#pragma unroll 1
  for (int i = 0; i < 2 * (D / 16); ++i) {
    const int ft = i / 2, kind = i % 2;
    auto ones = [&](uint32_t x) { return x == (kind ? 0xff80u : 0x7f80u) || (x & 0x7fffu) > 0x7f80u ? 0x3f80u : 0u; };
    u32x4 vf = lds_read_tr2(v_read + 32 * ft, v_read + 32 * ft, 0, 16 * ChunkTile<D>::RB);
#pragma unroll
    for (int e = 0; e < 4; ++e) vf[e] = ones(vf[e] & 0xffffu) | ones(vf[e] >> 16) << 16;
    const f32x4 count = mfma16(__builtin_bit_cast(bf16x8, vf), __builtin_bit_cast(bf16x8, w), f32x4{});
    uint32_t x = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) x |= (count[e] > 0.f ? 1u : 0u) << (2 * e + kind);
    if (x) {
      atomicOr(&found[ft / 4 * 64 + lane], x << (8 * (ft % 4)));
      *any = 1;
    }
  }
}
// Words of V without what is not finite.
__device__ __forceinline__ void clean_words(uint32_t* words, int n, int lane) {
#pragma unroll 1
  for (int i = lane; i < n; i += 64) {
    const uint32_t x = words[i];
    words[i] = ((x & 0x7f80u) == 0x7f80u ? 0u : x & 0xffffu) | ((x & 0x7f800000u) == 0x7f800000u ? 0u : x & 0xffff0000u);
  }
}
// What was found, added to a lane's sums (feature tile ft: four from sums[16 * ft]).
template <int D>
__device__ __forceinline__ void add_odd(float* sums, const uint32_t* found, int lane) {
#pragma unroll 1
  for (int i = 0; i < D / 4; ++i) {
    const uint32_t x = found[i / 16 * 64 + lane] >> (2 * (i % 16)) & 3;
    if (x) sums[16 * (i / 4) + i % 4] += x == 1 ? -kNegInf : x == 2 ? kNegInf : __builtin_nanf("");
  }
}

// Rows 16 t .. 16 t + 15 of drafted K or V, a lane's quarter of row c; a node that is not there may hold anything, nobody attends it, and it is
// not fetched.
template <class ROWS, bool V, int KK>
__device__ __forceinline__ void draft_rows(uint64_t nodes, int b, int h, int t, int c, int g, u32x4 (&x)[KK]) {
  const CacheAttnParams& p = params_in_memory();
  const uint16_t* const of = V ? p.v_draft : p.k_draft;
  const bool here = nodes >> (16 * t + c) & 1;
#pragma unroll
  for (int kk = 0; kk < KK; ++kk)
    x[kk] = here ? *reinterpret_cast<const u32x4*>(of + b * p.kv_ss + h * p.kv_sh + (16 * t + c) * p.kv_sn + ROWS::feature(kk, g)) : u32x4{};
}

// A query's result, or its part of a split: eight features from d.
template <int D>
__device__ __forceinline__ void put_result(const CacheAttnParams& p, int b, int h, int node, int split, int d, const float (&o)[8], float m, float l) {
  const int64_t row = ((int64_t)b * p.heads + h) * p.nodes + node;
  if (p.num_splits == 1) {
    bf16x8 out;
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = (__bf16)(l == 0.f ? 0.f : o[e] / l);
    *reinterpret_cast<bf16x8*>(p.o + b * p.q_ss + h * p.q_sh + node * p.q_sn + d) = out;
    if (d == 0 && p.lse) p.lse[row] = l == 0.f ? kNegInf : m * p.scale + __logf(l);
  } else {
    f32x4* const to = reinterpret_cast<f32x4*>(p.part_acc + (row * p.num_splits + split) * D + d);
    to[0] = f32x4{o[0], o[1], o[2], o[3]};
    to[1] = f32x4{o[4], o[5], o[6], o[7]};
    if (d == 0) {
      p.part_ml[(row * p.num_splits + split) * 2] = m;
      p.part_ml[(row * p.num_splits + split) * 2 + 1] = l;
    }
  }
}

// The launch of a decode step over 8 or 4 bits (all but the merge of splits).
hipError_t launch_cache_decode(const CacheAttnParams& p, hipStream_t stream);
// The launch for more than 16 nodes (all but the merge of splits).
hipError_t launch_cache_attn_shared(const CacheAttnParams& p, hipStream_t stream);

}  // namespace s2
