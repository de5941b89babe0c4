// Internal: what the kernels of attention of a chunk of new tokens over a paged cache (cache_chunk_kernel.hip, cache_chunk_wide_kernel.hip) have in common: the
// tiles of a launch, and the walk over the blocks that a tile's rows keep.
#pragma once
#include <hip/hip_runtime.h>

#include "cache_attn.h"

namespace s2 {

// A tile of a launch: `rows` (0: there is no such tile) new tokens of sequence b from its row `row` on, which is the token at position `pos`; the first new
// token is at position `start`.
struct ChunkTileAt {
  int b, row, rows;
  int skipped;          // queries of the tile before its first row
  int64_t pos, start;
};
// Tiles of up to kChunkFew rows begin at a sequence's first new token, larger ones at multiples of their rows in its positions, so that a tile lies in as few
// block rows as it can.  Either every sequence has as many as the longest may need (the last ones, which few need, behind all others: between them they left
// compute units idle that got two of them, 4 sequences of 256 rows with 1024 + 2048 tokens each to attend 97 us, so 76), or (packed) there are those of the rows that there are: sequence
// b, whose rows begin at lo, has the tiles from lo / rows + 2 b on, as many at least as it needs, and the last one that begins at or before a tile is found 64
// sequences at a time.  Of up to 64 sequences (sorted) a lane to a sequence counts its tiles, and they go by where they end, latest first: the longest work does not
// begin last (64 sequences of 1 to 12 rows 222 us to 212, 4 of up to 256 rows 56 to 42, 12 of up to 1024 rows 180 to 176; at worst 12 of up to 40 rows 53 to 58).
// (a sequence's rows in the tensors)
__device__ __forceinline__ int chunk_rows(const CacheChunkParams& p, int lo, int hi) {
  const int from = min(max(lo, 0), p.num_rows);
  return (int)min((int64_t)(min(max(hi, from), p.num_rows) - from), max(p.max_new - (from - (int64_t)lo), (int64_t)0));
}
__device__ __forceinline__ ChunkTileAt chunk_tile_at(const CacheChunkParams& p, int t) {
  ChunkTileAt x;
  int tile, lo, hi, start;
  if (!p.packed && !p.sorted) {
    const int begun = p.seq_tiles - 1, last = t - p.nseq * begun;
    x.b = last < 0 ? t / p.by_tiles : last;
    tile = last < 0 ? t - x.b * begun : begun;
    lo = load_const<int32_t>(p.cu + x.b);
    hi = load_const<int32_t>(p.cu + x.b + 1);
    start = load_const<int32_t>(p.start + x.b);
  } else if (p.sorted) {
    const int lane = threadIdx.x & 63, b = min(lane, p.nseq - 1);
    const int from = p.cu[b], to = p.cu[b + 1], at = p.start[b];
    const int rows = lane < p.nseq ? chunk_rows(p, from, to) : 0;
    const int64_t begin = (int64_t)at + (min(max(from, 0), p.num_rows) - (int64_t)from);
    const int64_t skipped = p.tile_shift > 6 ? begin & ((1 << p.tile_shift) - 1) : 0;
    const int tiles = rows > 0 ? (int)((skipped + rows - 1) >> p.tile_shift) + 1 : 0;
    const int ends = (int)min(max(begin + rows, (int64_t)0), (int64_t)p.max_len);
    int before = 0;
    for (int c0 = 0; c0 < p.nseq; c0 += 8)
#pragma unroll
      for (int c = c0; c < c0 + 8; ++c) {  // (lanes without a sequence have no tiles)
        const int other = __builtin_amdgcn_readlane(ends, c), of = __builtin_amdgcn_readlane(tiles, c);
        before += other > ends || (other == ends && c < lane) ? of : 0;
      }
    const uint64_t mine = __ballot(t >= before && t - before < tiles);
    x.b = mine ? __builtin_ctzll(mine) : 0;
    lo = __builtin_amdgcn_readlane(from, x.b);
    hi = mine ? __builtin_amdgcn_readlane(to, x.b) : lo;
    start = __builtin_amdgcn_readlane(at, x.b);
    tile = __builtin_amdgcn_readlane(tiles, x.b) - 1 - (t - __builtin_amdgcn_readlane(before, x.b));
    tile = mine ? tile : 0;
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

// The kernel's parameters as they lie in memory (see params_in_memory in cache_attn.h): what is done once to 64 units, or to 16, reads them there.
__device__ __forceinline__ const CacheChunkParams& chunk_params() {
  auto at = (const __attribute__((address_space(4))) CacheChunkParams*)(uintptr_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  return *(const CacheChunkParams*)at;
}

// (loaded as a whole: word by word, where each is used, they are a dozen trips to memory one after the other)
__device__ __forceinline__ ChunkLookUp chunk_look_up() {
  typedef uint32_t u32x16 __attribute__((ext_vector_type(16)));
  const char* const at = reinterpret_cast<const char*>(&chunk_params().look_up);
  struct {
    u32x16 a, b;
  } w = {load_const<u32x16>(at), load_const<u32x16>(at + 64)};
  asm volatile("" : "+s"(w.a), "+s"(w.b));
  return __builtin_bit_cast(ChunkLookUp, w);
}

// Positions [lo, hi) of a tile that the table has room for, and the block rows they lie in (eight at most).
struct ChunkRows {
  int lo, hi, row0, n_rows;
};
__device__ __forceinline__ ChunkRows chunk_block_rows(const CacheChunkParams& p, const ChunkTileAt& x) {
  ChunkRows r;
  r.lo = (int)min(max(x.pos, (int64_t)0), (int64_t)p.max_len);
  r.hi = (int)min(max(x.pos + x.rows, (int64_t)0), (int64_t)p.max_len);
  r.row0 = r.lo >> p.c.block_shift;
  r.n_rows = r.lo < r.hi ? ((r.hi - 1) >> p.c.block_shift) - r.row0 + 1 : 0;
  return r;
}
// A lane's query: row `row` of a tile (negative, or beyond its rows: there is none).
struct ChunkQuery {
  int pos, rel;  // its position, and its block row counted from the tile's first; -1 and 0 where there is none
  bool there;
};
__device__ __forceinline__ ChunkQuery chunk_query(const CacheChunkParams& p, const ChunkTileAt& x, const ChunkRows& r, int row) {
  const int64_t pos = x.pos + row;
  ChunkQuery q;
  q.there = row >= 0 && row < x.rows && pos >= r.lo && pos < r.hi;
  q.pos = q.there ? (int)pos : -1;
  q.rel = q.there ? (q.pos >> p.c.block_shift) - r.row0 : 0;
  return q;
}

// 64 tokens: of one block, or (SMALL) four pieces of 16 of the list's blocks, as a wavefront holds them.  What masks need of its pieces lies in LDS, for the last four units.
struct ChunkUnit {
  int64_t off, scale_off;    // where the wavefront's own piece begins, its scales (bytes in either pool)
  int rows;                  // tokens to read of it
  int flags;
  __device__ __forceinline__ bool on(int half) const { return flags >> half & 1; }  // some query of the wavefront attends some token of the half
  __device__ __forceinline__ bool there() const { return flags >> 3 & 1; }          // (there is no unit of no tokens)
  __device__ __forceinline__ bool some() const { return flags >> 2 & 1; }           // some query of the workgroup may not attend some token
};

// What a tile's look-ups need, in LDS: scalar registers hold it no longer than they take (see params_in_memory in cache_attn.h).
struct ChunkScope {
  ChunkRows r;
  int b, h, split;
  int first_row;      // block row of the chunk's first token, for what is counted
  int first_tile;
  int bits[4], last[4];  // of each wavefront's own queries: their block rows, the last one's position
  __device__ __forceinline__ void init(const CacheChunkParams& p, const ChunkTileAt& x, const ChunkRows& r_, int h_, int split_) {
    r = r_;
    b = x.b;
    h = h_;
    split = split_;
    first_row = (int)min(max(x.start, (int64_t)0), (int64_t)p.max_len - 1) >> p.c.block_shift;
    first_tile = x.pos == x.start || x.pos <= 0;
  }
};
// (a word of it, the same for the wavefront)
__device__ __forceinline__ int scope_word(const int& of) {
  return __builtin_amdgcn_readfirstlane(*(const volatile __attribute__((address_space(3))) int*)(uintptr_t)lds_addr(&of));
}
__device__ __forceinline__ ChunkScope scope_now(const ChunkScope& of) {
  ChunkScope s;
  s.r.lo = scope_word(of.r.lo);
  s.r.hi = scope_word(of.r.hi);
  s.r.row0 = scope_word(of.r.row0);
  s.r.n_rows = scope_word(of.r.n_rows);
  s.b = scope_word(of.b);
  s.h = scope_word(of.h);
  s.split = scope_word(of.split);
  s.first_row = scope_word(of.first_row);
  s.first_tile = scope_word(of.first_tile);
  return s;
}

// The units of a split.  In closed form the blocks that any row of the tile keeps are those of its first row and the blocks after them up to the last; lists are
// walked row by row, each block in the turn of the first row that keeps it.  Lanes look units up 64 at a time (SMALL: 16, a lane to a piece).
template <bool SMALL>
struct ChunkWalk {
  static constexpr int NB = SMALL ? 4 : 1, kTokens = 64 / NB, kUnits = 64 / NB;
  static constexpr int kRing = 4 * NB;  // pieces in LDS (a wavefront's own)
  const ChunkScope& scope;
  int wave, first, step;             // whose queries and pieces these are; unit `first` of the split, and every step-th
  uint32_t ring;                     // where the pieces lie
  int n_missing = 0;
  int turn = -1, u_now = 0, u_end = 0;
  int info = 0, at = 0;              // of this lane's unit (piece): tokens to read | block rows that keep them << 8, position of the first
  uint32_t off[2] = {0, 0}, scale_off[2] = {0, 0};
  uint64_t live = 0, some = 0, on[2] = {0, 0};

  // (scope_: in LDS, filled for the workgroup; ring_: room for kRing pairs of words there; q0, q1: a lane's first query and its last)
  __device__ __forceinline__ ChunkWalk(ChunkScope& scope_, int n_rows, int wave_, const void* ring_, const ChunkQuery& q0, const ChunkQuery& q1, int first_ = 0,
                                       int step_ = 1)
      : scope(scope_), wave(wave_), first(first_), step(step_), ring(lds_addr(ring_)) {
    if (n_rows == 0) turn = 1 << 20;  // (nothing to look up)
    int my_bits = 0;
#pragma unroll 1
    for (int i = 0; i < n_rows; ++i) my_bits |= __any((q0.there && q0.rel == i) || (q1.there && q1.rel == i)) ? 1 << i : 0;
    int last = max(q0.pos, q1.pos);
#pragma unroll
    for (int i = 1; i < 64; i *= 2) last = max(last, __shfl_xor(last, i, 64));
    // (read again by the wavefront itself)
    scope_.bits[wave] = my_bits;
    scope_.last[wave] = last;
  }

  __device__ static uint64_t of_units(uint64_t pieces) {
    if (!SMALL) return pieces;
    pieces |= pieces >> 1;
    return (pieces | pieces >> 2) & 0x1111111111111111ull;
  }

  __device__ __forceinline__ static RowBlocks blocks_of(const ChunkLookUp& p, const ChunkScope& s, int turn_) {
    RowBlocks rb = row_blocks(p, s.h, s.r.row0 + turn_);
    if (!p.row_ptr) rb.count = rb.n_stripe + (s.r.row0 + s.r.n_rows - rb.local_lo);
    return rb;
  }

  // Looks up the next units that there are; false: there are none.
  __device__ __forceinline__ bool look_up() {
    const ChunkLookUp p = chunk_look_up();
    const ChunkScope s = scope_now(scope);
    const ChunkRows& r = s.r;
    const int sh = p.block_shift, S = 1 << sh, turns = p.row_ptr ? r.n_rows : 1;
    RowBlocks rb;
    if (u_now < u_end) rb = blocks_of(p, s, turn);
    while (u_now >= u_end) {
      if (turn + 1 >= turns) return false;
      ++turn;
      rb = blocks_of(p, s, turn);
      const int units = (int)((((int64_t)rb.count << sh) + 63) >> 6);
      const int even = units / p.by_splits, rest = units - even * p.num_splits;
      u_now = even * s.split + rest * s.split / p.by_splits + first;
      u_end = even * (s.split + 1) + rest * (s.split + 1) / p.by_splits;
    }
    const int lane = lane_now();
    const int u = u_now + step * (lane / NB), l = 64 * u + 16 * (lane % NB), n = l >> sh, skip = l & (S - 1);
    u_now += step * kUnits;
    const bool inside = u < u_end && n < rb.count;
    const int blk = inside ? rb.block_of_lane(n) : 0;
    at = blk * S + skip;
    int rows = inside ? min(max(r.hi - at, 0), kTokens) : 0, bits = 0;
#pragma unroll 1
    for (int i = 0; i < r.n_rows; ++i) {
      const RowBlocks other = p.row_ptr ? row_blocks(p, s.h, r.row0 + i) : RowBlocks{};
      if (rows > 0 && row_keeps(p, other, s.h, r.row0 + i, blk, n)) {
        if (i < turn) rows = 0;  // (read in that row's turn)
        bits |= 1 << i;
      }
    }
    if (bits == 0) rows = 0;
    int page = rows > 0 ? p.table[((int64_t)s.b * p.heads + s.h) * p.max_blocks + blk] : 0;
    const bool held = page >= 0 && page < p.num_pages;
    if (__any(rows > 0 && !held) && p.missing) {
      // a block counts once: in the tile of the first of the chunk's rows that keeps it (in closed form no row drops a block and keeps it later)
      bool counts = rows > 0 && !held && skip == 0;
      if (!s.first_tile) {
        if (p.row_ptr) {
#pragma unroll 1
          for (int i = s.first_row; i < r.row0; ++i) {
            const RowBlocks other = row_blocks(p, s.h, i);
            if (counts && row_keeps(p, other, s.h, i, blk, n)) counts = false;
          }
        } else {
          counts = counts && blk * S >= r.lo;
        }
      }
      n_missing += __popcll(__ballot(counts));
    }
    if (!held) page = rows = 0;
    info = rows | bits << 8;
    const int64_t o = page * p.page + skip * p.tok, so = page * p.scale_page + skip * p.scale_tok;
    off[0] = (uint32_t)o;
    off[1] = (uint32_t)(o >> 32);
    scale_off[0] = (uint32_t)so;
    scale_off[1] = (uint32_t)(so >> 32);
    const int all = (1 << r.n_rows) - 1;
    live = of_units(__ballot(rows > 0));
    some = of_units(__ballot(rows < kTokens || bits != all || at + rows - 1 > r.lo));
    const bool mine = (bits & scope_word(scope.bits[wave])) != 0;
    const int my_last = scope_word(scope.last[wave]);
    if (SMALL) {
      const uint64_t x = __ballot(mine && rows > 0 && at <= my_last);
      on[0] = (x | x >> 1) & 0x1111111111111111ull;
      on[1] = (x >> 2 | x >> 3) & 0x1111111111111111ull;
    } else {
      on[0] = __ballot(mine && rows > 0 && at <= my_last);
      on[1] = __ballot(mine && rows > 32 && at + 32 <= my_last);
    }
    return true;
  }

  // Whether a unit with a token to read is looked up.
  __device__ __forceinline__ bool find() {
    while (live == 0)
      if (!look_up()) return false;
    return true;
  }
  // The next one of those, as unit n (SMALL: the units of a look-up are NB lanes apart): N pieces of 16 tokens from `piece` on.
  __device__ __forceinline__ void take(int n, ChunkUnit& w) { take(n, wave, &w); }
  template <int N = 1>
  __device__ __forceinline__ void take(int n, int piece, ChunkUnit* w) {
    const int i = __builtin_ctzll(live);
    live &= live - 1;
    const int mine = lane_now() - i;
    if (mine >= 0 && mine < NB)
      *(__attribute__((address_space(3))) u32x2*)(uintptr_t)(ring + 8 * ((n & 3) * NB + mine)) = u32x2{(uint32_t)info, (uint32_t)at};
#pragma unroll
    for (int t = 0; t < N; ++t) {
      const int own = SMALL ? i + piece + t : i;
      auto both = [&](const uint32_t (&x)[2]) __attribute__((always_inline)) {
        return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)x[1], own) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x[0], own));
      };
      w[t].flags = (int)(on[0] >> i & 1) | (int)(on[1] >> i & 1) << 1 | (int)(some >> i & 1) << 2 | 8;
      w[t].off = both(off);
      w[t].scale_off = both(scale_off);
      w[t].rows = __builtin_amdgcn_readlane(info, own) & 255;
    }
  }
  __device__ __forceinline__ bool next(int n, ChunkUnit& w) {
    if (find()) {
      take(n, w);
      return true;
    }
    w = ChunkUnit{};  // (no rows: loading it fetches nothing)
    return false;
  }
};

// Tokens that the query at position `pos`, in the tile's block row `rel`, attends of a piece (tokens to read | block rows << 8, position of its first), bits.
__device__ __forceinline__ uint64_t piece_seen(int info, int at, int rel, int pos) {
  const int rows = min(info & 255, pos - at + 1);
  if (!(info >> 8 >> rel & 1) || rows <= 0) return 0;
  return rows >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << rows) - 1;
}
// The same of unit n.
template <bool SMALL>
__device__ __forceinline__ uint64_t chunk_seen(const ChunkWalk<SMALL>& walk, int n, int rel, int pos) {
  constexpr int NB = ChunkWalk<SMALL>::NB;
  uint64_t seen = 0;
#pragma unroll
  for (int t = 0; t < NB; ++t) {
    const u32x2 x = *(const __attribute__((address_space(3))) u32x2*)(uintptr_t)(walk.ring + 8 * ((n & 3) * NB + t));
    seen |= piece_seen((int)x[0], (int)x[1], rel, pos) << (16 * t);
  }
  return seen;
}

// Where a row's result goes, or its part of a split: eight features from d of the tile's row `row`.
template <int D>
__device__ __forceinline__ void put_chunk_row(const CacheChunkParams& p, const ChunkTileAt& x, int h, int row, int split, int d, const float (&o)[8], float m,
                                              float l) {
  if (p.num_splits == 1) {
    bf16x8 out;
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = (__bf16)(l == 0.f ? 0.f : o[e] / l);
    *reinterpret_cast<bf16x8*>(p.o + (x.row + row) * p.q_sr + h * p.q_sh + d) = out;
    if (d == 0 && p.lse) p.lse[(int64_t)h * p.num_rows + x.row + row] = l == 0.f ? kNegInf : m * p.scale + __logf(l);
  } else {
    // (rows of a sequence are counted from its first one in the tensors)
    const int64_t at = (((int64_t)x.b * p.heads + h) * p.max_new + (x.pos - x.start) + row) * p.num_splits + split;
    f32x4* const to = reinterpret_cast<f32x4*>(p.part_acc + at * D + d);
    to[0] = f32x4{o[0], o[1], o[2], o[3]};
    to[1] = f32x4{o[4], o[5], o[6], o[7]};
    if (d == 0) {
      p.part_ml[at * 2] = m;
      p.part_ml[at * 2 + 1] = l;
    }
  }
}

// The launch for tiles of 128 rows (all but the merge of splits).
hipError_t launch_cache_chunk_wide(const CacheChunkParams& p, hipStream_t stream);

}  // namespace s2
