// Rows written into a paged cache, quantised on the way, and read back (section 4.1's cache in bf16, 8 or 4 bits).
//
// One power of two to 32 features of a row: with a the largest magnitude, 2^e is the smallest for which a * 2^-e rounds into the code's
// range (below 464 in e4m3, 7 in e2m1).  bf16 magnitudes order as their bit patterns do, so a is an integer maximum over
// four lanes of eight features, and e the exponent field of a + (what carries a mantissa of 1.8125 or 1.75 into the next exponent).
// Scaling by a power of two is exact: the one rounding is that of the conversion instruction, and what is read back is exact in bf16.
//
// Both move bytes and nothing else; D/8 lanes take a row, 16 bytes of bf16 each.  A whole cache read back moves 5.0 TB/s (32 heads of 32768 x 128 over
// e4m3, 162 us; a kernel that only streams, a byte read to two written, reaches 6.3 at this size), prompts written 4.6 (8 of 1001 to 16384 tokens over e4m3, of
// which the mask keeps a few blocks in a hundred, 50 us; such a kernel 5.7); the tokens of a decode step are a launch, 4 us.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <limits>

#include "kernels.h"
#include "kv_cache.h"

namespace s2 {

namespace {

// Tile `i` of a call: rows [row, row + p.tile_rows) of the n of sequence b, which begin at lo of the batch's numbering and at position `start`, for
// p.tile_heads heads from `head`.
struct Tile {
  int b, row, head, lo, n, start;
};
// Either each sequence has as many tiles as the longest may need, or (packed) there are those of the rows that there are: then sequence b, whose rows
// begin at lo, has the tiles from lo / tile_rows + b on, one more at most than its rows need, and the last sequence that begins at or before a tile is
// found 64 at a time.  Of single rows it has those from lo on, and no tile without a row is between them.
__device__ __forceinline__ Tile tile_of(const KvRowsParams& p, int i) {
  Tile s;
  const int groups = p.by_heads_groups;  // tiles side by side take heads of the same rows
  const int t = i / p.div_groups;
  s.head = (i - t * groups) * p.tile_heads;
  if (!p.packed) {
    s.b = t / p.div_tiles;
    s.row = (t - s.b * p.row_tiles) * p.tile_rows;
    s.lo = load_const<int32_t>(p.cu + s.b);
    s.n = min(load_const<int32_t>(p.cu + s.b + 1) - s.lo, p.max_rows);
    s.start = load_const<int32_t>(p.start + s.b);
    return s;
  }
  const int lane = threadIdx.x & 63;
  int first = 0, count = p.nseq;
  for (;;) {
    const int step = (count + 63) >> 6;
    const bool is = lane * step < count;
    const int b = first + (is ? lane * step : 0);
    const int lo = p.cu[b], hi = p.cu[b + 1], start = p.start[b];
    const int tile = (min(max(lo, 0), p.bound) >> p.tile_shift) + (p.tile_shift ? b : 0);
    const int before = __popcll(__ballot(is && tile <= t));
    const int last = max(before - 1, 0);
    if (step == 1) {
      s.b = first + last;
      s.lo = __builtin_amdgcn_readlane(lo, last);
      s.start = __builtin_amdgcn_readlane(start, last);
      const int from = min(max(s.lo, 0), p.bound) - s.lo, end = min(max(__builtin_amdgcn_readlane(hi, last), 0), p.bound) - s.lo;
      s.row = from + (t - __builtin_amdgcn_readlane(tile, last)) * p.tile_rows;
      s.n = before ? min(end, p.max_rows) : 0;
      if (!before) s.row = 0;
      return s;
    }
    first += last * step;
    count = min(step, count - last * step);
  }
}

// A lane's eight features of a row, quantised, to `pool` (+ its lane's bytes) and the scale's byte to `scale` (a lane in four).
template <int D, int FMT>
__device__ __forceinline__ void put_row(const u32x4& x, int c, uint8_t* pool, uint8_t* scale_to) {
  if constexpr (FMT == S2_KV_BF16) {
    *reinterpret_cast<u32x4*>(pool + 16 * c) = x;
  } else {
    uint32_t a = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) a = max(a, max(x[e] & 0x7fffu, (x[e] >> 16) & 0x7fffu));
    a = max(a, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0xB1, 0xf, 0xf, true));  // (quads of lanes: 1032, 2301)
    a = max(a, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0x4E, 0xf, 0xf, true));
    constexpr int kCarry = FMT == S2_KV_MXFP8 ? 24 : 32, kTop = FMT == S2_KV_MXFP8 ? 8 : 2;
    const bool held = a < 0x7f00u;
    const uint32_t byte = held ? (uint32_t)max((int)((a + kCarry) >> 7) - kTop, 17) : 255u;
    const float scale = scale_of(held ? byte : 127u);
    if constexpr (FMT == S2_KV_MXFP8) {
      u32x2 w;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        s16x2_ r = {0, 0};
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, two_of(x[2 * e]), scale, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, two_of(x[2 * e + 1]), scale, true);
        w[e] = held ? __builtin_bit_cast(uint32_t, r) : 0u;
      }
      *reinterpret_cast<u32x2*>(pool + 8 * c) = w;
    } else {
      uint32_t w = 0;
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, two_of(x[0]), scale, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, two_of(x[1]), scale, 1);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, two_of(x[2]), scale, 2);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, two_of(x[3]), scale, 3);
      *reinterpret_cast<uint32_t*>(pool + 4 * c) = held ? w : 0u;
    }
    if (c % 4 == 0) scale_to[c / 4] = (uint8_t)byte;
  }
}

// A tile is a wavefront's: a lane looks up the page of one of its (row, head) pairs, and what then moves, 64 * 8 / D pairs to an instruction and two such
// in flight at a time, are those that the cache holds: of a long prompt it is a few, and a tile without one costs a lookup.
template <int D, int FMT>
__global__ __launch_bounds__(256) void kv_append_kernel(const KvRowsParams p) {
  constexpr int LPR = D / 8, RPI = 64 / LPR;  // lanes to a row, rows to an instruction
  const int lane = threadIdx.x & 63, c = lane % LPR, mine = lane / LPR;
  const int at = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (at >= p.num_tiles) return;
  if (p.packed && p.skipped && at == 0) {  // what no tile is for: items that are none
    int none = 0;
    for (int b = lane; b < p.nseq; b += 64) {
      const int lo = p.cu[b], n = min(p.cu[b + 1] - lo, p.max_rows);
      const int from = min(max(-lo, 0), max(n, 0)), end = max(min(n, p.bound - lo), from);
      none += max(n, 0) - (end - from);
    }
    for (int x = 32; x; x >>= 1) none += __shfl_xor(none, x, 64);
    if (lane == 0 && none > 0) atomicAdd(p.skipped, none * p.c.heads);
  }
  const Tile s = tile_of(p, at);
  if (s.row >= s.n) return;
  // my pair
  const int pairs = p.tile_rows * p.tile_heads;
  const int head = s.head + (lane >> p.tile_shift), item = s.row + (lane & (p.tile_rows - 1));
  const bool there = lane < pairs && item < s.n && head < p.c.heads;
  const int64_t pos = (int64_t)s.start + item, blk = pos >> p.c.block_shift;
  const int in_page = (int)(pos & ((1 << p.c.block_shift) - 1));
  int row = s.lo + item, page = -1;
  if (there && pos >= 0 && blk < p.c.max_blocks) page = p.c.table[((int64_t)s.b * p.c.heads + head) * p.c.max_blocks + blk];
  if (there && p.rows) row = row >= 0 && row < p.num_items ? p.rows[row] : -1;
  const bool held = row >= 0 && row < p.num_rows && page >= 0 && page < p.c.num_pages;
  if (p.skipped) {
    const int left_out = __popcll(__ballot(there && !held));
    if (lane == 0 && left_out > 0) atomicAdd(p.skipped, left_out);
  }
  for (uint64_t todo = __ballot(held); todo;) {
    constexpr int NI = 2;
    u32x4 x[NI][2];
    int from[NI];
    bool good[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      // pairs that are held, RPI at a time: the one of my lanes
      from[i] = 0;
      good[i] = false;
#pragma unroll
      for (int r = 0; r < RPI; ++r) {
        if (mine == r) {
          from[i] = todo ? __builtin_ctzll(todo) : 0;
          good[i] = todo != 0;
        }
        todo &= todo - 1;
      }
      const int r = __shfl(row, from[i], 64);
      const int64_t src = r * p.stride_row + (s.head + (from[i] >> p.tile_shift)) * p.stride_head + 8 * c;
#pragma unroll
      for (int kv = 0; kv < 2; ++kv)
        if (good[i]) x[i][kv] = *reinterpret_cast<const u32x4*>((kv ? p.v : p.k) + src);
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int pg = __shfl(page, from[i], 64), in = __shfl(in_page, from[i], 64);
      const int64_t to = pg * p.c.page + (int64_t)in * p.c.tok, scale_to = pg * p.c.scale_page + (int64_t)in * p.c.scale_tok;
      if (!good[i]) continue;
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) put_row<D, FMT>(x[i][kv], c, (kv ? p.c.v : p.c.k) + to, (kv ? p.c.vs : p.c.ks) + scale_to);
    }
  }
}

template <int D, int FMT>
__global__ __launch_bounds__(256) void kv_read_kernel(const KvRowsParams p) {
  constexpr int LPR = D / 8, RPI = 256 / LPR;
  const Tile s = tile_of(p, blockIdx.x);
  const int tid = threadIdx.x, c = tid % LPR, first = tid / LPR;
  for (int i = first; i < p.tile_rows * p.tile_heads; i += RPI) {
    const int head = s.head + i / p.tile_rows, item = s.row + i % p.tile_rows;
    if (item >= s.n || head >= p.c.heads) continue;
    const int row = s.lo + item;
    if (row < 0 || row >= p.num_rows) continue;
    const int64_t pos = (int64_t)s.start + item, blk = pos >> p.c.block_shift;
    int page = -1;
    if (pos >= 0 && blk < p.c.max_blocks) page = p.c.table[((int64_t)s.b * p.c.heads + head) * p.c.max_blocks + blk];
    const bool held = page >= 0 && page < p.c.num_pages;
    const int in_page = (int)(pos & ((1 << p.c.block_shift) - 1));
    const int64_t from = page * p.c.page + (int64_t)in_page * p.c.tok;
    const int64_t scale_from = page * p.c.scale_page + (int64_t)in_page * p.c.scale_tok + c / 4;
    const int64_t to = row * p.stride_row + head * p.stride_head + 8 * c;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      const uint8_t* const pool = (kv ? p.c.v : p.c.k) + from;
      u32x4 x = {};
      if (held) {
        if constexpr (FMT == S2_KV_BF16) {
          x = *reinterpret_cast<const u32x4*>(pool + 16 * c);
        } else {
          const float scale = scale_of((kv ? p.c.vs : p.c.ks)[scale_from]);
          if constexpr (FMT == S2_KV_MXFP8) {
            const u32x2 w = *reinterpret_cast<const u32x2*>(pool + 8 * c);
            uint32_t lo2[2], hi2[2];
            values8(w[0], scale, lo2);
            values8(w[1], scale, hi2);
            x = u32x4{lo2[0], lo2[1], hi2[0], hi2[1]};
          } else {
            x = values4(*reinterpret_cast<const uint32_t*>(pool + 4 * c), scale);
          }
        }
      }
      *reinterpret_cast<u32x4*>((kv ? p.v_out : p.k_out) + to) = x;
    }
  }
}

template <int D, int FMT>
hipError_t launch_rows(const KvRowsParams& p, hipStream_t stream) {
  if (p.k_out)
    hipLaunchKernelGGL((kv_read_kernel<D, FMT>), dim3(p.num_tiles), dim3(256), 0, stream, p);
  else
    hipLaunchKernelGGL((kv_append_kernel<D, FMT>), dim3((p.num_tiles + 3) / 4), dim3(256), 0, stream, p);
  return hipGetLastError();
}

template <int D>
hipError_t launch_format(const KvRowsParams& p, hipStream_t stream) {
  switch (p.c.format) {
    case S2_KV_BF16: return launch_rows<D, S2_KV_BF16>(p, stream);
    case S2_KV_MXFP8: return launch_rows<D, S2_KV_MXFP8>(p, stream);
    default: return launch_rows<D, S2_KV_MXFP4>(p, stream);
  }
}

}  // namespace

int64_t kv_rows_groups(KvRowsParams& p) {
  // Pairs of a row and a head to a tile: one to each D/8 lanes of a workgroup that reads (32 at D = 64, where with 16 half of the lanes had none: 32 heads of 32768
  // over e2m1 73 us instead of 81, 16 of 8192 over e4m3 300 instead of 314), 16 of a wavefront that writes (8 prompts over e4m3: 8 53 us, 16 50, 32 54, 64 61: with
  // more the last ones run alone, with fewer more is looked up at a time than moved), or fewer where there would not be eight wavefronts to a compute unit.
  // A sequence's tiles are for the rows that the longest may have, or, where that is less than a third of them, a batch's are for the rows that there are: a tile
  // without rows costs less than a tile's search for its sequence.  us, for the longest and for the rows that there are: 8 prompts over e4m3 whose tiles have rows to
  // 21 % 13.9 and 12.0, 30 % 16.3 and 15.2, 39 % 17.7 and 18.1, 47 % 49.0 and 50.7, 82 % 27.0 and 33.4; read back 98 and 87, 123 and 118, 149 and 151, -, 271 and
  // 314; 63 sequences of a token and one of 8192 (1.8 %) 63 and 11, read back 387 and 21.
  auto tiles = [&](int pairs) {
    auto shape = [&](int64_t rows) {
      p.tile_shift = 0;
      while ((1 << p.tile_shift) < pairs && (1 << p.tile_shift) < rows) ++p.tile_shift;
      p.tile_rows = 1 << p.tile_shift;
      p.tile_heads = pairs / p.tile_rows;
      p.by_heads_groups = (p.c.heads + p.tile_heads - 1) / p.tile_heads;
    };
    shape(std::min<int64_t>(p.max_rows, ((int64_t)p.bound + p.nseq - 1) / p.nseq));
    const int64_t of_all = p.tile_shift ? (p.bound >> p.tile_shift) + (int64_t)p.nseq : std::max(p.bound, 1);
    const int64_t packed = of_all * p.by_heads_groups;
    p.packed = true;
    p.row_tiles = (int)std::min<int64_t>(of_all, std::numeric_limits<int32_t>::max());
    const KvRowsParams by_rows = p;
    shape(p.max_rows);
    p.row_tiles = (int)(((int64_t)p.max_rows + p.tile_rows - 1) / p.tile_rows);
    const int64_t by_longest = (int64_t)p.nseq * p.row_tiles * p.by_heads_groups;
    p.packed = 3 * packed < by_longest || (p.k_out ? by_longest : (by_longest + 3) / 4) > kMostGroups;
    if (!p.packed) return by_longest;
    p = by_rows;
    return packed;
  };
  int pairs = p.k_out ? 2048 / p.c.head_dim : 16;
  while (!p.k_out && pairs > 512 / p.c.head_dim && tiles(pairs) < 2048) pairs /= 2;
  const int64_t n = tiles(pairs);
  p.div_groups = fast_div(p.by_heads_groups);
  p.div_tiles = fast_div(p.row_tiles);
  p.num_tiles = (int)std::min<int64_t>(n, std::numeric_limits<int32_t>::max());
  return p.k_out ? n : (n + 3) / 4;
}

hipError_t launch_kv_rows(const KvRowsParams& p, hipStream_t stream) {
  return p.c.head_dim == 128 ? launch_format<128>(p, stream) : launch_format<64>(p, stream);
}

}  // namespace s2
