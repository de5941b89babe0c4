// Attention of a chunk of new tokens to each sequence over a paged cache in bf16, 8 or 4 bits that holds their keys and values already (section 4.1's cache,
// section 5.3's prefill in chunks).
//
// o_i = sum_j p_ij v_j / sum_j p_ij, p_ij = exp(scale q_i k_j - max), over the cached tokens j <= i that the block row of i keeps.  Queries of a tile share
// what they read: a tile of 16 rows makes 64 D flops of a token's K and V, so that a tile of a few rows is bound by the cache's bytes and one of 128 by
// matrix instructions.
//
// Three forms, by rows to a sequence.  Up to 32: each wavefront takes tokens of its own against all rows (cache_chunk_few.h; 64 sequences of 1 to 12 rows of
// 32 heads after 8192 to 32768 tokens, e4m3, 210 us, 5.6 TB/s).  33 to 64, below: the four wavefronts of a workgroup share a unit of 64 tokens: each
// fetches a piece of 16 of them, brings it to bf16 once and writes its K and V rows into LDS (ChunkTile); then each takes 16 queries against the whole unit (64
// sequences of 1 to 40 rows, bf16, 283 us, 5.3 TB/s; one of 40 rows after 32768 tokens, 512 workgroups of three units each, 18 us and 4 for the splits' sums).
// More: tiles of 128 rows (cache_chunk_wide_kernel.hip).  In all of them scores are formed as keys x queries, so that a lane holds one query and the
// probabilities are the second operand of the product with V as they stand.  Up to 64 rows P goes to V in two bf16 terms, 16 bits together, as in a decode step.
#include <hip/hip_runtime.h>

#include "cache_chunk.h"
#include "cache_chunk_few.h"
#include "config.h"

namespace s2 {

namespace {

// Up to 16 * NQ queries of one (sequence, head), one split of what they attend.
template <int D, int FMT, int NQ, bool SMALL>
__global__ __launch_bounds__(256, NQ == 2 ? (D == 64 ? 3 : 2) : D == 64 ? 4 : FMT == S2_KV_BF16 ? 2 : 3) void cache_chunk_few_kernel(const CacheChunkParams p) {
  __shared__ ChunkFewShared<D, NQ, SMALL> sh;
  const int th = blockIdx.x / p.by_splits, split = blockIdx.x - th * p.num_splits;
  const int tile = th / p.by_heads, h = th - tile * p.heads;
  const ChunkTileAt x = chunk_tile_at(p, tile);
  if (x.rows <= 0) return;
  const ChunkRows r = chunk_block_rows(p, x);
  chunk_few<D, FMT, NQ, SMALL>(p, x, r, h, split, sh);
}

// A workgroup: 64 queries of one (sequence, head), one split of what they attend.
template <int D, int FMT, bool SMALL>
__global__ __launch_bounds__(256, D == 64 ? 4 : 3) void cache_chunk_kernel(const CacheChunkParams p) {
  using Rows = CacheRows<D, FMT>;
  using Tile = ChunkTile<D>;
  using Pieces = ChunkWalk<SMALL>;
  constexpr int W = 4, KK = D / 32, FT = D / 16, kOdd = FT / 4 * 64;
  constexpr int RS = D + 4;           // floats to a row where results are turned
  static_assert(W * 16 * RS * 4 <= 2 * Tile::kBytes, "the wavefronts' sums fit where K and V were");

  __shared__ __align__(16) uint16_t sh_kv[2][Tile::kElems];
  __shared__ u32x2 sh_pieces[W][Pieces::kRing];
  __shared__ ChunkScope sh_scope;
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
  const ChunkRows r = chunk_block_rows(p, x);
  const int row_q = 16 * wave + c;
  const ChunkQuery q = chunk_query(p, x, r, row_q);
  bf16x8 qf[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk)
    qf[kk] = q.there ? *reinterpret_cast<const bf16x8*>(p.q + (x.row + row_q) * p.q_sr + h * p.q_sh + 32 * kk + 8 * g) : bf16x8{};
  const bool any_q = __any(q.there);

  for (int i = tid; i < W * kOdd; i += 64 * W) sh_odd[i] = 0;
  if (tid == 0) {
    sh_any_odd = sh_unit_odd[0] = sh_unit_odd[1] = 0;
    sh_scope.init(p, x, r, h, split);
  }
  __syncthreads();

  f32x4 acc[FT];
  float m_run = kNegInf, l_run = 0.f;
#pragma unroll
  for (int ft = 0; ft < FT; ++ft) acc[ft] = f32x4{};

  const uint32_t at_k = lds_addr(sh_kv[0]), at_v = lds_addr(sh_kv[1]);
  // (writes without bank conflicts: see cache_attn_shared_kernel.hip)
  const bool turned = ((c >> 3 ^ c >> 2) & 1) != 0;
  const int gw = FMT == S2_KV_BF16 && turned ? g ^ 1 : g;
  const uint32_t write = (16 * wave + c) * Tile::RB;
  const uint32_t k_read = at_k + Tile::row_lane(lane), v_read = at_v + Tile::tr_lane(lane);
  Pieces walk(sh_scope, r.n_rows, wave, sh_pieces[wave], q, q);

  typename Rows::Part kr, vr;
  auto load = [&](auto is_v, const ChunkUnit& w, typename Rows::Part& to) __attribute__((always_inline)) {
    constexpr bool V = decltype(is_v)::value;
    const uint8_t* const at = (V ? p.c.v : p.c.k) + w.off;
    const uint8_t* const scale_at = Rows::kScaled ? (V ? p.c.vs : p.c.ks) + w.scale_off : nullptr;
    Rows::load(to, at, scale_at, w.rows, p.c.tok, p.c.scale_tok, (SMALL ? 0 : 16 * wave) + c, gw);
  };
  constexpr std::false_type kK{};
  constexpr std::true_type kV{};
  auto put_part = [&](auto is_v, const typename Rows::Part& part, uint32_t to, bool some, int turn) __attribute__((always_inline)) {
    const int turn_of = Rows::kScaled && turned ? 16 : 0;
    u32x4 rows[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      rows[kk] = Rows::operand(part, g, kk, turned ? ~0u : 0u);
      *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(to + write + (kk % 2 ? -turn_of : turn_of) + 2 * Rows::feature(kk, gw)) = rows[kk];
    }
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

  auto attend = [&](const ChunkUnit& w, int n) __attribute__((always_inline)) {
    const bool odd = w.some() && sh_unit_odd[n & 1];  // (the same for all wavefronts)
    f32x4 s[4];
    if (any_q) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          const bf16x8 k = __builtin_bit_cast(bf16x8, lds_read16(k_read, Tile::row_off(t, kk)));
          s[t] = mfma16(k, qf[kk], kk ? s[t] : f32x4{});
        }
      uint64_t seen = 0;
      if (w.some()) {
        seen = chunk_seen<SMALL>(walk, n, q.rel, q.pos);
#pragma unroll
        for (int t = 0; t < 4; ++t) mask_scores(s[t], seen, t, g);
      }
      float mx = kNegInf;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[t][e]);
      mx = max_halves(max_rows(mx));
      const float m_new = fmaxf(m_run, mx);
      const float mc = m_new == kNegInf ? 0.f : m_new * cl;
      if (__any(m_new > m_run)) {
        const float alpha = m_new > m_run ? fast_exp2(m_run * cl - mc) : 1.f;  // (see cache_attn_kernel.hip)
        l_run *= alpha;
        m_run = m_new;
#pragma unroll
        for (int ft = 0; ft < FT; ++ft) acc[ft] *= alpha;
      }
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[t][e] = fast_exp2(__builtin_fmaf(s[t][e], cl, -mc));
          l_run += s[t][e];
        }
      if (odd) {
#pragma unroll 1
        for (int u = 0; u < 2; ++u) count_odd<D>(v_read + 32 * u * Tile::RB, (uint32_t)(seen >> (32 * u)), sh_odd + wave * kOdd, &sh_any_odd, lane);
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
      bf16x8 pf, pr;
      two_terms(s[2 * u], s[2 * u + 1], pf, pr);
#pragma unroll
      for (int ft = 0; ft < FT; ++ft) {
        const bf16x8 vf = __builtin_bit_cast(bf16x8, lds_read_tr2(v_read, v_read, Tile::tr_off(u, ft), Tile::tr_off(u, ft) + 16 * Tile::RB));
        acc[ft] = mfma16(vf, pf, mfma16(vf, pr, acc[ft]));
      }
    }
  };

  {
    ChunkUnit w;
    bool more = walk.next(0, w);
    load(kK, w, kr);
    load(kV, w, vr);
    for (int n = 0; more; ++n) {
      ChunkUnit next;
      more = walk.next(n + 1, next);
      barrier();  // nobody reads the unit before any more
      put_part(kK, kr, at_k, false, n & 1);
      put_part(kV, vr, at_v, w.some(), n & 1);
      if (tid == 0) sh_unit_odd[~n & 1] = 0;
      load(kK, next, kr);
      load(kV, next, vr);
      barrier();
      attend(w, n);
      w = next;
    }
  }
  const CacheChunkParams& pe = chunk_params();
  if (pe.missing && tid == 0 && walk.n_missing > 0) atomicAdd(pe.missing, walk.n_missing);

  // results from query-on-lane to rows, through where K and V were
  l_run = sum_groups(l_run);
  if (g == 0) {
    sh_m[wave][c] = q.there ? m_run : kNegInf;
    sh_l[wave][c] = q.there ? l_run : 0.f;
  }
  __syncthreads();
  float* const sums = reinterpret_cast<float*>(sh_kv[0]);
  float* const mine = sums + row_q * RS + 4 * g;
#pragma unroll
  for (int ft = 0; ft < FT; ++ft) *reinterpret_cast<f32x4*>(mine + 16 * ft) = q.there ? acc[ft] : f32x4{};
  if (sh_any_odd && q.there) add_odd<D>(mine, sh_odd + wave * kOdd, lane);
  __syncthreads();
  constexpr int TPR = D / 8;  // threads to a query, eight features each
  for (int i = tid / TPR; i < x.rows; i += 64 * W / TPR) {
    const int d = 8 * (tid % TPR);
    float o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = sums[i * RS + d + e];
    put_chunk_row<D>(pe, x, h, i, split, d, o, sh_m[i / 16][i % 16], sh_l[i / 16][i % 16]);
  }
}

// Merges the splits, a wavefront to a row (see cache_attn_kernel.hip; 1280 rows of 16 splits 4.1 us, with a load at a time 5.7).  Rows that sequences may have, or, of up to 64
// sequences that have fewer, those that there are (406 of 7 sequences of up to 333, 13 heads: 5.3 us and 4.7).
template <int D>
__global__ __launch_bounds__(256) void cache_chunk_merge_kernel(const CacheChunkParams p) {
  constexpr int LPR = D / 4, NG = 64 / LPR;
  const int lane = threadIdx.x & 63, g = lane / LPR, c = lane % LPR, n = p.num_splits;
  const int of = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int b, h, i;
  if (!p.merge_rows) {
    const int bh = of / p.by_new;
    i = of - bh * p.max_new;
    if (bh >= p.nseq * p.heads) return;
    b = bh / p.by_heads;
    h = bh - b * p.heads;
  } else {
    const int row = of / p.by_heads;
    if (row >= p.num_rows) return;
    h = of - row * p.heads;
    // the last sequence whose rows begin there or before
    const bool is = lane < p.nseq;
    const uint64_t before = __ballot(is && p.cu[is ? lane : 0] <= row);
    if (!before) return;
    b = 63 - __builtin_clzll(before);
    i = -1;
  }
  const int lo = load_const<int32_t>(p.cu + b), hi = load_const<int32_t>(p.cu + b + 1);
  const int from = min(max(lo, 0), p.num_rows);
  if (i < 0) i = of / p.by_heads - from;
  if (i >= chunk_rows(p, lo, hi)) return;
  const int64_t item = ((int64_t)b * p.heads + h) * p.max_new + i;
  const float* const ml = p.part_ml + item * n * 2;
  const f32x4* const part = reinterpret_cast<const f32x4*>(p.part_acc) + item * n * LPR + c;
  const float ms = lane < n ? ml[2 * lane] : kNegInf, ls = lane < n ? ml[2 * lane + 1] : 0.f;
  // (kEach loads on their way at a time, the first ones along with the statistics)
  constexpr int kEach = 4;
  f32x4 y[kEach];
  auto load = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < kEach; ++k) y[k] = part[(int64_t)min(s0 + k * NG + g, n - 1) * LPR];
  };
  load(0);
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
    for (int k = 0; k < kEach; ++k) {
      const int s = s0 + k * NG + g;
      const float of = __shfl(weight, s & 63, 64);
      if (s < n) a += y[k] * of;
    }
    s0 += kEach * NG;
    if (s0 >= n) break;
    load(s0);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (LPR == 16) a[e] = sum_rows(a[e]);
    a[e] = sum_halves(a[e]);
  }
  if (lane >= LPR) return;
  bf16x4 out;
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = (__bf16)(l == 0.f ? 0.f : a[e] / l);
  const int64_t row = from + i;
  *reinterpret_cast<bf16x4*>(p.o + row * p.q_sr + h * p.q_sh + 4 * c) = out;
  if (lane == 0 && p.lse) p.lse[(int64_t)h * p.num_rows + row] = l == 0.f ? kNegInf : m * p.scale + __logf(l);
}

template <int D, int FMT>
void launch_blocks(const CacheChunkParams& p, hipStream_t stream) {
  const dim3 grid(p.num_tiles * p.heads * p.num_splits), block(256);
  const bool small = p.block_size < 64;
  if (p.max_new > 32) {
    if (small)
      hipLaunchKernelGGL((cache_chunk_kernel<D, FMT, true>), grid, block, 0, stream, p);
    else
      hipLaunchKernelGGL((cache_chunk_kernel<D, FMT, false>), grid, block, 0, stream, p);
  } else if (p.max_new > 16) {
    if (small)
      hipLaunchKernelGGL((cache_chunk_few_kernel<D, FMT, 2, true>), grid, block, 0, stream, p);
    else
      hipLaunchKernelGGL((cache_chunk_few_kernel<D, FMT, 2, false>), grid, block, 0, stream, p);
  } else {
    if (small)
      hipLaunchKernelGGL((cache_chunk_few_kernel<D, FMT, 1, true>), grid, block, 0, stream, p);
    else
      hipLaunchKernelGGL((cache_chunk_few_kernel<D, FMT, 1, false>), grid, block, 0, stream, p);
  }
}

template <int D>
hipError_t launch_dim(const CacheChunkParams& p, hipStream_t stream) {
  hipError_t e;
  if (p.tile_shift > 6) {
    e = launch_cache_chunk_wide(p, stream);
  } else {
    switch (p.c.format) {
      case S2_KV_BF16: launch_blocks<D, S2_KV_BF16>(p, stream); break;
      case S2_KV_MXFP8: launch_blocks<D, S2_KV_MXFP8>(p, stream); break;
      default: launch_blocks<D, S2_KV_MXFP4>(p, stream); break;
    }
    e = hipGetLastError();
  }
  if (e != hipSuccess || p.num_splits == 1) return e;
  const int64_t rows = (int64_t)p.heads * (p.merge_rows ? p.num_rows : (int64_t)p.nseq * p.max_new);
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
  p.sorted = p.nseq > 1 && p.nseq <= 64;
  p.seq_tiles = (int)each;
  p.num_tiles = (int)std::min<int64_t>(tiles, kMostGroups + 1);
  return tiles;
}

hipError_t launch_cache_chunk(const CacheChunkParams& params, hipStream_t stream) {
  CacheChunkParams p = params;
  p.by_heads = fast_div(p.heads);
  p.by_splits = fast_div(p.num_splits);
  p.by_new = fast_div(p.max_new);
  p.merge_rows = p.nseq > 1 && p.nseq <= 64 && p.num_rows < (int64_t)p.nseq * p.max_new;
  p.by_stride = fast_div(p.stride > 0 ? p.stride : 1);
  p.by_tiles = fast_div(std::max(p.seq_tiles - 1, 1));
  ChunkLookUp& l = p.look_up;
  l.table = p.c.table;
  l.page = p.c.page;
  l.scale_page = p.c.scale_page;
  l.row_ptr = p.row_ptr;
  l.col_idx = p.col_idx;
  l.missing = p.missing;
  l.tok = p.c.tok;
  l.scale_tok = p.c.scale_tok;
  l.max_blocks = p.c.max_blocks;
  l.num_pages = p.c.num_pages;
  l.block_shift = p.c.block_shift;
  l.heads = p.heads;
  l.num_splits = p.num_splits;
  l.local_blocks = p.local_blocks;
  l.stride = p.stride;
  l.window_blocks = p.window_blocks;
  l.dense = p.dense;
  l.head_index_base = p.head_index_base;
  l.num_blocks = p.num_blocks;
  l.by_splits = p.by_splits;
  l.by_stride = p.by_stride;
  return p.c.head_dim == 128 ? launch_dim<128>(p, stream) : launch_dim<64>(p, stream);
}

}  // namespace s2
