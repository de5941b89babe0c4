// Attention over a paged cache for more than 32 queries to a sequence (see cache_attn_kernel.hip for the mathematics and the operands' layouts).
//
// A tile of 16 queries needs 32 accumulators a lane (D = 128), so that one wavefront holds two tiles at most without spilling; and a wavefront to each
// tile with K and V of its own would fetch and dequantise the cache once per tile.  So the four wavefronts of a workgroup share a unit of 64 tokens: each
// fetches a piece of 16 of them, brings it to bf16 once and writes its K and V rows into LDS (ChunkTile: row reads and transpose reads of these
// fragments without bank conflicts); then each takes one tile of queries against the whole unit.  The next unit's bytes are on their way while this one
// is worked on; two barriers a unit, whose waits other workgroups of the compute unit fill.
//
// 64 nodes of 16 sequences over bf16 (32 heads of 31 to 46 blocks of 64 tokens, D = 128) take 130 us, 4.8 TB/s.  Over 4 bits it is the compute unit: vector
// instructions take 53 % of a SIMD's cycles, matrix instructions 32 %, the LDS is busy 35 % of the time (a unit is 32 KB of writes and 128 KB of reads), in one chain a
// unit; 64 nodes of 64 sequences 293 us, of which the bytes are 115 (with bank conflicts in the writes 10 more).  Loads two units ahead: 1 % faster for 64 sequences over bf16, else up to 13 % slower.
#include <hip/hip_runtime.h>

#include "cache_attn.h"
#include "config.h"

namespace s2 {

namespace {

// Wavefronts to a SIMD that the registers are limited for: as many as fit without spilling.
constexpr int waves_for(int D) { return D == 64 ? 4 : 3; }

template <int D, int FMT, bool SMALL>
__global__ __launch_bounds__(256, waves_for(D)) void cache_attn_shared_kernel(const CacheAttnParams p) {
  using Rows = CacheRows<D, FMT>;
  using Tile = ChunkTile<D>;
  constexpr int W = 4, KK = D / 32, FT = D / 16;
  constexpr int RS = D + 4;           // floats to a row where results are turned
  static_assert(W * 16 * RS * 4 <= 2 * Tile::kBytes, "the wavefronts' sums fit where K and V were");

  __shared__ __align__(16) uint16_t sh_kv[2][Tile::kElems];
  __shared__ float sh_m[W][16], sh_l[W][16];
  __shared__ uint32_t sh_odd[W * FT / 4 * 64];  // (count_odd)
  __shared__ uint32_t sh_any_odd, sh_unit_odd[2];

  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int item = blockIdx.x;
  const int bh = item / p.by_splits, split = item - bh * p.num_splits;
  const int b = bh / p.by_heads, h = bh - b * p.heads;
  const float cl = p.scale_log2e;

  int L = load_const<int32_t>(p.seq_lens + b);
  L = min(max(L, 0), p.max_len);
  const Nodes nodes = nodes_of(p, b, L, lane);
  // the query of my column
  const int node = 16 * wave + c;
  const int rel_q = __shfl(nodes.rel, node, 64);
  const bool there_q = nodes.all >> node & 1;
  const bool any_q = (nodes.all >> (16 * wave) & 0xffff) != 0;
  bf16x8 qf[KK];  // (features as K lies in LDS: 32 kk + 8 g ..)
#pragma unroll
  for (int kk = 0; kk < KK; ++kk)
    qf[kk] = there_q ? *reinterpret_cast<const bf16x8*>(p.q + b * p.q_ss + h * p.q_sh + node * p.q_sn + 32 * kk + 8 * g) : bf16x8{};

  for (int i = tid; i < W * FT / 4 * 64; i += 64 * W) sh_odd[i] = 0;
  if (tid == 0) sh_any_odd = sh_unit_odd[0] = sh_unit_odd[1] = 0;

  f32x4 acc[FT];
  float m_run = kNegInf, l_run = 0.f;
#pragma unroll
  for (int ft = 0; ft < FT; ++ft) acc[ft] = f32x4{};

  const uint32_t at_k = lds_addr(sh_kv[0]), at_v = lds_addr(sh_kv[1]);
  // ChunkTile's stride suits its reads; in writes of 16 bytes two rows 8 apart meet in the same banks, unless one of them writes the 16 bytes beside those that
  // the other writes.  So half of the rows take these the other way round: another quarter of the row (bf16) or the two operands of 32 bytes exchanged.
  const bool turned = ((c >> 3 ^ c >> 2) & 1) != 0;
  const int gw = FMT == S2_KV_BF16 && turned ? g ^ 1 : g;
  const uint32_t write = (16 * wave + c) * Tile::RB;
  const uint32_t k_read = at_k + Tile::row_lane(lane), v_read = at_v + Tile::tr_lane(lane);
  Walk<SMALL> walk(b, h, L, nodes, split, 0, 1, wave);

  typename Rows::Part kr, vr;
  // My piece of a unit.
  auto load = [&](auto is_v, const Unit<SMALL>& w, typename Rows::Part& x) __attribute__((always_inline)) {
    constexpr bool V = decltype(is_v)::value;
    const int page = w.my_page[0], skip = Unit<SMALL>::skip(w.my_info[0]);
    const uint8_t* const at = (V ? p.c.v : p.c.k) + page * p.c.page + skip * p.c.tok;
    const uint8_t* const scale_at = Rows::kScaled ? (V ? p.c.vs : p.c.ks) + page * p.c.scale_page + skip * p.c.scale_tok : nullptr;
    Rows::load(x, at, scale_at, Unit<SMALL>::rows(w.my_info[0]), p.c.tok, p.c.scale_tok, (SMALL ? 0 : 16 * wave) + c, gw);
  };
  constexpr std::false_type kK{};
  constexpr std::true_type kV{};
  auto put = [&](auto is_v, const u32x4 (&rows)[KK], uint32_t to, int turn_of, bool mixed, int turn) __attribute__((always_inline)) {
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
      *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(to + write + (kk % 2 ? -turn_of : turn_of) + 2 * Rows::feature(kk, gw)) = rows[kk];
    if (decltype(is_v)::value && mixed) {
      asm volatile("");  // (else looked for in every unit)
      if (odd_bits(rows)) sh_unit_odd[turn] = 1;
    }
  };
  auto put_part = [&](auto is_v, typename Rows::Part& x, uint32_t to, bool mixed, int turn) __attribute__((always_inline)) {
    u32x4 rows[KK];
    if constexpr (Rows::kScaled) Rows::turn(x, turned);
    Rows::operands(x, g, rows);
    put(is_v, rows, to, Rows::kScaled && turned ? 16 : 0, mixed, turn);
  };
  // (what it has asked of the LDS is done before a wavefront is past it; loads from memory stay on their way)
  auto barrier = [&]() __attribute__((always_inline)) {
    wait_lds();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  // A unit in LDS against my queries.
  auto attend = [&](bool some, bool mixed, int turn, auto see) __attribute__((always_inline)) {
    const bool odd = mixed && sh_unit_odd[turn];  // (the same for all wavefronts)
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
      if (some) {
        seen = see();
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
        for (int u = 0; u < 2; ++u) count_odd<D>(v_read + 32 * u * Tile::RB, (uint32_t)(seen >> (32 * u)), sh_odd + wave * FT / 4 * 64, &sh_any_odd, lane);
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

  int turn = 0;
  {
    Unit<SMALL> w;
    bool more = walk.template next<false>(p, w);
    load(kK, w, kr);
    load(kV, w, vr);
    for (; more; turn ^= 1) {
      Unit<SMALL> next;
      more = walk.template next<true>(p, next);
      barrier();  // nobody reads the unit before any more
      put_part(kK, kr, at_k, w.mixed, turn);
      put_part(kV, vr, at_v, w.mixed, turn);
      if (tid == 0) sh_unit_odd[turn ^ 1] = 0;
      load(kK, next, kr);
      load(kV, next, vr);
      barrier();
      attend(w.some, w.mixed, turn, [&] { return unit_seen(w, rel_q); });
      w = next;
    }
  }
  if (split == p.num_splits - 1 && nodes.all) {  // the drafted tokens: a unit of their own
    barrier();
    u32x4 rows[KK];
    draft_rows<Rows, false>(nodes.all, b, h, wave, c, gw, rows);
    put(kK, rows, at_k, 0, true, turn);
    draft_rows<Rows, true>(nodes.all, b, h, wave, c, gw, rows);
    put(kV, rows, at_v, 0, true, turn);
    barrier();
    attend(true, true, turn, [&] { return drafts_seen(nodes, h, node, rel_q); });
  }
  const CacheAttnParams& pe = params_in_memory();
  if (pe.missing && tid == 0 && walk.n_missing > 0) atomicAdd(pe.missing, walk.n_missing);

  // results from query-on-lane to rows, through where K and V were
  l_run = sum_groups(l_run);
  if (g == 0) {
    sh_m[wave][c] = there_q ? m_run : kNegInf;
    sh_l[wave][c] = there_q ? l_run : 0.f;
  }
  __syncthreads();
  float* const sums = reinterpret_cast<float*>(sh_kv[0]);
  float* const mine = sums + (16 * wave + c) * RS + 4 * g;
#pragma unroll
  for (int ft = 0; ft < FT; ++ft) *reinterpret_cast<f32x4*>(mine + 16 * ft) = there_q ? acc[ft] : f32x4{};
  if (sh_any_odd && there_q) add_odd<D>(mine, sh_odd + wave * FT / 4 * 64, lane);
  __syncthreads();
  constexpr int TPR = D / 8;  // threads to a query, eight features each
  for (int i = tid / TPR; i < pe.nodes; i += 64 * W / TPR) {
    const int d = 8 * (tid % TPR);
    float o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = sums[i * RS + d + e];
    put_result<D>(pe, b, h, i, split, d, o, sh_m[i / 16][i % 16], sh_l[i / 16][i % 16]);
  }
}

template <int D, int FMT>
hipError_t launch_blocks(const CacheAttnParams& p, hipStream_t stream) {
  const dim3 grid(p.nseq * p.heads * p.num_splits), block(256);
  if (p.block_size < 64)
    hipLaunchKernelGGL((cache_attn_shared_kernel<D, FMT, true>), grid, block, 0, stream, p);
  else
    hipLaunchKernelGGL((cache_attn_shared_kernel<D, FMT, false>), grid, block, 0, stream, p);
  return hipGetLastError();
}

template <int D>
hipError_t launch_dim(const CacheAttnParams& p, hipStream_t stream) {
  switch (p.c.format) {
    case S2_KV_BF16: return launch_blocks<D, S2_KV_BF16>(p, stream);
    case S2_KV_MXFP8: return launch_blocks<D, S2_KV_MXFP8>(p, stream);
    default: return launch_blocks<D, S2_KV_MXFP4>(p, stream);
  }
}

}  // namespace

hipError_t launch_cache_attn_shared(const CacheAttnParams& p, hipStream_t stream) {
  return p.c.head_dim == 128 ? launch_dim<128>(p, stream) : launch_dim<64>(p, stream);
}

}  // namespace s2
