// Attention of a chunk of more than 64 new tokens over a paged cache: tiles of 128 rows, 32 to a wavefront (see cache_chunk_kernel.hip for the mathematics).
//
// Matrix instructions bound it (41 % of a SIMD's cycles), and beside them the vector instructions of the softmax and of bringing rows to bf16 (51 %): 2048 rows of 32 heads
// after 30720 tokens over e4m3, 512 workgroups of 47 units, 115 us among many such calls (850 TFLOP/s), 118 in a trace of 300, up to 137 in shorter runs; the forward of the same rows
// over contiguous bf16, timed in turn, 94 among many, up to 109.  A SIMD overlaps the two where they alternate finely in
// one instruction stream (sched_util.h), so the loop is software pipelined by halves of a unit, 32 tokens: in half step j a wavefront forms the scores of half j, turns those of
// half j - 1 into probabilities and adds the product of half j - 2's with V, which are independent of each other, in one hand-written sequence of slots, a
// matrix instruction to each.  V lags behind K by a unit, so that both tiles of a trip are used up in it and one barrier a trip is enough: meanwhile each
// wavefront brings its 16 rows of the next unit's K, and of this one's V, from registers to bf16 in the other stage, and asks for those after them.
//
// The reference maximum of a query moves only where a score exceeds it by more than 2^8 (a probability is then up to 2^8, rounded as any other): one of 32 queries has a
// new maximum in nearly every half step of the first hundred.  Where it moves, the accumulators lack the half whose probabilities were formed against the
// old one: they are scaled a half step later, when it has been added.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache_chunk.h"
#include "cache_chunk_few.h"
#include "config.h"

namespace s2 {

namespace {

template <int D, int FMT, bool SMALL>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void cache_chunk_wide_kernel(const CacheChunkParams p) {
  using Rows = CacheRows<D, FMT>;
  using Tile = DmaTile<D>;  // (the strides at which 16 rows are written without bank conflicts, too)
  using Pieces = ChunkWalk<SMALL>;
  constexpr int W = 4, MW = 32, KK = D / 16, DT = D / 32, KO = D / 32;  // KO: operands of eight features to a lane's part of a row
  constexpr int NS = 2 * KK;                                            // slots: KK of the scores, 2 * DT of the product with V
  constexpr int RB = Tile::kStride * 2;
  constexpr int kLead = D == 128 ? 5 : 3, kRing = kLead + 1;  // fragments are asked for so many slots ahead
  constexpr int RS = D + 4;                    // floats to a row where results are turned
  static_assert(2 * DT == KK && W * MW * RS * 4 <= 4 * Tile::kBytes, "the wavefronts' sums fit where K and V were");

  __shared__ __align__(16) uint16_t sh_kv[4][Tile::kElems];  // two stages of K, two of V
  __shared__ u32x2 sh_pieces[W][Pieces::kRing];
  __shared__ ChunkScope sh_scope;
  __shared__ ChunkTileAt sh_tile;
  __shared__ uint32_t sh_v_odd[4][2];  // whether the V of a trip, modulo four, holds what is not finite, by halves

  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int th = blockIdx.x / p.by_splits, split = blockIdx.x - th * p.num_splits;
  const int tile = th / p.by_heads, h = th - tile * p.heads;
  const float cl = p.scale_log2e;

  const ChunkTileAt x0 = chunk_tile_at(p, tile);
  if (x0.rows <= 0) return;
  const ChunkRows r0 = chunk_block_rows(p, x0);
  // A tile of few rows (a short chunk among long ones, the end of one) would leave wavefronts without a query: theirs take tokens of their own instead (12 chunks of up to
  // 1024 rows over e4m3 105 us to 95, 40 of up to 300 226 to 191, 4 of 2048 as before).  Expected not to be: else the loop below goes without registers that this one takes.
  if (__builtin_expect(__builtin_amdgcn_readfirstlane(x0.rows) <= 32, 0)) {
    using Few = ChunkFewShared<D, 2, SMALL>;
    static_assert(sizeof(Few) <= sizeof(sh_kv), "it fits where K and V are otherwise");
    chunk_few<D, FMT, 2, SMALL>(p, x0, r0, h, split, *reinterpret_cast<Few*>(sh_kv));
    return;
  }
  const ChunkQuery q0 = chunk_query(p, x0, r0, MW * wave + l32 - x0.skipped);
  bf16x8 qf[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk)
    qf[kk] = q0.there ? *reinterpret_cast<const bf16x8*>(p.q + (x0.row + MW * wave + l32 - x0.skipped) * p.q_sr + h * p.q_sh + 16 * kk + 8 * half) : bf16x8{};
  if (tid < 8) sh_v_odd[tid / 2][tid % 2] = 0;
  if (tid == 0) {
    sh_scope.init(p, x0, r0, h, split);
    sh_tile = x0;
  }
  __syncthreads();
  Pieces walk(sh_scope, r0.n_rows, wave, sh_pieces[wave], q0, q0);
  // what my query attends of half H of unit u, bits
  auto seen_of = [&](int u, int H) S2_INLINE {
    const ChunkQuery q = chunk_query(chunk_params(), sh_tile, sh_scope.r, MW * wave + (lane_now() & 31) - sh_tile.skipped);
    return chunk_seen<SMALL>(walk, u, q.rel, q.pos) >> (32 * H);
  };

  f32x16 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = f32x16{};
  float m_run = kNegInf, mc = 0.f, l_run = 0.f, alpha = 1.f;  // mc: the maximum as exponents have it, 0 while nothing was seen
  // how far a score may exceed it (finite, also where 2^8 is out of reach of any score: the first has to move it from -inf)
  const float tau = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, fminf(8.f / cl, 3.4e38f))));
  bool scaled = false;                                        // whether alpha is to be applied to the accumulators

  const uint32_t write = lds_addr(sh_kv) + (16 * wave + (lane & 15)) * RB + 2 * Rows::feature(0, lane >> 4);  // (feature(kk, g) is feature(kk, 0) further on)
  const uint32_t k_read = lds_addr(sh_kv) + l32 * RB + 16 * half, v_read = lds_addr(sh_kv) + 2 * Tile::tr_base(lane);
  constexpr int kV0 = 2 * Tile::kBytes;

  // (kept in registers: left to itself the compiler fetches them where they are used, and waits for the LDS as well)
  const uint8_t *k_pool = p.c.k, *v_pool = p.c.v, *k_scales = p.c.ks, *v_scales = p.c.vs;
  int tok = p.c.tok, scale_tok = p.c.scale_tok;
  asm volatile("" : "+s"(k_pool), "+s"(v_pool), "+s"(tok));
  if constexpr (Rows::kScaled) asm volatile("" : "+s"(k_scales), "+s"(v_scales), "+s"(scale_tok));
  const int my_row = (SMALL ? 0 : 16 * wave) + (lane & 15), lane_at = my_row * tok + Rows::kLoadBytes * (lane >> 4), scale_at = my_row * scale_tok;
  typename Rows::Part kr, vr;
  auto load = [&](auto is_v, const ChunkUnit& w, typename Rows::Part& to) S2_INLINE {
    constexpr bool V = decltype(is_v)::value;
    Rows::load_at(to, (V ? v_pool : k_pool) + w.off, Rows::kScaled ? (V ? v_scales : k_scales) + w.scale_off : nullptr, w.rows, tok, scale_tok, lane_at, scale_at);
  };
  constexpr std::false_type kK{};
  constexpr std::true_type kV{};
  // operand kk of my row of 16 into a stage
  auto put = [&](const typename Rows::Part& part, int g, int kk, uint32_t to) S2_INLINE {
    *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(to + 2 * Rows::feature(kk, 0)) = Rows::operand(part, g, kk, 0);
  };
  // (what it has asked of the LDS is done before a wavefront is past it; loads from memory stay on their way)
  auto barrier = [&]() S2_INLINE {
    wait_lds();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  // scores of two halves, then their probabilities in 32 bits: register r is token 8 * (r / 4) + 4 * half + r % 4 of the half, lane % 32 the query
  f32x16 s0 = f32x16{}, s1 = f32x16{};
  // the same as operands: rounded to bf16, as in the forward of a whole sequence: off by up to 2^-8 of a probability, 2.3e-3 of a result instead of 1.7e-3 (relative L2).  (In two
  // terms, 16 bits, as for fewer rows, V is multiplied twice: 2048 rows over e4m3 140 us and 174, 12 ragged chunks over bf16 206 and 235, 7 over e2m1 23.4 and 24.8.)
  u32x4 pb0[2] = {u32x4{}, u32x4{}}, pb1[2] = {u32x4{}, u32x4{}};

  // The fragments of a trip, in one ring through both of its half steps: of half f / NS the rows of K, then those of V, transposed.
  bf16x8 fr[kRing];
  uint32_t ks = 0, vs = 0;
  auto frag_load = [&](auto fc) S2_INLINE {
    constexpr int f = decltype(fc)::value % NS, H = decltype(fc)::value / NS;
    if constexpr (f < KK)
      fr[decltype(fc)::value % kRing] = __builtin_bit_cast(bf16x8, lds_read16(ks, 32 * H * RB + 32 * f));
    else
      fr[decltype(fc)::value % kRing] = __builtin_bit_cast(bf16x8, lds_read_tr(vs, kV0 + (32 * H + 16 * ((f - KK) / DT)) * RB + 64 * ((f - KK) % DT), RB));
  };
  static_assert(kLead <= KK, "of the second half no V is asked for in the first");
  auto first_frags = [&]() S2_INLINE { static_for<kLead>([&](auto fc) S2_INLINE { frag_load(fc); }); };

  // Half step H of trip t: scores of half H of unit t (sn), probabilities of the half before it (sc, pc), the product of half H of unit t - 1 (pp) with V.  on_n, on_s:
  // whether the first two are mine; some_n: whether a token of the unit is not attended by some query.  Where nothing is mine it all runs the same, with zeros: a
  // branch around it has the compiler move the accumulators between registers.
  auto half_step = [&](auto hc, int t, bool on_n, bool on_s, bool some_n, f32x16& sn, f32x16& sc, u32x4 (&pc)[2], u32x4 (&pp)[2],
                       auto&& beside) S2_INLINE {
    constexpr int H = decltype(hc)::value;
    float mc_use = on_s ? mc : __builtin_inff();  // (not mine: its scores are zeros, its probabilities 0)
    asm volatile("" : "+v"(mc_use));
    float mx = kNegInf;
    // 16 scores in three stages - scale and shift, exponential, sum and pack - each a slot behind the one before it
    constexpr auto upto = [](int sl) { return std::max(0, std::min(16, (16 * (sl + 1) + NS - 3) / (NS - 2))); };
    static_assert(upto(NS - 3) >= 16, "packed in time");
    if constexpr (H == 0) first_frags();
    S2_FENCE();
    static_for<NS>([&](auto slc) S2_INLINE {
      constexpr int sl = decltype(slc)::value;
      if constexpr (H * NS + sl + kLead < 2 * NS) frag_load(std::integral_constant<int, H * NS + sl + kLead>{});
      if constexpr (sl < KK)
        sn = mfma32(fr[(H * NS + sl) % kRing], qf[sl], sl == 0 ? f32x16{} : sn);
      else
        acc[(sl - KK) % DT] = mfma32(fr[(H * NS + sl) % kRing], __builtin_bit_cast(bf16x8, pp[(sl - KK) / DT]), acc[(sl - KK) % DT]);
#pragma unroll
      for (int e = upto(sl - 1); e < upto(sl); ++e) sc[e] = __builtin_fmaf(sc[e], cl, -mc_use);
#pragma unroll
      for (int e = upto(sl - 2); e < upto(sl - 1); ++e) sc[e] = fast_exp2(sc[e]);
#pragma unroll
      for (int e = upto(sl - 3); e < upto(sl - 2); ++e) {
        l_run += sc[e];
        if (e & 1) {
          pc[e >> 3][(e & 7) >> 1] = pack2(sc[e - 1], sc[e]);
          asm volatile("" : "+v"(pc[e >> 3][(e & 7) >> 1]));  // (here, not where it is used, half a trip on)
        }
      }
      // maximum of the new scores, once their products are done
      constexpr int M0 = KK + 2, kMax = D == 128 ? 4 : 8;
      static_assert((NS - M0) * kMax >= 16, "all sixteen");
      if constexpr (sl >= M0) {
#pragma unroll
        for (int e = kMax * (sl - M0); e < std::min(16, kMax * (sl - M0 + 1)); e += 2) mx = fmaxf(fmaxf(mx, sn[e]), sn[e + 1]);
      }
      beside(slc);
      // Nothing to execute: ties the running sum and maximum to this slot, or the optimiser collects their additions and comparisons after the last product.
      asm volatile("" : "+v"(l_run), "+v"(mx));
      S2_FENCE();
    });
    if (scaled) {
      asm volatile("");  // (a branch: else the accumulators are multiplied by 1 in every half step)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[dt][r] *= alpha;
      scaled = false;
    }
    if (on_n) {
      if (some_n) {
        const uint32_t seen = (uint32_t)seen_of(t, H) >> (4 * (lane_now() >> 5));
        mx = kNegInf;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          sn[r] = seen >> (8 * (r / 4) + r % 4) & 1 ? sn[r] : kNegInf;
          mx = fmaxf(mx, sn[r]);
        }
      }
      // (a lane's own scores are enough to see whether any of a query's is above its maximum)
      if (__any(mx - m_run > tau)) {  // (-inf minus itself is not a number, and no reason to move)
        const float top = max_halves(mx);
        const bool moves = top - m_run > tau;
        // (What another query's maximum does leaves this one's result as it is.  Never 0, but the smallest number there is: by the time that it is applied, a half step later,
        // infinities of V that belong to the scores that moved it have been added, and 0 times those is none.)
        alpha = moves ? fmaxf(fast_exp2(m_run * cl - top * cl), 0x1p-149f) : 1.f;
        m_run = moves ? top : m_run;
        mc = m_run == kNegInf ? 0.f : m_run * cl;
        l_run *= alpha;
        scaled = true;
      }
    } else {
      sn = f32x16{};
    }
  };

  {
    constexpr std::integral_constant<int, 0> first{};
    constexpr std::integral_constant<int, 1> second{};
    ChunkUnit prev{}, cur{}, next{};
    // (the second unit is one of the first look-up's or none: an empty one among the others changes nothing, and one place less looks up)
    bool more = walk.find();  // whether there may be more units
    if (more) walk.take(0, cur);
    if (more && walk.live != 0) walk.take(1, next);
    load(kK, cur, kr);
    static_for<KO>([&](auto kk) S2_INLINE { put(kr, lane >> 4, decltype(kk)::value, write); });
    static_for<KO>([&](auto kk) S2_INLINE {  // (no V before the first: zeros, which a probability of 0 leaves)
      *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(write + kV0 + 2 * Rows::feature(decltype(kk)::value, 0)) = u32x4{};
    });
    load(kK, next, kr);
    load(kV, cur, vr);
    barrier();
    for (int t = 0;; ++t) {
      const uint32_t to = ((t + 1) & 1) * (uint32_t)Tile::kBytes;
      ChunkUnit then;
      more = more && walk.next(t + 2, then);
      if (!more) then = ChunkUnit{};
      const int g = lane_now() >> 4;
      if (tid < 2) sh_v_odd[(t + 3) & 3][tid] = 0;  // (read a trip ago, written a trip from now)
      if (prev.some() && (sh_v_odd[t & 3][0] | sh_v_odd[t & 3][1])) {  // (the same for all wavefronts)
        // What a query does not attend stays out of its result whatever it holds, but 0 times an infinity or NaN is none: such values of V are added to the sums of
        // the queries that attend them here, and taken out of V.
        const uint64_t seen = seen_of(t - 1, 0);
#pragma unroll 1
        for (int i = 0; i < 64; ++i) {
          const uint32_t row = lds_addr(sh_kv) + kV0 + (t & 1) * (uint32_t)Tile::kBytes + i * RB + 8 * half;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const u32x2 v = *(const __attribute__((address_space(3))) u32x2*)(uintptr_t)(row + 64 * dt + 16 * q);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t bits = e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16;
                acc[dt][4 * q + e] += (seen >> i & 1) && (bits & 0x7f800000u) == 0x7f800000u ? __builtin_bit_cast(float, bits) : 0.f;
              }
            }
        }
        barrier();
        clean_words(reinterpret_cast<uint32_t*>(sh_kv[2 + (t & 1)]) + 16 * wave * RB / 4, 16 * RB / 4, lane);
        barrier();
      }
      ks = k_read + (t & 1) * (uint32_t)Tile::kBytes;
      vs = v_read + (t & 1) * (uint32_t)Tile::kBytes;
      asm volatile("" : "+v"(ks), "+v"(vs));
      half_step(first, t, cur.on(0), prev.on(1), cur.some(), s0, s1, pb1, pb0, [&](auto slc) S2_INLINE {
        constexpr int sl = decltype(slc)::value;
        if constexpr (sl < KO) put(kr, g, sl, write + to);
        if constexpr (sl == KO) load(kK, then, kr);
      });
      half_step(second, t, cur.on(1), cur.on(0), cur.some(), s1, s0, pb0, pb1, [&](auto slc) S2_INLINE {
        constexpr int sl = decltype(slc)::value;
        if constexpr (sl < KO) put(vr, g, sl, write + kV0 + to);
        if constexpr (sl == KO) load(kV, next, vr);
      });
      if (cur.some()) {  // whether my rows of its V are all finite
        u32x4 v[KO];
        static_for<KO>([&](auto kk) S2_INLINE { v[decltype(kk)::value] = lds_read16(write + kV0 + to, 2 * Rows::feature(decltype(kk)::value, 0)); });
        if (odd_bits(v)) sh_v_odd[(t + 1) & 3][wave >> 1] = 1;
      }
      barrier();
      // (the last unit's probabilities meet its V in the trip after its own)
      if (!more && !cur.there() && !next.there()) break;
      prev = cur;
      cur = next;
      next = then;
    }
  }
  const CacheChunkParams& pe = chunk_params();
  if (pe.missing && tid == 0 && walk.n_missing > 0) atomicAdd(pe.missing, walk.n_missing);

  // results from query-on-lane to rows, through where K and V were: a wavefront's 32 are its own
  const ChunkTileAt x = sh_tile;
  const float l = sum_halves(l_run);
  const bool there = chunk_query(pe, x, sh_scope.r, MW * wave + l32 - x.skipped).there;
  float* const sums = reinterpret_cast<float*>(sh_kv[0]) + MW * wave * RS;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 w = f32x4{acc[dt][4 * g], acc[dt][4 * g + 1], acc[dt][4 * g + 2], acc[dt][4 * g + 3]};
      *reinterpret_cast<f32x4*>(sums + l32 * RS + 32 * dt + 8 * g + 4 * half) = there ? w : f32x4{};
    }
  if (half == 0) {  // (where the rows' padding is)
    sums[l32 * RS + D] = there ? m_run : kNegInf;
    sums[l32 * RS + D + 1] = there ? l : 0.f;
  }
  constexpr int TPR = D / 8;  // lanes to a query, eight features each
  for (int i = lane / TPR; i < MW; i += 64 / TPR) {
    const int row = MW * wave + i - x.skipped, d = 8 * (lane % TPR);
    if (row < 0 || row >= x.rows) continue;
    float o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = sums[i * RS + d + e];
    put_chunk_row<D>(pe, x, sh_scope.h, row, sh_scope.split, d, o, sums[i * RS + D], sums[i * RS + D + 1]);
  }
}

template <int D, int FMT>
void launch_blocks(const CacheChunkParams& p, hipStream_t stream) {
  const dim3 grid(p.num_tiles * p.heads * p.num_splits), block(256);
  if (p.block_size < 64)
    hipLaunchKernelGGL((cache_chunk_wide_kernel<D, FMT, true>), grid, block, 0, stream, p);
  else
    hipLaunchKernelGGL((cache_chunk_wide_kernel<D, FMT, false>), grid, block, 0, stream, p);
}

template <int D>
hipError_t launch_dim(const CacheChunkParams& p, hipStream_t stream) {
  switch (p.c.format) {
    case S2_KV_BF16: launch_blocks<D, S2_KV_BF16>(p, stream); break;
    case S2_KV_MXFP8: launch_blocks<D, S2_KV_MXFP8>(p, stream); break;
    default: launch_blocks<D, S2_KV_MXFP4>(p, stream); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_chunk_wide(const CacheChunkParams& p, hipStream_t stream) {
  return p.c.head_dim == 128 ? launch_dim<128>(p, stream) : launch_dim<64>(p, stream);
}

}  // namespace s2
