// A decode step over a paged cache in 8 or 4 bits (section 4.1): one query to a (sequence, head).
//
// One multiply-add to a value held: bytes bound it, and vector instructions come next (two values to a conversion, two products to a dot
// product of bf16 pairs, one product with P to an instruction: 2 instructions a value, 6.4 us of the chip for what 4 bits bring in 10).  So no
// matrix instruction and no LDS on the way: a wavefront takes 64 tokens at a time, 16 rows to a piece and four lanes to a row (CacheRows), a lane
// forms its quarter of a row's score, the four quarters are added by lane permutations, and the row's probability is then where its V
// is: a lane accumulates its quarter of the features over the rows of its own, and rows are added up once at the end.  Probabilities stay in 32 bits.
//
// 64 x 32 heads of 8192 to 32768 x 128: e4m3 213 us (5.5 TB/s), e2m1 in blocks of 16 73 us (5.0 TB/s); one sequence of 32768 over e4m3 11.8 us with
// its merge.  As matrix products, as in cache_attn_kernel.hip, with one of 16 columns in use, where a unit is a chain of LDS round trips (1250 cycles for its
// scores, 2850 for its sums): 217, 119 and 16.7 us.
#include <hip/hip_runtime.h>

#include "cache_attn.h"
#include "config.h"

namespace s2 {

namespace {

__device__ __forceinline__ float dot2(uint32_t a, uint32_t b, float c) {
  return __builtin_amdgcn_fdot2_f32_bf16(two_of(a), two_of(b), c, false);
}

// Wavefronts to a SIMD that the registers are limited for: as many as fit without spilling (e4m3, D = 128, with two instead of three: 213 and 213 us for 64 x 32
// heads of 8192 to 32768, 3 to 6 % slower at 256 to 1024 (sequence, head) pairs).
constexpr int waves_for(int D, int FMT) { return D == 128 && FMT == S2_KV_MXFP8 ? 3 : 4; }

// W: wavefronts to a workgroup.
template <int D, int FMT, bool SMALL, int W>
__global__ __launch_bounds__(64 * W, waves_for(D, FMT)) void cache_decode_kernel(const CacheAttnParams p) {
  using Rows = CacheRows<D, FMT>;
  constexpr int KK = D / 32, NF = D / 4;  // operands of eight features, features to a lane

  __shared__ float sh_m[W], sh_l[W];
  __shared__ float sh_acc[W][D];

  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int item = blockIdx.x;
  const int bh = item / p.by_splits, split = item - bh * p.num_splits;
  const int b = bh / p.by_heads, h = bh - b * p.heads;
  const float cl = p.scale_log2e;

  int L = load_const<int32_t>(p.seq_lens + b);
  L = min(max(L, 1), p.max_len);
  Nodes one{};
  one.row0 = (L - 1) >> p.c.block_shift;
  one.n_rows = 1;
  Walk<SMALL> walk(b, h, L, one, split, wave, W, 0);
  u32x4 q[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) q[kk] = *reinterpret_cast<const u32x4*>(p.q + b * p.q_ss + h * p.q_sh + Rows::feature(kk, g));

  typename Rows::Part kr[4], vr[4];
  auto load = [&](const Unit<SMALL>& w, const uint8_t* pool, const uint8_t* scales, typename Rows::Part (&x)[4]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < Unit<SMALL>::NB; ++i) {
      const int page = w.page[i], skip = Unit<SMALL>::skip(w.info[i]);
      const uint8_t* const at = pool + page * p.c.page + skip * p.c.tok;
      const uint8_t* const scale_at = scales + page * p.c.scale_page + skip * p.c.scale_tok;
#pragma unroll
      for (int t = 0; t < 4 / Unit<SMALL>::NB; ++t) Rows::load(x[i + t], at, scale_at, Unit<SMALL>::rows(w.info[i]), p.c.tok, p.c.scale_tok, 16 * t + c, g);
    }
  };

  float acc[NF], m_run = kNegInf, l_run = 0.f, s[4];
#pragma unroll
  for (int i = 0; i < NF; ++i) acc[i] = 0.f;
  auto scores = [&](const Unit<SMALL>& w) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      u32x4 k[KK];
      Rows::operands(kr[t], g, k);
      float x = 0.f, y = 0.f;  // (two chains)
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        x = dot2(k[kk][0], q[kk][0], x);
        y = dot2(k[kk][1], q[kk][1], y);
        x = dot2(k[kk][2], q[kk][2], x);
        y = dot2(k[kk][3], q[kk][3], y);
      }
      x = sum_groups(x + y);
      const int rows = Unit<SMALL>::rows(w.info[SMALL ? t : 0]) - (SMALL ? 0 : 16 * t);
      s[t] = c < rows ? x : kNegInf;
    }
  };
  auto sums = [&]() __attribute__((always_inline)) {
    float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    mx = fmaxf(mx, of_neighbour<1>(mx));
    mx = fmaxf(mx, of_neighbour<2>(mx));
    mx = fmaxf(mx, of_neighbour<4>(mx));
    mx = fmaxf(mx, of_neighbour<8>(mx));
    const float m_new = fmaxf(m_run, mx);
    const float mc = m_new == kNegInf ? 0.f : m_new * cl;
    if (__any(m_new > m_run)) {
      const float alpha = fast_exp2(m_run * cl - mc);  // (-inf before the first token: 0)
      l_run *= alpha;
      m_run = m_new;
#pragma unroll
      for (int i = 0; i < NF; ++i) acc[i] *= alpha;
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const float pr = fast_exp2(__builtin_fmaf(s[t], cl, -mc));
      l_run += pr;
      Rows::add_times(vr[t], g, pr, acc);
    }
  };

  {
    Unit<SMALL> w;
    if (walk.template next<false>(p, w)) {
      load(w, p.c.k, p.c.ks, kr);
      load(w, p.c.v, p.c.vs, vr);
      for (bool more = true; more;) {
        Unit<SMALL> next;
        more = walk.template next<true>(p, next);
        // the next unit's K goes into the registers that the scores have freed, its V into those that the sums free
        scores(w);
        __builtin_amdgcn_sched_barrier(0);
        load(next, p.c.k, p.c.ks, kr);
        __builtin_amdgcn_sched_barrier(0);
        sums();
        __builtin_amdgcn_sched_barrier(0);
        load(next, p.c.v, p.c.vs, vr);
        w = next;
      }
    }
  }
  const CacheAttnParams& pe = params_in_memory();
  if (pe.missing && lane == 0 && walk.n_missing > 0) atomicAdd(pe.missing, walk.n_missing);

  // the rows of the wavefront, then the wavefronts
  auto over_rows = [](float x) __attribute__((always_inline)) {
    x += of_neighbour<1>(x);
    x += of_neighbour<2>(x);
    x += of_neighbour<4>(x);
    return x + of_neighbour<8>(x);
  };
  l_run = over_rows(l_run);
#pragma unroll
  for (int i = 0; i < NF; ++i) acc[i] = over_rows(acc[i]);
  if (lane == 0) {
    sh_m[wave] = m_run;
    sh_l[wave] = l_run;
  }
  if (c == 0) {
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int e = 0; e < 8; ++e) sh_acc[wave][Rows::feature(kk, g) + e] = acc[8 * kk + e];
  }
  __syncthreads();
  if (tid >= D / 8) return;
  const int d = 8 * tid;
  float m = kNegInf, l = 0.f, o[8];
#pragma unroll
  for (int w = 0; w < W; ++w) m = fmaxf(m, sh_m[w]);
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = 0.f;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const float weight = sh_l[w] == 0.f ? 0.f : fast_exp2((sh_m[w] - m) * cl);  // (no sum: no token)
    l += sh_l[w] * weight;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] += sh_acc[w][d + e] * weight;
  }
  put_result<D>(pe, b, h, 0, split, d, o, m, l);
}

template <int D, int FMT, int W>
void launch_blocks(const CacheAttnParams& p, hipStream_t stream) {
  const dim3 grid(p.nseq * p.heads * p.num_splits), block(64 * W);
  if (p.block_size < 64)
    hipLaunchKernelGGL((cache_decode_kernel<D, FMT, true, W>), grid, block, 0, stream, p);
  else
    hipLaunchKernelGGL((cache_decode_kernel<D, FMT, false, W>), grid, block, 0, stream, p);
}

template <int D, int FMT>
hipError_t launch_waves(const CacheAttnParams& p, hipStream_t stream) {
  if (p.nseq * p.heads * p.num_splits <= kCacheWideGroups)
    launch_blocks<D, FMT, 8>(p, stream);
  else
    launch_blocks<D, FMT, 4>(p, stream);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_decode(const CacheAttnParams& p, hipStream_t stream) {
  const bool mx8 = p.c.format == S2_KV_MXFP8;
  if (p.c.head_dim == 128) return mx8 ? launch_waves<128, S2_KV_MXFP8>(p, stream) : launch_waves<128, S2_KV_MXFP4>(p, stream);
  return mx8 ? launch_waves<64, S2_KV_MXFP8>(p, stream) : launch_waves<64, S2_KV_MXFP4>(p, stream);
}

}  // namespace s2
