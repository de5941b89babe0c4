// Norm of the rows of queries and keys and rotation by position, forward and backward, between a projection's layout and that of the attention calls.
//
// Forward, of a row x at position t: y = R_t (w x r), r = 1 / sqrt(mean(x^2) + eps), where R_t turns pair i of the first rotary_dim features by t * inv_freq[i].
// Each feature of y is a sum of two, x_f (w_f cos) and its partner's x_p (w_p (-+ sin)), both times r: the factors are the same for all heads of a row.
// Backward: with xh = x r and g' = R_t^T g, dw = sum g' xh and dx = r (w g' - xh mean(w g' xh)); r is formed again from x, which dw needs anyway.
//
// It moves bytes, and they bound it where there are many rows; a decode step's (64 x 32 heads 5.4 us) is the launch and two trips to memory.  D / 8 lanes take a row of D features, 16 bytes each, a wavefront 512 / D heads of one token at a time.  The angles of a token are formed once
// for its heads, a pair to a lane, and go through LDS: position times frequency and the whole turns that it holds in 64 bits (a far position's angle has no
// digits left for its fraction in 32), sine and cosine of what is left in 32.
//
// The weights' gradients are summed in registers over what a wavefront takes, over the wavefronts of a workgroup through LDS, and over workgroups by a
// second launch, in an order that the sizes alone decide (1024 parts of 2 x 128 sums 4.6 us; with eight groups of threads to 32 features instead of 64 to 16, 7.5).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kernels.h"
#include "kv_cache.h"
#include "sched_util.h"

namespace s2 {

namespace {

constexpr int kRopeWaves = 4;

// One row's features of a lane, as they lie, and their partners' (what is turned together with them).
struct Eight {
  u32x4 own, other;
};

__device__ __forceinline__ float lower(uint32_t x) { return __builtin_bit_cast(float, x << 16); }
__device__ __forceinline__ float upper(uint32_t x) { return __builtin_bit_cast(float, x & 0xffff0000u); }
__device__ __forceinline__ float feature_of(const u32x4& x, int e) { return e & 1 ? upper(x[e >> 1]) : lower(x[e >> 1]); }

// A row's part that nothing here reads again.  (Of 32 heads, 32768 tokens, forward: 225 us with ordinary loads and stores, 222 with these loads, 208 with such stores as
// well, 202 with the next heads' loads before these heads' sums, 5.3 TB/s, a large copy's rate; without the arithmetic 200.  Of 4 x 16 heads, 8192 tokens, backward: 169
// with these loads, 158 with such stores, 155 with the next heads' loads first, 5.2 TB/s.)
__device__ __forceinline__ u32x4 load_once(const uint16_t* at) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at)); }

// A row's part of the results; FAR: of more than kFarBytes.
template <bool FAR>
__device__ __forceinline__ void store(uint16_t* at, const u32x4& x) {
  if (FAR)
    __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(at));
  else
    *reinterpret_cast<u32x4*>(at) = x;
}

// sum over the D / 8 lanes of a row
template <int D>
__device__ __forceinline__ float row_sum(float x) {
  x += of_neighbour<1>(x);
  x += of_neighbour<2>(x);
  x += of_neighbour<4>(x);
  if (D == 128) x += of_neighbour<8>(x);
  return x;
}

// What a lane's features have to do with their partners.
struct Turn {
  bool on;        // they are rotated
  bool swapped;   // neighbours are partners: in the same lane
  int lane;       // else the lane that holds them
};
template <int D>
__device__ __forceinline__ Turn turn_of(const QkRopeParams& p, int lane) {
  const int c = lane % (D / 8), half = p.rotary_dim / 16;
  Turn t;
  t.on = 8 * c < p.rotary_dim;
  t.swapped = p.interleaved != 0;
  t.lane = !t.on || t.swapped ? lane : c < half ? lane + half : lane - half;
  return t;
}
__device__ __forceinline__ u32x4 partners(const u32x4& x, const Turn& t) {
  u32x4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = t.swapped ? x[i] << 16 | x[i] >> 16 : (uint32_t)__shfl((int)x[i], t.lane, 64);
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = t.on ? y[i] : 0;  // (an infinity times a factor of 0 is none)
  return y;
}

// cos and sin of a token's pairs into LDS, a pair to a lane
__device__ __forceinline__ void angles(const QkRopeParams& p, int position, float2* to, int lane) {
  float c = 1.f, s = 0.f;
  if (2 * lane < p.rotary_dim) {
    const double turns = (double)position * (double)p.inv_freq[lane] * 0.15915494309189533577;  // 1 / (2 pi)
    sincospif((float)(2.0 * (turns - __builtin_rint(turns))), &s, &c);
  }
  to[lane] = float2{c, s};
  __builtin_amdgcn_wave_barrier();
}
// A lane's cos, and sin with the sign that its partner enters with (forward).
template <int D>
__device__ __forceinline__ void factors(const QkRopeParams& p, const float2* cs, const Turn& t, int c, float (&co)[8], float (&si)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int half = p.rotary_dim / 2, f = 8 * c + e;
    const int pair = !t.on ? 0 : t.swapped ? f / 2 : f < half ? f : f - half;
    const bool first = t.swapped ? e % 2 == 0 : f < half;
    const float2 x = cs[pair];
    co[e] = t.on ? x.x : 1.f;
    si[e] = t.on ? (first ? -x.y : x.y) : 0.f;
  }
}
// The weights of a lane's features.
__device__ __forceinline__ void weights(const float* w, int from, float (&to)[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(w + from), b = *reinterpret_cast<const f32x4*>(w + from + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    to[e] = a[e];
    to[4 + e] = b[e];
  }
}

template <int D, bool FAR>
__global__ __launch_bounds__(64 * kRopeWaves) void qk_rope_kernel(const QkRopeParams p) {
  constexpr int LPR = D / 8, HPW = 64 / LPR;
  __shared__ float2 cs[kRopeWaves][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane % LPR, mine = lane / LPR;
  const int item = blockIdx.x * kRopeWaves + wave;
  if (item >= p.rows * p.head_groups) return;
  const int row = item / p.by_groups, group = item - row * p.head_groups;
  const int64_t b = row / p.by_seqlen;
  const int t = row - (int)b * p.seqlen;
  const Turn turn = turn_of<D>(p, lane);
  angles(p, p.positions ? load_const<int32_t>(p.positions + row) : t, cs[wave], lane);
  float co[8], si[8];
  factors<D>(p, cs[wave], turn, c, co, si);
  const int h0 = group * p.heads_each, h1 = min(h0 + p.heads_each, p.heads);
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (!p.x[which]) continue;
    const uint16_t* const x = p.x[which] + b * p.x_sb + t * p.x_st + 8 * c;
    uint16_t* const y = p.y[which] + b * p.y_sb + t * p.y_st + 8 * c;
    const bool norm = p.weight[which] != nullptr;
    float own[8], other[8];  // the factors with the weights
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      own[e] = co[e];
      other[e] = si[e];
    }
    if (norm) {
      float w[8], wo[8];
      weights(p.weight[which], 8 * c, w);
      weights(p.weight[which], 8 * (turn.lane % LPR), wo);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        own[e] *= w[e];
        other[e] = turn.on ? other[e] * (turn.swapped ? wo[e ^ 1] : wo[e]) : 0.f;  // (0 times an infinite weight is none)
      }
    }
    auto load = [&](int h) __attribute__((always_inline)) { return h < h1 ? load_once(x + h * p.x_sh) : u32x4{}; };
    u32x4 next = load(h0 + mine);
    for (int h = h0 + mine; h - mine < h1; h += HPW) {
      const bool is = h < h1;
      const u32x4 v = next;
      next = load(h + HPW);
      const u32x4 vo = partners(v, turn);
      float r = 1.f;
      if (norm) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(feature_of(v, e), feature_of(v, e), sum);
        r = rsqrtf(row_sum<D>(sum) * (1.f / D) + p.eps);
      }
      u32x4 out;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a = __builtin_fmaf(feature_of(vo, 2 * i), other[2 * i], feature_of(v, 2 * i) * own[2 * i]);
        const float z = __builtin_fmaf(feature_of(vo, 2 * i + 1), other[2 * i + 1], feature_of(v, 2 * i + 1) * own[2 * i + 1]);
        out[i] = pack2(a * r, z * r);
      }
      if (is) store<FAR>(y + h * p.y_sh, out);
    }
  }
}

template <int D, bool FAR>
__global__ __launch_bounds__(64 * kRopeWaves) void qk_rope_bwd_kernel(const QkRopeParams p) {
  constexpr int LPR = D / 8, HPW = 64 / LPR;
  __shared__ float2 cs[kRopeWaves][64];
  __shared__ float sums[kRopeWaves][2][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane % LPR, mine = lane / LPR;
  const Turn turn = turn_of<D>(p, lane);
  float dw[2][8];
#pragma unroll
  for (int i = 0; i < 16; ++i) dw[i / 8][i % 8] = 0.f;
  const int items = p.rows * p.head_groups;
  for (int item = blockIdx.x * kRopeWaves + wave; item < items; item += p.parts * kRopeWaves) {
    const int row = item / p.by_groups, group = item - row * p.head_groups;
    const int64_t b = row / p.by_seqlen;
    const int t = row - (int)b * p.seqlen;
    angles(p, p.positions ? load_const<int32_t>(p.positions + row) : t, cs[wave], lane);
    float co[8], si[8];
    factors<D>(p, cs[wave], turn, c, co, si);
    const int h0 = group * p.heads_each, h1 = min(h0 + p.heads_each, p.heads);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      if (!p.x[which]) continue;
      const int64_t at_x = b * p.x_sb + t * p.x_st + 8 * c, at_y = b * p.y_sb + t * p.y_st + 8 * c;
      const bool norm = p.weight[which] != nullptr;
      float w[8];
      if (norm) weights(p.weight[which], 8 * c, w);
      u32x4 g_next{}, x_next{};
      auto load = [&](int h) __attribute__((always_inline)) {
        g_next = h < h1 ? load_once(p.g[which] + at_y + h * p.y_sh) : u32x4{};
        x_next = h < h1 ? load_once(p.x[which] + at_x + h * p.x_sh) : u32x4{};
      };
      load(h0 + mine);
      for (int h = h0 + mine; h - mine < h1; h += HPW) {
        const bool is = h < h1;
        const u32x4 gv = g_next, v = x_next;
        load(h + HPW);
        const u32x4 go = partners(gv, turn);
        float g[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = __builtin_fmaf(feature_of(go, e), -si[e], feature_of(gv, e) * co[e]);
        u32x4 out;
        if (norm) {
          float sum = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(feature_of(v, e), feature_of(v, e), sum);
          const float r = rsqrtf(row_sum<D>(sum) * (1.f / D) + p.eps);
          float dot = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float xh = feature_of(v, e) * r, gx = g[e] * xh;
            if (is) dw[which][e] += gx;  // (a head that is not there has no row: with eps = 0 its r is an infinity)
            dot = __builtin_fmaf(gx, w[e], dot);
          }
          dot = row_sum<D>(dot) * (1.f / D);
#pragma unroll
          for (int e = 0; e < 8; ++e) g[e] = r * __builtin_fmaf(-feature_of(v, e) * r, dot, g[e] * w[e]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = pack2(g[2 * i], g[2 * i + 1]);
        if (is) store<FAR>(p.y[which] + at_x + h * p.x_sh, out);
      }
    }
  }
  if (!p.part) return;
  // the lane groups of a wavefront, then its workgroup
#pragma unroll
  for (int which = 0; which < 2; ++which)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float x = dw[which][e];
      if (D == 64) x += dpp<0x128>(x);  // (eight lanes on: row_ror)
      x = sum_groups(x);
      if (lane < LPR) sums[wave][which][8 * c + e] = x;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * D; i += 64 * kRopeWaves) {
    float x = 0.f;
#pragma unroll
    for (int w = 0; w < kRopeWaves; ++w) x += sums[w][i / D][i % D];
    p.part[(int64_t)blockIdx.x * 2 * D + i] = x;
  }
}

// 16 features of one weight's gradient: 64 groups of threads take a part in 64 each, their sums go two by two.
constexpr int kSumFeatures = 16, kSumGroups = 64;
template <int D>
__global__ __launch_bounds__(kSumFeatures * kSumGroups) void qk_rope_weights_kernel(const QkRopeParams p) {
  __shared__ float sums[kSumGroups][kSumFeatures];
  const int f = threadIdx.x % kSumFeatures, g = threadIdx.x / kSumFeatures;
  const int which = blockIdx.x / (D / kSumFeatures), d = kSumFeatures * (blockIdx.x % (D / kSumFeatures)) + f;
  if (!p.x[which] || !p.weight[which]) return;
  const float* const part = p.part + which * D + d;
  float x = 0.f;
#pragma unroll 8
  for (int i = g; i < p.parts; i += kSumGroups) x += part[(int64_t)i * 2 * D];
  sums[g][f] = x;
#pragma unroll
  for (int n = kSumGroups / 2; n > 0; n /= 2) {
    __syncthreads();
    if (g < n) sums[g][f] = x += sums[g + n][f];
  }
  if (g == 0) p.d_weight[which][d] = x;
}

// Heads to a wavefront: all of a token's (its angles are formed once) where there are tokens enough for the chip, else as few as a
// wavefront takes at a time.
void head_groups(QkRopeParams& p, int64_t waves) {
  const int at_once = 512 / p.head_dim, steps = (p.heads + at_once - 1) / at_once;
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>(steps, waves / std::max<int64_t>(1, p.rows)));
  p.heads_each = (int)((steps + want - 1) / want) * at_once;
  p.head_groups = (p.heads + p.heads_each - 1) / p.heads_each;
  p.by_groups = fast_div(p.head_groups);
  p.by_seqlen = fast_div(std::max(1, p.seqlen));
}

constexpr int64_t kFwdWaves = 8192;
// Bytes of results beyond which they go past the caches.  The cache behind the L2s holds 256 MB, of everything that passes: four states in turn, each call alone and with what
// reads its results (forward: the attention; backward: a matrix product), us with ordinary stores and with such ones:
//   results      forward alone     with the attention    backward alone    with the product
//    16 MB        15.0   14.4        37.9   40.2            18.9   18.7       86.2   87.2
//    64 MB        32.8   32.4       114    117              43.8   46.6      153    157
//    96 MB        41.3   39.4       163    166              69.6   66.5      211    214
//   128 MB        56.1   54.8       224    230              91.8   84.5      261    260
//   256 MB       100     96.5       429    433             172    156        452    451
//   384 MB       160    148         805    820             254    234        701    695
constexpr int64_t kFarBytes = 64 << 20;
constexpr int kBwdParts = 1024;

bool is_far(const QkRopeParams& p) { return (int64_t)p.rows * p.heads * p.head_dim * 2 * ((p.x[0] != nullptr) + (p.x[1] != nullptr)) > kFarBytes; }

}  // namespace

int64_t qk_rope_groups(const QkRopeParams& params) {
  QkRopeParams p = params;
  head_groups(p, kFwdWaves);
  return ((int64_t)p.rows * p.head_groups + kRopeWaves - 1) / kRopeWaves;
}

hipError_t launch_qk_rope(const QkRopeParams& params, hipStream_t stream) {
  QkRopeParams p = params;
  head_groups(p, kFwdWaves);
  const bool far = is_far(p);
  const dim3 grid((p.rows * p.head_groups + kRopeWaves - 1) / kRopeWaves), block(64 * kRopeWaves);
  if (p.head_dim == 128) {
    if (far)
      hipLaunchKernelGGL((qk_rope_kernel<128, true>), grid, block, 0, stream, p);
    else
      hipLaunchKernelGGL((qk_rope_kernel<128, false>), grid, block, 0, stream, p);
  } else {
    if (far)
      hipLaunchKernelGGL((qk_rope_kernel<64, true>), grid, block, 0, stream, p);
    else
      hipLaunchKernelGGL((qk_rope_kernel<64, false>), grid, block, 0, stream, p);
  }
  return hipGetLastError();
}

int qk_rope_parts(int rows, int heads, int head_dim) {
  QkRopeParams p{};
  p.rows = rows;
  p.heads = heads;
  p.head_dim = head_dim;
  p.seqlen = 1;
  head_groups(p, (int64_t)kBwdParts * kRopeWaves);
  return (int)std::clamp<int64_t>(((int64_t)rows * p.head_groups + kRopeWaves - 1) / kRopeWaves, 1, kBwdParts);
}

hipError_t launch_qk_rope_bwd(const QkRopeParams& params, hipStream_t stream) {
  QkRopeParams p = params;
  head_groups(p, (int64_t)kBwdParts * kRopeWaves);
  p.parts = qk_rope_parts(p.rows, p.heads, p.head_dim);
  const dim3 grid(p.parts), block(64 * kRopeWaves);
  const bool far = is_far(p);
  if (p.head_dim == 128) {
    if (far)
      hipLaunchKernelGGL((qk_rope_bwd_kernel<128, true>), grid, block, 0, stream, p);
    else
      hipLaunchKernelGGL((qk_rope_bwd_kernel<128, false>), grid, block, 0, stream, p);
  } else {
    if (far)
      hipLaunchKernelGGL((qk_rope_bwd_kernel<64, true>), grid, block, 0, stream, p);
    else
      hipLaunchKernelGGL((qk_rope_bwd_kernel<64, false>), grid, block, 0, stream, p);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.part) return e;
  if (p.head_dim == 128)
    hipLaunchKernelGGL(qk_rope_weights_kernel<128>, dim3(2 * 128 / kSumFeatures), dim3(kSumFeatures * kSumGroups), 0, stream, p);
  else
    hipLaunchKernelGGL(qk_rope_weights_kernel<64>, dim3(2 * 64 / kSumFeatures), dim3(kSumFeatures * kSumGroups), 0, stream, p);
  return hipGetLastError();
}

}  // namespace s2
