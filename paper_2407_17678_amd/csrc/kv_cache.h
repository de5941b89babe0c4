// Internal: rows of a paged cache in bf16, e4m3 or e2m1 with one power-of-two scale to 32 features, as the kernels hold them.
//
// A wavefront takes rows 16 at a time, lane = 16 * g + r: row r, a quarter of its bytes.  Which quarter is chosen so that an
// instruction fetches whole runs of 64 bytes of a row; the features that a lane then holds are permuted, which a contraction over
// features does not see as long as the other operand is permuted alike (feature()).  Eight features are one operand of an MFMA.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/s2attn.h"
#include "device_util.h"
#include "kernels.h"

namespace s2 {

typedef __bf16 bf16x2_ __attribute__((ext_vector_type(2)));
typedef short s16x2_ __attribute__((ext_vector_type(2)));

// A word as two bf16 values.  (A function, so that a vector's element is copied first: this compiler's __builtin_bit_cast takes element 0 for
// any element that it is given where it lies.)
__device__ __forceinline__ bf16x2_ two_of(uint32_t word) { return __builtin_bit_cast(bf16x2_, word); }

// 2^(byte - 127) as the conversions take it; byte 255 is an infinity, with which they give NaN for every code.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// Four e4m3 codes, or eight e2m1 codes, times a scale as bf16, without rounding.
__device__ __forceinline__ void values8(uint32_t codes, float scale, uint32_t (&out)[2]) {
  out[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false));
  out[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true));
}
__device__ __forceinline__ u32x4 values4(uint32_t codes, float scale) {
  u32x4 x;
  x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
  x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
  x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
  x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  return x;
}

template <int D, int FMT>
struct CacheRows {
  static constexpr bool kScaled = FMT != S2_KV_BF16;
  static constexpr int kRowBytes = FMT == S2_KV_BF16 ? 2 * D : FMT == S2_KV_MXFP8 ? D : D / 2;
  static constexpr int kLaneBytes = kRowBytes / 4;
  static constexpr int kDwords = kLaneBytes / 4;
  static constexpr int kLoadBytes = kLaneBytes < 16 ? kLaneBytes : 16;
  static constexpr int kLoads = kLaneBytes / kLoadBytes;
  static constexpr int kFrags = D / 32;  // operands of eight features

  // the first of the eight features that operand kk of lane group g holds
  __device__ static __forceinline__ int feature(int kk, int g) {
    if (FMT == S2_KV_BF16) return 32 * kk + 8 * g;
    if (FMT == S2_KV_MXFP8) return 64 * (kk >> 1) + 16 * g + 8 * (kk & 1);
    return D / 4 * g + 8 * kk;
  }

  // A lane's part of 16 rows: its bytes, and the scale bytes of its row.
  struct Part {
    uint32_t x[kDwords];
    uint32_t scales;
  };

  // rows 0 .. 15 from `at`, of which `rows` exist: the others read as zeros and are not fetched
  __device__ static __forceinline__ void load(Part& p, const uint8_t* at, const uint8_t* scales_at, int rows, int tok, int scale_tok, int r, int g) {
    load_at(p, at, scales_at, rows, tok, scale_tok, r * tok + kLoadBytes * g, r * scale_tok);
  }
  // the same, a lane's bytes beginning at lane_at and its scales at scale_at
  __device__ static __forceinline__ void load_at(Part& p, const uint8_t* at, const uint8_t* scales_at, int rows, int tok, int scale_tok, int lane_at, int scale_at) {
    const auto buf = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(at), 0, rows * tok, 0x00020000);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      if constexpr (kLoadBytes == 16) {
        const u32x4 w = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(buf, lane_at + 64 * j, 0, 0));
#pragma unroll
        for (int e = 0; e < 4; ++e) p.x[4 * j + e] = w[e];
      } else {
        const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(buf, lane_at, 0, 0));
        p.x[0] = w[0];
        p.x[1] = w[1];
      }
    }
    if constexpr (kScaled) {
      const auto sbuf = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(scales_at), 0, rows * scale_tok, 0x00020000);
      p.scales = D == 128 ? __builtin_amdgcn_raw_buffer_load_b32(sbuf, scale_at, 0, 0)
                          : (uint32_t)__builtin_amdgcn_raw_buffer_load_b16(sbuf, scale_at, 0, 0);
    }
  }

  // its operands
  __device__ static __forceinline__ void operands(const Part& p, int g, u32x4 (&out)[kFrags]) {
    if constexpr (FMT == S2_KV_BF16) {
#pragma unroll
      for (int kk = 0; kk < kFrags; ++kk) out[kk] = u32x4{p.x[4 * kk], p.x[4 * kk + 1], p.x[4 * kk + 2], p.x[4 * kk + 3]};
    } else if constexpr (FMT == S2_KV_MXFP8) {
      const uint32_t mine = p.scales >> (8 * (g >> 1));  // the 16 features of a load lie in block 2 * load + g / 2
#pragma unroll
      for (int kk = 0; kk < kFrags; ++kk) {
        const float s = scale_of((mine >> (16 * (kk >> 1))) & 255);
        uint32_t lo[2], hi[2];
        values8(p.x[2 * kk], s, lo);
        values8(p.x[2 * kk + 1], s, hi);
        out[kk] = u32x4{lo[0], lo[1], hi[0], hi[1]};
      }
    } else {
      const float s = scale_of((p.scales >> (8 * (D == 128 ? g : g >> 1))) & 255);
#pragma unroll
      for (int kk = 0; kk < kFrags; ++kk) out[kk] = values4(p.x[kk], s);
    }
  }

  // 8 or 4 bits: a lane's bytes with the operands 2 i and 2 i + 1 in each other's place
  __device__ static __forceinline__ void turn(Part& p, bool turned) {
    constexpr int N = FMT == S2_KV_MXFP8 ? 2 : 1;  // dwords to an operand
#pragma unroll
    for (int i = 0; i < kDwords; ++i)
      if (i % (2 * N) < N) {
        const uint32_t x = p.x[i], y = p.x[i + N];
        p.x[i] = turned ? y : x;
        p.x[i + N] = turned ? x : y;
      }
  }

  // Operand kk as operands() gives it, or (8 or 4 bits, where `turned` is all ones instead of 0) the one beside it in its pair.
  __device__ static __forceinline__ u32x4 operand(const Part& p, int g, int kk, uint32_t turned) {
    auto of = [&](int i, int j) __attribute__((always_inline)) { return (p.x[i] & ~turned) | (p.x[j] & turned); };
    if constexpr (FMT == S2_KV_BF16) {
      return u32x4{p.x[4 * kk], p.x[4 * kk + 1], p.x[4 * kk + 2], p.x[4 * kk + 3]};
    } else if constexpr (FMT == S2_KV_MXFP8) {
      const float s = scale_of((p.scales >> (8 * (g >> 1)) >> (16 * (kk >> 1))) & 255);
      uint32_t lo[2], hi[2];
      values8(of(2 * kk, 2 * (kk ^ 1)), s, lo);
      values8(of(2 * kk + 1, 2 * (kk ^ 1) + 1), s, hi);
      return u32x4{lo[0], lo[1], hi[0], hi[1]};
    } else {
      const float s = scale_of((p.scales >> (8 * (D == 128 ? g : g >> 1))) & 255);
      return values4(of(kk, kk ^ 1), s);
    }
  }

  // acc[8 * kk + e] += pr * (feature e of operand kk), in 32 bits
  __device__ static __forceinline__ void add_times(const Part& p, int g, float pr, float (&acc)[D / 4]) {
    static_assert(kScaled, "");
    const uint32_t mine = p.scales >> (8 * (FMT == S2_KV_MXFP4 && D == 128 ? g : g >> 1));
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {  // pairs
      typedef float f32x2_ __attribute__((ext_vector_type(2)));
      const float s = scale_of((FMT == S2_KV_MXFP8 ? mine >> (16 * (i / 8)) : mine) & 255);
      f32x2_ v;
      if constexpr (FMT == S2_KV_MXFP8) {
        v = i % 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(p.x[i / 2], s, true) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(p.x[i / 2], s, false);
      } else {
        const uint32_t x = p.x[i / 4];
        v = i % 4 == 0   ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x, s, 0)
            : i % 4 == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x, s, 1)
            : i % 4 == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x, s, 2)
                         : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x, s, 3);
      }
      acc[2 * i] = __builtin_fmaf(pr, v[0], acc[2 * i]);
      acc[2 * i + 1] = __builtin_fmaf(pr, v[1], acc[2 * i + 1]);
    }
  }
};

}  // namespace s2
