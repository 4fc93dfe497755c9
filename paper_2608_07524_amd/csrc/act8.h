// Device side of the 8-bit activation checkpoints, shared by the kernels that
// write or read them, and the wavefront sums of the row-wise kernels.
//
// A checkpoint of a bf16 row holds one 8-bit code an element and one scale byte
// for each group of 32 consecutive columns (the last group of a row may be
// shorter).  With qmax = 127 (int8) or 448 (e4m3), k is the smallest integer >=
// -126 with max |x| <= qmax 2^k over the group; the byte is k + 127, the code
// x / 2^k rounded to the format (nearest, ties to even), the value it stands for
// code 2^k.  Powers of two make both directions exact but for that one rounding:
// x 2^-k and code 2^k are exact in fp32 and code 2^k is exact in bf16 (2^128, to
// which values next to it round, is infinity there), so a checkpoint is the same
// bits wherever it is made, and reading it back in bf16 loses nothing.  (A scale that
// is not a power of two would use the range of int8 better, by 0.4 bit on average, and
// round twice.)  A group that holds a NaN or an infinity gets byte 255 and codes 0,
// which read back as NaN.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dcp.h"

namespace dcp {

constexpr int kActGroup = 32;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), CTRL, 0xf, 0xf, false));
}
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __uint_as_float(dpp<CTRL>(__float_as_uint(v)));
}
constexpr int kQuadXor1 = 0xB1, kQuadXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;

// Sum over each aligned run of L lanes (a power of two up to 64), the same in all
// of them: within 16 lanes by data-parallel moves of the vector ALU, across them by
// lane swaps; no trip through LDS.
template <int L>
__device__ __forceinline__ float lane_total(float v) {
  if constexpr (L >= 2) v = dpp_add<kQuadXor1>(v);
  if constexpr (L >= 4) v = dpp_add<kQuadXor2>(v);
  if constexpr (L >= 8) v = dpp_add<kHalfMirror>(v);
  if constexpr (L >= 16) v = dpp_add<kMirror>(v);
  if constexpr (L >= 32) {
    const u32x2 s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
  if constexpr (L >= 64) {
    const u32x2 s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
  return v;
}

// Largest magnitude of a lane's 8 values, as bf16 bits (ordered as integers, NaN
// above infinity).
__device__ __forceinline__ uint32_t top_bits(bf16x8 v) {
  const u32x4 w = __builtin_bit_cast(u32x4, v);
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = max(m, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
  return m;
}

// The same over the group's four lanes (lanes 4i .. 4i+3 hold one group).
__device__ __forceinline__ uint32_t group_top(uint32_t m) {
  m = max(m, dpp<kQuadXor1>(m));
  return max(m, dpp<kQuadXor2>(m));
}

// Scale byte of a group from its largest magnitude: mantissas that would pass
// qmax (int8: 127 = 1.984375 2^6, mantissa bits 0x7e; e4m3: 448 = 1.75 2^8, 0x60)
// carry into the exponent.
template <int FMT>
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  constexpr uint32_t carry = FMT == DCP_ACT_INT8 ? 0x01 : 0x1f;
  constexpr int down = FMT == DCP_ACT_INT8 ? 6 : 8;
  const int e = int((top + carry) >> 7) - down;
  return top >= 0x7f80u ? 255u : uint32_t(max(e, 1));
}

// Codes of a lane's 8 values under scale byte b.
template <int FMT>
__device__ __forceinline__ u32x2 encode8(bf16x8 v, uint32_t b) {
  const float inv = __uint_as_float((254u - b) << 23);
  u32x2 r;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = float(v[4 * h + i]);
    if constexpr (FMT == DCP_ACT_INT8) {
      // 1.5 2^23 puts the integer, rounded to nearest even, into the low bits
      uint32_t c[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = __float_as_uint(__builtin_fmaf(x[i], inv, 12582912.f));
      r[h] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(c[3], c[2], 0x0c0c0400u),
                                   __builtin_amdgcn_perm(c[1], c[0], 0x0c0c0400u), 0x05040100u);
    } else {
      int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
      r[h] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, w, true));
    }
  }
  return b == 255u ? u32x2{0u, 0u} : r;
}

// The values that 8 codes under scale byte b stand for (exact).
template <int FMT>
__device__ __forceinline__ void decode8(u32x2 c, uint32_t b, float (&x)[8]) {
  const float s = __uint_as_float(b << 23);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if constexpr (FMT == DCP_ACT_INT8) {
      const uint32_t u = c[h] ^ 0x80808080u;  // code + 128, unsigned
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * h + i] = (float((u >> (8 * i)) & 0xffu) - 128.f) * s;
    } else {
      typedef float f32x2 __attribute__((ext_vector_type(2)));
      const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(int(c[h]), false);
      const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(int(c[h]), true);
      x[4 * h] = lo[0] * s;
      x[4 * h + 1] = lo[1] * s;
      x[4 * h + 2] = hi[0] * s;
      x[4 * h + 3] = hi[1] * s;
    }
  }
}

// The same times m, rounded once, for 2^k m below 2^121: int8 passes 128 2^k m.  A row's
// scale 1 / rms holds that, being 0 in fp32 where k is 121 or 122; m = 1 does not.
template <int FMT>
__device__ __forceinline__ void decode8_scaled(u32x2 c, uint32_t b, float m, float (&x)[8]) {
  if constexpr (FMT == DCP_ACT_INT8) {
    const float s = __uint_as_float(b << 23) * m, off = -128.f * s;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t u = c[h] ^ 0x80808080u;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * h + i] = __builtin_fmaf(float((u >> (8 * i)) & 0xffu), s, off);
    }
  } else {
    decode8<FMT>(c, b, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= m;
  }
}

// GELU, tanh form, through the logistic function: with w = k0 (u + k1 u^3),
// (1 + tanh w) / 2 = s(2w) = 1 / (1 + e^(-2w)), so a = u s and
// da/du = s + 2 k0 u s (1 - s) (1 + 3 k1 u^2).  s is 0 or 1 in fp32 beyond |u| = 16,
// where the powers of u are cut so that they stay finite.
__device__ __forceinline__ void gelu_and_slope(float u, float* a, float* slope) {
  constexpr float k0 = 0.7978845608028654f, k1 = 0.044715f, log2e = 1.4426950408889634f;
  const float c = fminf(fmaxf(u, -16.f), 16.f), cc = c * c;
  const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-2.f * k0 * log2e * c * (1.f + k1 * cc)));
  *a = u * s;
  *slope = s + u * (s * (1.f - s) * (2.f * k0 + 6.f * k0 * k1 * cc));
}

// Eight consecutive values of a stored activation: bf16, or codes and their byte.
template <int FMT>
struct Held8 {
  u32x2 c;
  uint32_t b;
  __device__ __forceinline__ void load(const void* p, const uint8_t* scales, int64_t at, int64_t group) {
    c = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(p) + at);
    b = scales[group];
  }
  __device__ __forceinline__ void get(float (&x)[8]) const { decode8<FMT>(c, b, x); }
  __device__ __forceinline__ void get_scaled(float m, float (&x)[8]) const { decode8_scaled<FMT>(c, b, m, x); }
};
template <>
struct Held8<DCP_ACT_BF16> {
  bf16x8 v;
  __device__ __forceinline__ void load(const void* p, const uint8_t*, int64_t at, int64_t) {
    v = *reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(p) + at);
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = float(v[i]);
  }
  __device__ __forceinline__ void get_scaled(float m, float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = float(v[i]) * m;
  }
};

}  // namespace dcp
