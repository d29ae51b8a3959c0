// ss_w4.hpp -- the 4-bit vocabulary table: layout, decoding, argument checks.
//
// A row holds ceil(H / 128) blocks of 64 bytes; dword 4 g + j of a block (g, j
// = 0..3) holds columns 32 j + 8 g .. + 7.  The order is the matrix
// instruction's: its B operand asks lane (n, g) for row n and columns 8 g .. + 7
// of a step j of 32 columns, so one 16-byte load a lane feeds the four steps
// of a block, whatever the group size, and the other operand (the hidden
// states) is read in its natural order.  Rows stay contiguous, so the lookup
// reads whole cache lines.  A wave's load covers 16 rows by 64 bytes; on
// this card such loads stream at 6.1 to 6.4 TB/s, the same as loads of 1 KB
// that lie together (measured over 268 MB).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ss.h"

namespace ss {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Kinds of table: integers with groups of 128, 64 and 32 columns, and E2M1.
enum W4Kind { kInt128 = 0, kInt64 = 1, kInt32 = 2, kMx = 3 };

constexpr int kBlockCols = 128;
constexpr int kBlockBytes = 64;
__host__ __device__ constexpr int w4_group(int kind) { return kind == kInt128 ? 128 : kind == kInt64 ? 64 : 32; }
__host__ __device__ constexpr int w4_groups(int kind) { return kBlockCols / w4_group(kind); }  // of a block
__host__ __device__ constexpr int w4_scale_bytes(int kind) { return kind == kMx ? 4 : 2 * w4_groups(kind); }  // of a block

__host__ __device__ inline int w4_blocks(int H) { return (H + kBlockCols - 1) / kBlockCols; }

// The kind of a table, or -1 if its sizes or format are not offered.
inline int w4_kind(const ss_w4* t) {
  if (t->V < 1 || t->V > SS_MAX_V || t->H < 1 || t->H > SS_MAX_H) return -1;
  const int G = t->group;
  if (t->fmt == SS_W4_MX) {
    if (G != 32 || t->H % 32) return -1;
    return kMx;
  }
  if (t->fmt != SS_W4_INT || (G != 32 && G != 64 && G != 128) || t->H % G) return -1;
  return G == 128 ? kInt128 : G == 64 ? kInt64 : kInt32;
}

inline bool w4_aligned(const void* p) { return p && ((uintptr_t)p & 15u) == 0; }

__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }

// float32 to bfloat16, nearest with ties to even (NaN stays NaN)
__device__ __forceinline__ uint32_t bf16_bits(float x) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x);
}

// Two bfloat16 of a pair of floats.
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) { return bf16_bits(lo) | bf16_bits(hi) << 16; }

__device__ __forceinline__ uint32_t as_u32(bf16x2 v) { return __builtin_bit_cast(uint32_t, v); }

// The eight elements of a dword as bfloat16, two a register.
//   E2M1: the hardware conversion, times a power of two; exact.
//   Integers: the bytes s0000mmm of a half are E4M3 numbers of the lowest binades,
//   m * 2^-9 with their sign, so the conversion times 2^9 gives the integer; exact
//   in bfloat16.  Seven instructions for eight elements (four for E2M1).  The
//   group's scale is left to the caller: a product of integer and scale has up
//   to 11 bits and would be rounded in bfloat16, the sum over a group is scaled in float32.
// `scale` (E2M1) is mx_bits of the group's scale.
template <int KIND>
__device__ __forceinline__ u32x4 w4_expand(uint32_t w, float scale) {
  u32x4 r;
  if constexpr (KIND == kMx) {
    r.x = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
    r.y = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
    r.z = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
    r.w = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  } else {
    const uint32_t a = w & 0x87878787u, b = __builtin_amdgcn_alignbit(w, w, 4) & 0x87878787u;
    r.x = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 512.0f, false));
    r.y = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 512.0f, true));
    r.z = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 512.0f, false));
    r.w = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 512.0f, true));
  }
  return r;
}

// The scale of an E2M1 group as the conversions take it: they read the exponent field alone, 0 as 2^-127
// and 255 as NaN.
__device__ __forceinline__ float mx_bits(uint32_t x) { return __uint_as_float(x << 23); }

// The scale of an E2M1 group: 2^(x - 127), x = 0 the subnormal 2^-127, x = 255 NaN.
__device__ __forceinline__ float mx_scale(uint32_t x) {
  return x ? __uint_as_float(x == 255u ? 0x7FC00000u : x << 23) : __uint_as_float(0x00400000u);
}

// Eight columns of a row, `left` of which it has, in float32.  `wide`: rows start at multiples of
// 16 bytes (wide_rows).
template <int DT>
__device__ __forceinline__ void row_load8(const void* p, int64_t at, int left, bool wide, float x[8]) {
  if (DT == SS_F32) {
    const float* f = reinterpret_cast<const float*>(p) + at;
    if (wide && left >= 8) {
      const float4 a = reinterpret_cast<const float4*>(f)[0], b = reinterpret_cast<const float4*>(f)[1];
      x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = i < left ? f[i] : 0.0f;
    }
  } else {
    const uint16_t* h = reinterpret_cast<const uint16_t*>(p) + at;
    if (wide && left >= 8) {
      const uint4 a = *reinterpret_cast<const uint4*>(h);
      const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) x[2 * i] = bf16_value(u[i] & 0xFFFFu), x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = i < left ? bf16_value(h[i]) : 0.0f;
    }
  }
}

template <int DT>
__device__ __forceinline__ void row_store8(void* p, int64_t at, int left, bool wide, const float x[8]) {
  if (DT == SS_F32) {
    float* f = reinterpret_cast<float*>(p) + at;
    if (wide && left >= 8) {
      reinterpret_cast<float4*>(f)[0] = make_float4(x[0], x[1], x[2], x[3]);
      reinterpret_cast<float4*>(f)[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) f[i] = x[i];
    }
  } else {
    uint16_t* h = reinterpret_cast<uint16_t*>(p) + at;
    if (wide && left >= 8) {
      *reinterpret_cast<uint4*>(h) =
          make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) h[i] = (uint16_t)bf16_bits(x[i]);
    }
  }
}

// Whether octets of columns of every row start at multiples of 16 bytes.
inline bool wide_rows(const void* p, int64_t ld, int dt) {
  return ((uintptr_t)p & 15u) == 0 && (ld * (dt == SS_F32 ? 4 : 2)) % 16 == 0;
}

}  // namespace ss
