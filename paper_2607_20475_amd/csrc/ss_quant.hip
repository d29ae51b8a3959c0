// ss_quant.hip -- the 4-bit form of a vocabulary table (ss_quant_w4).
//
// Each weight is read once and each code written once: bound by memory.  A
// wave takes strips of 512 columns of a row, eight a lane: an octet that follows on
// the lane before where all rows are bfloat16, two quads 256 columns apart where one
// side is float32, so that a wave's loads and stores are 16 bytes a lane and
// lie together either way.  The lanes of a group agree on its largest magnitude
// by shuffles; two lanes with the halves of an octet join them into its dword.
//   V = 131072, H = 4096, bfloat16 with values, int128: 408 us, 5.9 TB/s read and written; V = 32768, H = 2048, float32 with values,
// mx: 99 us, 5.8 TB/s (a fill alone reaches 6.8).
#include <hip/hip_runtime.h>

#include "ss_w4.hpp"

namespace ss {

struct QArgs {
  const void* w;
  uint32_t* codes;
  void* scales;
  void* values;
  int64_t ld, ld_values;
  int V, H, nb;
  int row_waves;          // of a row: one, or the workgroup's four
  int wide_in, wide_out;  // rows of w / values can be read / written 16 bytes at a time
};

// Magnitudes |x| / s rounded to integers (ties to even) as floats; up to 7 (a normal s is at least amax / 7 less
// half a step of bfloat16: quotients stay below 7.02).  inv is 1 / s rounded.
//   bfloat16: the quotient of two 8-bit significands is a tie or at least 2^-10 away from
//   one, and |x| * inv is off by less than 2^-20: rounded to multiples of 2^-13 it is a tie
//   exactly where the quotient is one.
//   float32: |x| * inv rounded is off by one at most, where the quotient is close to a tie.  There d =
//   |x| - m s is exact (a multiple of |x|'s last place, no larger than |x|), so comparing it with
//   s / 2 decides as the exact quotient does; a tie moves an odd m only, to the even neighbour.
template <int DT>
__device__ __forceinline__ float magnitude(float x, float s, float inv) {
  const float r = fabsf(x) * inv;
  if constexpr (DT == SS_BF16) {
    return __builtin_rintf((r + 1536.0f) - 1536.0f);  // 1.5 * 2^10: a last place of 2^-13
  } else {
    const float m = __builtin_rintf(r), d = __builtin_fmaf(-m, s, fabsf(x)), half = 0.5f * s;
    const float bound = __uint_as_float(__float_as_uint(half) - ((uint32_t)m & 1u));
    return fabsf(d) > bound ? m + (d > 0.0f ? 1.0f : -1.0f) : m;
  }
}

// Replaces byte `at` of `to` by a small float's integer.
__device__ __forceinline__ uint32_t put_byte(float m, int at, uint32_t to) {
  return __builtin_amdgcn_cvt_pk_u8_f32(m, at, to);
}

// Four columns of a row in float32; `wide`: aligned.
template <int DT>
__device__ __forceinline__ void load4(const void* p, int64_t at, bool wide, float x[4]) {
  if constexpr (DT == SS_F32) {
    const float* f = reinterpret_cast<const float*>(p) + at;
    if (wide) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(f);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = v[i];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = f[i];
    }
  } else {
    const uint16_t* h = reinterpret_cast<const uint16_t*>(p) + at;
    if (wide) {
      const uint2 u = *reinterpret_cast<const uint2*>(h);
      x[0] = __uint_as_float(u.x << 16), x[1] = __uint_as_float(u.x & 0xFFFF0000u);
      x[2] = __uint_as_float(u.y << 16), x[3] = __uint_as_float(u.y & 0xFFFF0000u);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = bf16_value(h[i]);
    }
  }
}

template <int DT>
__device__ __forceinline__ void store4(void* p, int64_t at, bool wide, const float x[4]) {
  if constexpr (DT == SS_F32) {
    float* f = reinterpret_cast<float*>(p) + at;
    if (wide) {
      *reinterpret_cast<f32x4*>(f) = f32x4{x[0], x[1], x[2], x[3]};
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = x[i];
    }
  } else {
    uint16_t* h = reinterpret_cast<uint16_t*>(p) + at;
    if (wide) {
      *reinterpret_cast<uint2*>(h) = make_uint2(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = (uint16_t)bf16_bits(x[i]);
    }
  }
}

// The codes of N columns (8: an octet, 4: its half `hi`) as their bits of the octet's dword, their group's scale
// (written if `write`), and the values.  LANES lanes hold a group.
template <int KIND, int DT, int VDT, int N, int LANES>
__device__ __forceinline__ uint32_t quantise(float x[N], bool hi, void* scales, int64_t group, bool write, float val[N]) {
  // magnitudes as bits: order is preserved and what is not finite is largest
  uint32_t top = 0u;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const uint32_t m = __float_as_uint(x[k]) & 0x7FFFFFFFu;
    top = m > top ? m : top;
  }
#pragma unroll
  for (int d = 1; d < LANES; d *= 2) {
    const uint32_t other = __shfl_xor(top, d);
    top = other > top ? other : top;
  }
  const bool finite = top < 0x7F800000u;
  uint32_t word = 0u;
  if constexpr (KIND == kMx) {
    // floor(log2 top) - 2 + 127, from the exponent field (0 for subnormals)
    const int e = (int)(top >> 23) - 2;
    const uint32_t sb = !finite ? 255u : (uint32_t)(e < 0 ? 0 : e);
    const float s = mx_bits(sb);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[0], x[1], s, 0);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[2], x[3], s, 1);
    if constexpr (N == 8) {
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[4], x[5], s, 2);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[6], x[7], s, 3);
    }
    if (!finite) word = 0u;
    if (write) reinterpret_cast<uint8_t*>(scales)[group] = (uint8_t)sb;
    if constexpr (VDT >= 0) {
      const f32x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, s, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, s, 1);
      val[0] = v0.x, val[1] = v0.y, val[2] = v1.x, val[3] = v1.y;
      if constexpr (N == 8) {
        const f32x2 v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, s, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, s, 3);
        val[4] = v2.x, val[5] = v2.y, val[6] = v3.x, val[7] = v3.y;
      }
    }
    if (N == 4 && hi) word <<= 16;
  } else {
    const float amax = __uint_as_float(top);
    const uint32_t sb = finite ? bf16_bits(amax / 7.0f) : 0x7FC0u;
    if (write) reinterpret_cast<uint16_t*>(scales)[group] = (uint16_t)sb;
    const float s0 = bf16_value(sb);
    float s = s0;
    if (amax < 0x1p-60f) {
      // taken 2^64 times larger (exact), so that 1 / s exists; a subnormal scale may be so much smaller
      // than amax / 7 that quotients pass 7
      s *= 0x1p64f;
#pragma unroll
      for (int k = 0; k < N; ++k) x[k] = __builtin_amdgcn_fmed3f(x[k] * 0x1p64f, -7.0f * s, 7.0f * s);
    }
    const float inv = s > 0.0f ? 1.0f / s : 0.0f;
    uint32_t part[N / 4], sign[N / 4];
#pragma unroll
    for (int h = 0; h < N / 4; ++h) {
      part[h] = 0u;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float m = magnitude<DT>(x[4 * h + k], s, inv);
        part[h] = put_byte(m, k, part[h]);
        if constexpr (VDT >= 0) val[4 * h + k] = __builtin_copysignf(m, x[4 * h + k]) * s0;
      }
      const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(x[4 * h + 1]), __float_as_uint(x[4 * h]), 0x0C0C0703u);
      sign[h] = __builtin_amdgcn_perm(__float_as_uint(x[4 * h + 3]), __float_as_uint(x[4 * h + 2]), 0x07030C0Cu) | lo;
      part[h] |= sign[h] & 0x80808080u;
    }
    if constexpr (N == 8)
      word = part[0] | __builtin_amdgcn_alignbit(part[1], part[1], 28);
    else
      word = hi ? __builtin_amdgcn_alignbit(part[0], part[0], 28) : part[0];
    if (s <= 0.0f) word &= 0x80808080u | 0x08080808u;  // a zero scale: signs alone
    if (!finite) word = 0u;
  }
  if constexpr (VDT >= 0) {
    if (!finite) {
#pragma unroll
      for (int k = 0; k < N; ++k) val[k] = __uint_as_float(0x7FC00000u);
    }
  }
  return word;
}

// VDT: the type of `values`, or -1 for none.
template <int KIND, int DT, int VDT>
__global__ __launch_bounds__(256) void ss_quant_kernel(QArgs a) {
  constexpr int G = w4_group(KIND);
  constexpr bool QUADS = DT == SS_F32 || VDT == SS_F32;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int strips = (a.nb + 3) / 4;
  const int row = a.row_waves == 4 ? blockIdx.x : blockIdx.x * 4 + wave;
  if (row >= a.V) return;
  const int64_t in0 = (int64_t)row * a.ld, out0 = (int64_t)row * a.ld_values, block0 = (int64_t)row * a.nb;
  for (int s = a.row_waves == 4 ? wave : 0; s < strips; s += a.row_waves) {
    if constexpr (QUADS) {
      float x[2][4], val[2][4];
      uint32_t word[2];
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int col = s * 512 + p * 256 + lane * 4;
        if (col < a.H) {  // H is a multiple of the group: a group is in or out as a whole
          load4<DT>(a.w, in0 + col, a.wide_in, x[p]);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) x[p][k] = 0.0f;
        }
      }
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int col = s * 512 + p * 256 + lane * 4;
        word[p] = quantise<KIND, DT, VDT, 4, G / 4>(x[p], lane & 1, a.scales, block0 * w4_groups(KIND) + col / G,
                                                    lane % (G / 4) == 0 && col < a.nb * kBlockCols, val[p]);
        word[p] |= __shfl_xor(word[p], 1);
        if constexpr (VDT >= 0) {
          if (col < a.H) store4<VDT>(a.values, out0 + col, a.wide_out, val[p]);
        }
      }
      // even lanes write the first half's dword, odd lanes the second's
      const int o = s * 64 + (lane & 1) * 32 + (lane >> 1), ob = o & 15;
      if (o < a.nb * 16) a.codes[(block0 + (o >> 4)) * 16 + (ob & 3) * 4 + (ob >> 2)] = lane & 1 ? word[1] : word[0];
    } else {
      const int o = s * 64 + lane, ob = o & 15, col = o * 8;
      float x[8], val[8];
      if (col < a.H) {
        row_load8<DT>(a.w, in0 + col, 8, a.wide_in, x);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = 0.0f;
      }
      const uint32_t word = quantise<KIND, DT, VDT, 8, G / 8>(x, false, a.scales, block0 * w4_groups(KIND) + col / G,
                                                              lane % (G / 8) == 0 && o < a.nb * 16, val);
      if constexpr (VDT >= 0) {
        if (col < a.H) row_store8<VDT>(a.values, out0 + col, 8, a.wide_out, val);
      }
      // octet 4 j + g of its block -> dword 4 g + j
      if (o < a.nb * 16) a.codes[(block0 + (o >> 4)) * 16 + (ob & 3) * 4 + (ob >> 2)] = word;
    }
  }
}

template <int KIND, int DT>
static void launch_quant(const QArgs& a, int vdt, dim3 grid, hipStream_t st) {
  if (vdt == SS_F32)
    hipLaunchKernelGGL((ss_quant_kernel<KIND, DT, SS_F32>), grid, dim3(256), 0, st, a);
  else if (vdt == SS_BF16)
    hipLaunchKernelGGL((ss_quant_kernel<KIND, DT, SS_BF16>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((ss_quant_kernel<KIND, DT, -1>), grid, dim3(256), 0, st, a);
}

template <int DT>
static void launch_quant_kind(int kind, const QArgs& a, int vdt, dim3 grid, hipStream_t st) {
  switch (kind) {
    case kInt128: launch_quant<kInt128, DT>(a, vdt, grid, st); break;
    case kInt64: launch_quant<kInt64, DT>(a, vdt, grid, st); break;
    case kInt32: launch_quant<kInt32, DT>(a, vdt, grid, st); break;
    default: launch_quant<kMx, DT>(a, vdt, grid, st); break;
  }
}

}  // namespace ss

using namespace ss;

extern "C" {

size_t ss_w4_codes_bytes(const ss_w4* t) {
  if (!t || w4_kind(t) < 0) return 0;
  return (size_t)t->V * w4_blocks(t->H) * kBlockBytes;
}

size_t ss_w4_scales_bytes(const ss_w4* t) {
  const int kind = t ? w4_kind(t) : -1;
  if (kind < 0) return 0;
  return (size_t)t->V * w4_blocks(t->H) * w4_scale_bytes(kind);
}

ss_status ss_quant_w4(const void* w, int dtype, int64_t ld, const ss_w4* t, void* values, int values_dtype,
                      int64_t ld_values, void* stream) {
  if (!w || !t || (dtype != SS_F32 && dtype != SS_BF16)) return SS_ERR_INVALID_ARG;
  const int kind = w4_kind(t);
  if (kind < 0 || !w4_aligned(t->codes) || !w4_aligned(t->scales) || ld < t->H) return SS_ERR_INVALID_ARG;
  if (values && ((values_dtype != SS_F32 && values_dtype != SS_BF16) || ld_values < t->H)) return SS_ERR_INVALID_ARG;
  QArgs a = {};
  a.w = w;
  a.ld = ld;
  a.codes = reinterpret_cast<uint32_t*>(const_cast<void*>(t->codes));
  a.scales = const_cast<void*>(t->scales);
  a.values = values;
  a.ld_values = ld_values;
  a.V = t->V;
  a.H = t->H;
  a.nb = w4_blocks(t->H);
  a.wide_in = wide_rows(w, ld, dtype);
  a.wide_out = values && wide_rows(values, ld_values, values_dtype);
  a.row_waves = a.nb >= 16 ? 4 : 1;
  const dim3 grid((unsigned)(a.row_waves == 4 ? t->V : (t->V + 3) / 4));
  const int vdt = values ? values_dtype : -1;
  if (dtype == SS_BF16)
    launch_quant_kind<SS_BF16>(kind, a, vdt, grid, (hipStream_t)stream);
  else
    launch_quant_kind<SS_F32>(kind, a, vdt, grid, (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_HIP;
}

}  // extern "C"
