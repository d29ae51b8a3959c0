// ss_quant.hip -- the 4-bit form of a vocabulary table (ss_quant_w4).
//
// A thread takes eight consecutive columns, which become one dword of codes;
// the 4, 8 or 16 threads of a group agree on its largest magnitude by shuffles
// within the wavefront.  Each weight is read once and each code written once.
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
  int wide_in, wide_out;  // rows of w / values can be read / written 16 bytes at a time
};

// VDT: the type of `values`, or -1 for none.
template <int KIND, int DT, int VDT>
__global__ __launch_bounds__(256) void ss_quant_kernel(QArgs a) {
  constexpr int G = w4_group(KIND);
  const int octets = a.nb * 16;  // of a row
  const int64_t i = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
  const int64_t row64 = i / octets;
  if (row64 >= a.V) return;  // whole groups: octets is a multiple of 16
  const int row = (int)row64;
  const int o = (int)(i - row64 * octets);
  const int col = o * 8;
  const bool in = col < a.H;  // H is a multiple of the group: a group is in or out as a whole
  float x[8];
  if (in) {
    row_load8<DT>(a.w, (int64_t)row * a.ld + col, 8, a.wide_in, x);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = 0.0f;
  }
  // magnitudes as bits: order is preserved and what is not finite is largest
  uint32_t top = 0u;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const uint32_t m = __float_as_uint(x[k]) & 0x7FFFFFFFu;
    top = m > top ? m : top;
  }
#pragma unroll
  for (int d = 1; d < G / 8; d *= 2) {
    const uint32_t other = __shfl_xor(top, d);
    top = other > top ? other : top;
  }
  const bool finite = top < 0x7F800000u;
  uint32_t word = 0u;
  float val[8];
  const int64_t group = (int64_t)row * (a.nb * w4_groups(KIND)) + o / (G / 8);
  const bool first = o % (G / 8) == 0;
  if constexpr (KIND == kMx) {
    // floor(log2 top) - 2 + 127, from the exponent field (0 for subnormals)
    const int e = (int)(top >> 23) - 2;
    const uint32_t sb = !finite ? 255u : (uint32_t)(e < 0 ? 0 : e);
    const float s = mx_scale(finite ? sb : 127u);
    if (finite) {
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[0], x[1], s, 0);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[2], x[3], s, 1);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[4], x[5], s, 2);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[6], x[7], s, 3);
    }
    if (first) reinterpret_cast<uint8_t*>(a.scales)[group] = (uint8_t)sb;
    if constexpr (VDT >= 0) {
      const f32x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, s, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, s, 1);
      const f32x2 v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, s, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, s, 3);
      val[0] = v0.x, val[1] = v0.y, val[2] = v1.x, val[3] = v1.y, val[4] = v2.x, val[5] = v2.y, val[6] = v3.x, val[7] = v3.y;
    }
  } else {
    const float amax = __uint_as_float(top);
    const uint32_t sb = finite ? bf16_bits(amax / 7.0f) : 0x7FC0u;
    if (first) reinterpret_cast<uint16_t*>(a.scales)[group] = (uint16_t)sb;
    const float s0 = bf16_value(sb);
    // small groups are taken 2^64 times larger (exact), so that 1 / s exists
    const float up = amax < 0x1p-60f ? 0x1p64f : 1.0f;
    const float s = s0 * up;
    const bool ok = finite && s0 > 0.0f;
    const float inv = ok ? 1.0f / s : 0.0f, half = 0.5f * s;
    uint32_t c[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      // m is |x| / s rounded, off by one at most where the quotient is close to a
      // tie.  There d = |x| - m s is exact (a multiple of |x|'s last place, no larger
      // than |x|), so comparing it with s / 2 decides as the exact quotient
      // does; a tie moves an odd m only, to the even neighbour.
      const float ax = fabsf(x[k]) * up;
      int m = (int)__builtin_rintf(ax * inv);
      const float d = ok ? __builtin_fmaf(-(float)m, s, ax) : 0.0f;
      const float bound = __uint_as_float(__float_as_uint(half) - (uint32_t)(m & 1));
      if (fabsf(d) > bound) m += d > 0.0f ? 1 : -1;
      m = !ok ? 0 : m > 7 ? 7 : m;
      const uint32_t sign = finite ? __float_as_uint(x[k]) >> 31 : 0u;
      c[k] = (uint32_t)m | sign << 7;
      if constexpr (VDT >= 0) val[k] = __uint_as_float(__float_as_uint((float)m * s0) | sign << 31);
    }
    const uint32_t A = c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, B = c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24;
    word = A | (B << 4 | B >> 28);
  }
  if constexpr (VDT >= 0) {
    if (!finite) {
#pragma unroll
      for (int k = 0; k < 8; ++k) val[k] = __uint_as_float(0x7FC00000u);
    }
    if (in) row_store8<VDT>(a.values, (int64_t)row * a.ld_values + col, 8, a.wide_out, val);
  }
  const int ob = o & 15;  // octet 4 j + g of its block -> dword 4 g + j
  a.codes[((int64_t)row * a.nb + (o >> 4)) * 16 + (ob & 3) * 4 + (ob >> 2)] = word;
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
  const int64_t threads = (int64_t)t->V * a.nb * 16;
  // a launch has fewer than 2^32 threads in one direction
  const int64_t blocks = (threads + 255) / 256, most = 1 << 20;
  const dim3 grid((unsigned)(blocks < most ? blocks : most), (unsigned)((blocks + most - 1) / most));
  const int vdt = values ? values_dtype : -1;
  if (dtype == SS_BF16)
    launch_quant_kind<SS_BF16>(kind, a, vdt, grid, (hipStream_t)stream);
  else
    launch_quant_kind<SS_F32>(kind, a, vdt, grid, (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_HIP;
}

}  // extern "C"
