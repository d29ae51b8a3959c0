// ss_head.hip -- logits of hidden states under a 4-bit vocabulary table
// (ss_head_w4): logits[t, v] = sum_k h[t, k] W[v, k].
//
// The matrix instruction (16 x 16 x 32, bfloat16 with float32 sums) takes the hidden
// rows as its A operand and the table's rows as its B operand, so a lane's
// four results are one vocabulary row at four tokens, and the group's scale
// is one register.  Codes become bfloat16 exactly (w4_expand); integer
// tables sum a group unscaled and scale the sum in float32.  float32 hidden
// states are split into three bfloat16 parts whose sum they are (24 bits in three
// times 8), one matrix instruction each into the same sums.
//
// Two kernels:
//   ss_head_few_kernel   up to 16 tokens: bound by the table's read.  The four
//                        waves of a workgroup split the row's blocks and join their
//                        sums through LDS; hidden states come from the caches.
//   ss_head_many_kernel  more tokens: each wave has its own vocabulary rows,
//                        the workgroup shares the hidden states of a block of
//                        128 columns in LDS.
#include <hip/hip_runtime.h>

#include "ss_w4.hpp"

namespace ss {

struct HeadArgs {
  const __bf16* h;        // parts of the hidden states, [P][T, ld_h]
  int64_t ld_h, part;     // elements from one row / part to the next
  const uint8_t* codes;
  const uint8_t* scales;
  void* out;
  int64_t ld;
  int T, V, H, nb;
  int out_f32;
  int wide;               // out rows can be written several columns at a time
  int tblocks, vblocks;   // token and vocabulary blocks (many)
};

// --------------------------------------------------------------------------
// Hidden states as bfloat16 parts, or a copy whose rows start at multiples of 16 bytes
// --------------------------------------------------------------------------
template <int DT>
__global__ __launch_bounds__(256) void ss_head_parts_kernel(const void* h, int64_t ld, int T, int H, uint16_t* out) {
  const int64_t n = (int64_t)T * H;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t t = i / H, k = i - t * H;
    if constexpr (DT == SS_F32) {
      // cut, not rounded: each part takes the next eight bits, the rests are exact
      const float x = reinterpret_cast<const float*>(h)[t * ld + k];
      const uint32_t b0 = __float_as_uint(x);
      const float r1 = x - __uint_as_float(b0 & 0xFFFF0000u);
      const uint32_t b1 = __float_as_uint(r1);
      const float r2 = r1 - __uint_as_float(b1 & 0xFFFF0000u);
      const bool fine = (b0 & 0x7F800000u) != 0x7F800000u;
      // a NaN whose high bits are those of an infinity stays a NaN
      out[i] = (uint16_t)(b0 >> 16 | ((b0 & 0x7FFFFFFFu) > 0x7F800000u ? 0x40u : 0u));
      out[n + i] = fine ? (uint16_t)(b1 >> 16) : (uint16_t)0;
      out[2 * n + i] = fine ? (uint16_t)(__float_as_uint(r2) >> 16) : (uint16_t)0;
    } else {
      out[i] = reinterpret_cast<const uint16_t*>(h)[t * ld + k];
    }
  }
}

// --------------------------------------------------------------------------
// Pieces
// --------------------------------------------------------------------------
__device__ __forceinline__ bf16x8 as_bf16x8(uint4 v) { return __builtin_bit_cast(bf16x8, v); }

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// The scales of a row's block, as loaded: 2, 4 or 8 bytes.
template <int KIND>
struct ScaleWord {
  uint32_t lo, hi;
};

template <int KIND>
__device__ __forceinline__ ScaleWord<KIND> load_scales(const uint8_t* row, int block) {
  ScaleWord<KIND> s = {0u, 0u};
  const uint8_t* p = row + (int64_t)block * w4_scale_bytes(KIND);
  if constexpr (KIND == kInt128) {
    s.lo = *reinterpret_cast<const uint16_t*>(p);
  } else if constexpr (KIND == kInt32) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    s.lo = v.x, s.hi = v.y;
  } else {
    s.lo = *reinterpret_cast<const uint32_t*>(p);
  }
  return s;
}

// The scale of step j (32 columns) of a block.
template <int KIND>
__device__ __forceinline__ float step_scale(ScaleWord<KIND> s, int j) {
  if constexpr (KIND == kMx) {
    return mx_scale(s.lo >> (8 * j) & 255u);
  } else {
    const int i = j / (4 / w4_groups(KIND));
    const uint32_t w = i < 2 ? s.lo : s.hi;
    return i & 1 ? __uint_as_float(w & 0xFFFF0000u) : bf16_value(w & 0xFFFFu);
  }
}

__device__ __forceinline__ uint32_t dword(uint4 v, int j) { return j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w; }

// Writes NV consecutive columns of one token.
template <int NV>
__device__ __forceinline__ void store_cols(const HeadArgs& a, int t, int v, const float x[NV]) {
  const int64_t at = (int64_t)t * a.ld + v;
  if (a.out_f32) {
    float* o = reinterpret_cast<float*>(a.out) + at;
    if (NV == 4 && a.wide && v + NV <= a.V) {
      *reinterpret_cast<float4*>(o) = make_float4(x[0], x[1 % NV], x[2 % NV], x[3 % NV]);
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (v + i < a.V) o[i] = x[i];
    }
  } else {
    uint16_t* o = reinterpret_cast<uint16_t*>(a.out) + at;
    if (NV == 4 && a.wide && v + NV <= a.V) {
      *reinterpret_cast<uint2*>(o) = make_uint2(bf16_pair(x[0], x[1 % NV]), bf16_pair(x[2 % NV], x[3 % NV]));
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (v + i < a.V) o[i] = (uint16_t)bf16_bits(x[i]);
    }
  }
}

// --------------------------------------------------------------------------
// Up to 16 tokens
// --------------------------------------------------------------------------
constexpr int kFewWaves = 4;

template <int KIND, int P, int NV>
struct FewChunk {  // one block of 128 columns in registers
  uint4 w[NV];
  ScaleWord<KIND> s[NV];
  uint4 h[P][4];
};

template <int KIND, int P, int NV>
__global__ __launch_bounds__(256) void ss_head_few_kernel(HeadArgs a) {
  __shared__ float sums[kFewWaves][NV][4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
  const int v0 = blockIdx.x * (16 * NV);
  const int b0 = a.nb * wave / kFewWaves, b1 = a.nb * (wave + 1) / kFewWaves;
  const uint8_t* code[NV];
  const uint8_t* scale[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    // tile i takes rows n * NV + i: a lane's results are NV consecutive columns
    const int v = v0 + n * NV + i < a.V ? v0 + n * NV + i : a.V - 1;
    code[i] = a.codes + (int64_t)v * a.nb * kBlockBytes + g * 16;
    scale[i] = a.scales + (int64_t)v * a.nb * w4_scale_bytes(KIND);
  }
  // A rows beyond the last token repeat it; their results are not written
  const __bf16* h = a.h + (int64_t)(n < a.T ? n : a.T - 1) * a.ld_h + 8 * g;

  auto load = [&](FewChunk<KIND, P, NV>& c, int b) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      c.w[i] = *reinterpret_cast<const uint4*>(code[i] + (int64_t)b * kBlockBytes);
      c.s[i] = load_scales<KIND>(scale[i], b);
    }
    const int steps = (a.H - b * kBlockCols) / 32;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        c.h[p][j] = j < steps ? *reinterpret_cast<const uint4*>(h + p * a.part + b * kBlockCols + 32 * j) : make_uint4(0, 0, 0, 0);
  };
  f32x4 tot[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) tot[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto take = [&](const FewChunk<KIND, P, NV>& c, int b) {
    const int steps = (a.H - b * kBlockCols) / 32;  // of the row's last block: 1 to 4
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      f32x4 sum = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (j >= steps) break;
        const float s = step_scale<KIND>(c.s[i], j);
        const bf16x8 w = as_bf16x8(w4_expand<KIND>(dword(c.w[i], j), s));
#pragma unroll
        for (int p = 0; p < P; ++p) {
          if constexpr (KIND == kMx)
            tot[i] = mfma(as_bf16x8(c.h[p][j]), w, tot[i]);
          else
            sum = mfma(as_bf16x8(c.h[p][j]), w, sum);
        }
        if constexpr (KIND != kMx) {
          if ((j + 1) % (4 / w4_groups(KIND)) == 0) {  // the group ends
#pragma unroll
            for (int r = 0; r < 4; ++r) tot[i][r] = __builtin_fmaf(sum[r], s, tot[i][r]);
            sum = f32x4{0.f, 0.f, 0.f, 0.f};
          }
        }
      }
    }
  };
  if (b0 < b1) {
    FewChunk<KIND, P, NV> x, y;
    load(x, b0);
    for (int b = b0; b < b1; b += 2) {
      if (b + 1 < b1) load(y, b + 1);
      take(x, b);
      if (b + 2 < b1) load(x, b + 2);
      if (b + 1 < b1) take(y, b + 1);
    }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) sums[wave][i][r][lane] = tot[i][r];
  __syncthreads();
  // thread (token, column group): 16 x 16
  const int t = threadIdx.x >> 4, c = threadIdx.x & 15;
  if (t < a.T) {
    float x[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      x[i] = 0.0f;
#pragma unroll
      for (int w = 0; w < kFewWaves; ++w) x[i] += sums[w][i][t & 3][(t >> 2) * 16 + c];
    }
    store_cols<NV>(a, t, v0 + c * NV, x);
  }
}

// --------------------------------------------------------------------------
// More tokens
// --------------------------------------------------------------------------
constexpr int kManyWaves = 4;

template <int KIND, int P, int MT, int NV>
__global__ __launch_bounds__(256, 2) void ss_head_many_kernel(HeadArgs a) {
  constexpr int TOK = MT * 16;
  constexpr int SLOTS = P * TOK * 16;              // 16-byte pieces of a block's hidden states
  constexpr int PER = SLOTS / 256;                 // of a thread
  __shared__ uint4 hs[2][SLOTS];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
  // Workgroups go to the eight XCDs in turn; the token blocks of a vocabulary block
  // follow one another on the same XCD, whose L2 then holds its codes.
  const int slot = blockIdx.x >> 3;
  const int vb = (slot / a.tblocks) * 8 + (blockIdx.x & 7), tb = slot % a.tblocks;
  if (vb >= a.vblocks) return;
  const int v0 = (vb * kManyWaves + wave) * (16 * NV), t0 = tb * TOK;
  const uint8_t* code[NV];
  const uint8_t* scale[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = v0 + n * NV + i < a.V ? v0 + n * NV + i : a.V - 1;
    code[i] = a.codes + (int64_t)v * a.nb * kBlockBytes + g * 16;
    scale[i] = a.scales + (int64_t)v * a.nb * w4_scale_bytes(KIND);
  }
  // hidden states: piece q of part p, token t, at slot (q ^ t) & 15 of its row, so
  // that the 16 rows of an operand lie in different banks
  uint4 hr[PER];
  auto load_h = [&](int b) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int idx = threadIdx.x + i * 256;
      const int q = idx & 15, row = (idx >> 4) % TOK, p = (idx >> 4) / TOK;
      const int t = t0 + row < a.T ? t0 + row : a.T - 1;
      const int k = b * kBlockCols + q * 8;
      hr[i] = k < a.H
                  ? *reinterpret_cast<const uint4*>(a.h + p * a.part + (int64_t)t * a.ld_h + k)
                  : make_uint4(0, 0, 0, 0);
    }
  };
  auto put_h = [&](int buf) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int idx = threadIdx.x + i * 256;
      const int q = idx & 15, row = idx >> 4;
      hs[buf][row * 16 + ((q ^ row) & 15)] = hr[i];
    }
  };
  uint4 w[2][NV];
  ScaleWord<KIND> sc[2][NV];
  auto load_w = [&](int buf, int b) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      w[buf][i] = *reinterpret_cast<const uint4*>(code[i] + (int64_t)b * kBlockBytes);
      sc[buf][i] = load_scales<KIND>(scale[i], b);
    }
  };
  f32x4 tot[MT][NV];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int i = 0; i < NV; ++i) tot[m][i] = f32x4{0.f, 0.f, 0.f, 0.f};

  auto take = [&](int buf, int b) {
    const int steps = (a.H - b * kBlockCols) / 32;
    f32x4 sum[MT][NV];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j >= steps) break;
      bf16x8 A[P][MT];
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int m = 0; m < MT; ++m)
          A[p][m] = as_bf16x8(hs[buf][((p * MT + m) * 16 + n) * 16 + (((4 * j + g) ^ n) & 15)]);
      constexpr int per_group = KIND == kMx ? 1 : 4 / w4_groups(KIND);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const float s = step_scale<KIND>(sc[buf][i], j);
        const bf16x8 W = as_bf16x8(w4_expand<KIND>(dword(w[buf][i], j), s));
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          if constexpr (KIND == kMx) {
#pragma unroll
            for (int p = 0; p < P; ++p) tot[m][i] = mfma(A[p][m], W, tot[m][i]);
          } else {
            if (j % per_group == 0) sum[m][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 0; p < P; ++p) sum[m][i] = mfma(A[p][m], W, sum[m][i]);
            if ((j + 1) % per_group == 0) {
#pragma unroll
              for (int r = 0; r < 4; ++r) tot[m][i][r] = __builtin_fmaf(sum[m][i][r], s, tot[m][i][r]);
            }
          }
        }
      }
    }
  };
  // Waits for this wave's LDS accesses, then for the other waves; loads from
  // memory stay in flight over it.
  auto meet = [&]() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

  const int nb = a.nb;
  load_h(0);
  load_w(0, 0);
  put_h(0);
  if (nb > 1) load_h(1), load_w(1, 1);
  meet();
  for (int b = 0; b < nb; b += 2) {
    if (b + 1 < nb) put_h(1);
    if (b + 2 < nb) load_h(b + 2);
    take(0, b);
    if (b + 2 < nb) load_w(0, b + 2);
    meet();
    if (b + 1 < nb) {
      if (b + 2 < nb) put_h(0);
      if (b + 3 < nb) load_h(b + 3);
      take(1, b + 1);
      if (b + 3 < nb) load_w(1, b + 3);
      meet();
    }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int t = t0 + m * 16 + g * 4 + r;
      if (t < a.T) {
        float x[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i] = tot[m][i][r];
        store_cols<NV>(a, t, v0 + n * NV, x);
      }
    }
}

// --------------------------------------------------------------------------
// Host
// --------------------------------------------------------------------------
template <int KIND, int P>
static ss_status launch_head(HeadArgs& a, hipStream_t st) {
  if (a.T <= 16) {
    constexpr int NV = 4;
    const unsigned grid = (unsigned)((a.V + 16 * NV - 1) / (16 * NV));
    hipLaunchKernelGGL((ss_head_few_kernel<KIND, P, NV>), dim3(grid), dim3(256), 0, st, a);
    return SS_OK;
  }
  constexpr int NV = 4, most = P == 3 ? 2 : 4;
  const int tiles = (a.T + 15) / 16;
  a.tblocks = (tiles + most - 1) / most;
  const int mt = (tiles + a.tblocks - 1) / a.tblocks;
  a.vblocks = (a.V + 16 * NV * kManyWaves - 1) / (16 * NV * kManyWaves);
  const int64_t blocks = (int64_t)((a.vblocks + 7) / 8 * 8) * a.tblocks;
  if (blocks >= 1 << 24) return SS_ERR_UNSUPPORTED;  // 2^32 threads, over 2^36 logits
  const dim3 grid((unsigned)blocks);
  if (mt == 1)
    hipLaunchKernelGGL((ss_head_many_kernel<KIND, P, 1, NV>), grid, dim3(256), 0, st, a);
  else if (mt == 2)
    hipLaunchKernelGGL((ss_head_many_kernel<KIND, P, 2, NV>), grid, dim3(256), 0, st, a);
  if constexpr (P == 1) {
    if (mt == 3) hipLaunchKernelGGL((ss_head_many_kernel<KIND, P, 3, NV>), grid, dim3(256), 0, st, a);
    if (mt == 4) hipLaunchKernelGGL((ss_head_many_kernel<KIND, P, 4, NV>), grid, dim3(256), 0, st, a);
  }
  return SS_OK;
}

}  // namespace ss

using namespace ss;

extern "C" {

size_t ss_head_w4_bytes(int T, int H, int dtype) {
  if (T < 0 || T > SS_MAX_T || H < 1 || H > SS_MAX_H || (dtype != SS_F32 && dtype != SS_BF16)) return 0;
  const size_t n = (size_t)T * H * 2 * (dtype == SS_F32 ? 3 : 1);
  return n < 256 ? 256 : (n + 255) & ~(size_t)255;
}

ss_status ss_head_w4(const void* h, int dtype, int T, int64_t ld_h, const ss_w4* t, void* logits, int out_dtype,
                     int64_t ld, void* ws, size_t ws_bytes, void* stream) {
  if (!t || (dtype != SS_F32 && dtype != SS_BF16) || (out_dtype != SS_F32 && out_dtype != SS_BF16))
    return SS_ERR_INVALID_ARG;
  const int kind = w4_kind(t);
  if (kind < 0 || T < 0 || T > SS_MAX_T) return SS_ERR_INVALID_ARG;
  if (T == 0) return SS_OK;
  if (!h || !logits || !ws || !w4_aligned(t->codes) || !w4_aligned(t->scales) || ld_h < t->H || ld < t->V)
    return SS_ERR_INVALID_ARG;
  if (ws_bytes < ss_head_w4_bytes(T, t->H, dtype) || ((uintptr_t)ws & 15u)) return SS_ERR_WORKSPACE;
  const hipStream_t st = (hipStream_t)stream;
  HeadArgs a = {};
  a.codes = reinterpret_cast<const uint8_t*>(t->codes);
  a.scales = reinterpret_cast<const uint8_t*>(t->scales);
  a.out = logits;
  a.ld = ld;
  a.T = T;
  a.V = t->V;
  a.H = t->H;
  a.nb = w4_blocks(t->H);
  a.out_f32 = out_dtype == SS_F32;
  const int size = a.out_f32 ? 4 : 2;
  a.wide = ((uintptr_t)logits % (4 * size)) == 0 && ld % 4 == 0;
  const bool direct = dtype == SS_BF16 && ((uintptr_t)h & 15u) == 0 && ld_h % 8 == 0;
  if (direct) {
    a.h = reinterpret_cast<const __bf16*>(h);
    a.ld_h = ld_h;
  } else {
    const int64_t n = (int64_t)T * t->H;
    const int64_t blocks = (n + 255) / 256;
    const dim3 grid((unsigned)(blocks < 4096 ? blocks : 4096));
    if (dtype == SS_F32)
      hipLaunchKernelGGL(ss_head_parts_kernel<SS_F32>, grid, dim3(256), 0, st, h, ld_h, T, t->H, (uint16_t*)ws);
    else
      hipLaunchKernelGGL(ss_head_parts_kernel<SS_BF16>, grid, dim3(256), 0, st, h, ld_h, T, t->H, (uint16_t*)ws);
    a.h = reinterpret_cast<const __bf16*>(ws);
    a.ld_h = t->H;
    a.part = n;
  }
  ss_status done;
  if (dtype == SS_F32) {
    switch (kind) {
      case kInt128: done = launch_head<kInt128, 3>(a, st); break;
      case kInt64: done = launch_head<kInt64, 3>(a, st); break;
      case kInt32: done = launch_head<kInt32, 3>(a, st); break;
      default: done = launch_head<kMx, 3>(a, st); break;
    }
  } else {
    switch (kind) {
      case kInt128: done = launch_head<kInt128, 1>(a, st); break;
      case kInt64: done = launch_head<kInt64, 1>(a, st); break;
      case kInt32: done = launch_head<kInt32, 1>(a, st); break;
      default: done = launch_head<kMx, 1>(a, st); break;
    }
  }
  if (done != SS_OK) return done;
  return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_HIP;
}

}  // extern "C"
