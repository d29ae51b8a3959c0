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
// A workgroup shares the hidden states of a chunk of columns in LDS; each of
// its waves has its own vocabulary rows, whose codes go from memory to registers.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "ss_w4.hpp"

namespace ss {

struct HeadArgs {
  const void* h;          // hidden states, or their parts [P][T, ld_h]
  int64_t ld_h, part;     // elements from one row / part to the next
  const uint8_t* codes;
  const uint8_t* scales;
  void* out;
  int64_t ld;
  int T, V, H, nb;
  int out_f32;
  int wide;               // out rows can be written NV columns at a time
  int rows;               // tokens of a token block
  int tblocks, vblocks;   // token and vocabulary blocks
};

// --------------------------------------------------------------------------
// Hidden states as bfloat16 parts, or a copy whose rows start at multiples of 16 bytes
// --------------------------------------------------------------------------
// The parts of a float32, in the high halves: cut, not rounded, so that each takes the next eight bits
// and what is left is exact.
__device__ __forceinline__ void split3(uint32_t x, uint32_t part[3]) {
  const float r1 = __uint_as_float(x) - __uint_as_float(x & 0xFFFF0000u);
  const float r2 = r1 - __uint_as_float(__float_as_uint(r1) & 0xFFFF0000u);
  const bool fine = (x & 0x7F800000u) != 0x7F800000u;
  // a NaN whose high bits are those of an infinity stays a NaN
  part[0] = x | ((x & 0x7FFFFFFFu) > 0x7F800000u ? 0x400000u : 0u);
  part[1] = fine ? __float_as_uint(r1) : 0u;
  part[2] = fine ? __float_as_uint(r2) : 0u;
}

template <int DT>
__global__ __launch_bounds__(256) void ss_head_parts_kernel(const void* h, int64_t ld, int T, int H, uint16_t* out) {
  const int64_t n = (int64_t)T * H;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t t = i / H, k = i - t * H;
    if constexpr (DT == SS_F32) {
      uint32_t part[3];
      split3(reinterpret_cast<const uint32_t*>(h)[t * ld + k], part);
#pragma unroll
      for (int p = 0; p < 3; ++p) out[p * n + i] = (uint16_t)(part[p] >> 16);
    } else {
      out[i] = reinterpret_cast<const uint16_t*>(h)[t * ld + k];
    }
  }
}

// --------------------------------------------------------------------------
// Pieces
// --------------------------------------------------------------------------
__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// The scales of a row for CB blocks, as loaded.
template <int KIND, int CB>
struct Scales {
  static constexpr int kWords = CB * w4_scale_bytes(KIND) < 4 ? 1 : CB * w4_scale_bytes(KIND) / 4;
  uint32_t w[kWords];
};

// Loads them from `row` at block b; all CB blocks lie in the row.
template <int KIND, int CB>
__device__ __forceinline__ void load_scales(Scales<KIND, CB>& s, const uint8_t* row, int b) {
  constexpr int SB = w4_scale_bytes(KIND);
  const uint8_t* p = row + b * SB;
  __builtin_memcpy(s.w, __builtin_assume_aligned(p, SB < 4 ? 2 : 4), CB * SB);
}

// The scale of step j (32 columns) of block i.
template <int KIND, int CB>
__device__ __forceinline__ float step_scale(const Scales<KIND, CB>& s, int i, int j) {
  if constexpr (KIND == kMx) {
    return mx_bits(j == 3 ? s.w[i] >> 24 : s.w[i] >> (8 * j) & 255u);
  } else {
    const int k = i * w4_groups(KIND) + j / (4 / w4_groups(KIND));
    return k & 1 ? __uint_as_float(s.w[k / 2] & 0xFFFF0000u) : __uint_as_float(s.w[k / 2] << 16);
  }
}

__device__ __forceinline__ uint32_t dword(u32x4 v, int j) { return j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w; }

// Writes NV consecutive columns of one token.
template <int NV>
__device__ __forceinline__ void store_cols(const HeadArgs& a, int t, int v, const float x[NV]) {
  const int64_t at = (int64_t)t * a.ld + v;
  const bool whole = NV > 1 && a.wide && v + NV <= a.V;
  if (a.out_f32) {
    float* o = reinterpret_cast<float*>(a.out) + at;
    if (whole) {
      __builtin_memcpy(__builtin_assume_aligned(o, 4 * NV), x, 4 * NV);
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (v + i < a.V) o[i] = x[i];
    }
  } else {
    uint16_t* o = reinterpret_cast<uint16_t*>(a.out) + at;
    if (whole) {
      uint32_t y[(NV + 1) / 2];
#pragma unroll
      for (int i = 0; i < NV / 2; ++i) y[i] = bf16_pair(x[2 * i], x[2 * i + 1]);
      __builtin_memcpy(__builtin_assume_aligned(o, 2 * NV), y, 2 * NV);
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (v + i < a.V) o[i] = (uint16_t)bf16_bits(x[i]);
    }
  }
}

// --------------------------------------------------------------------------
// The product
// --------------------------------------------------------------------------
// SRC: where the hidden states come from, bfloat16 (P parts) or float32 split on the way (P = 3).
enum HeadSource { kFromBf16 = 0, kFromF32 = 1 };

// Threads have a workgroup of WAVES waves; each wave has NV tiles of 16 vocabulary rows and all MT tiles of
// 16 tokens, and takes CB blocks of columns (a chunk) at a time.
template <int KIND, int SRC, int P, int MT, int NV, int CB, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void ss_head_kernel(HeadArgs a) {
  constexpr int THREADS = WAVES * 64;
  constexpr int QS = CB * 16;                     // 16-byte pieces of a token's chunk
  constexpr int READ = SRC == kFromF32 ? 1 : P;   // parts that are read
  constexpr int LOADS = READ * MT * 16 * QS;
  constexpr int PER = (LOADS + THREADS - 1) / THREADS;
  extern __shared__ u32x4 hs[];                   // [2][P][rows][QS]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
  // Workgroups go to the eight XCDs in turn; the token blocks of a vocabulary block
  // follow one another on the same XCD, whose L2 then holds its codes.
  const int slot = blockIdx.x >> 3;
  const int vb = (slot / a.tblocks) * 8 + (blockIdx.x & 7), tb = slot % a.tblocks;
  if (vb >= a.vblocks) return;
  const int v0 = (vb * WAVES + wave) * (16 * NV), t0 = tb * MT * 16;
  const int rows = a.rows;                        // of hs: the tokens of a block, at most MT * 16
  const uint8_t* code[NV];
  const uint8_t* scale[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    // tile i takes rows n * NV + i: a lane's results are NV consecutive columns
    const int v = v0 + n * NV + i < a.V ? v0 + n * NV + i : a.V - 1;
    code[i] = a.codes + (int64_t)v * a.nb * kBlockBytes + g * 16;
    scale[i] = a.scales + (int64_t)v * a.nb * w4_scale_bytes(KIND);
  }

  const int nc = (a.nb + CB - 1) / CB;
  // Chunk c starts at block c * CB; the last one is moved back into the row, and skips the blocks that the
  // chunk before it had.  So every load is made, whole, in every turn of the loop: behind a condition,
  // the compiler would have to wait for all loads in flight where its branches meet.
    auto base = [&](int c) { return c * CB < a.nb - CB ? c * CB : a.nb - CB; };

  // Hidden states: piece q of row r lies at slot q ^ (r & 15), so that the 16 rows of an operand lie in
  // different banks.
  u32x4 hr[PER][SRC == kFromF32 ? 2 : 1];
  auto load_h = [&](int c) {
    const int k0 = base(c) * kBlockCols;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int idx = threadIdx.x + i * THREADS;
      const int row = idx / QS < READ * rows ? idx / QS : READ * rows - 1;
      const int r = READ == 1 ? row : row % rows, p = READ == 1 ? 0 : row / rows;
      const int t = t0 + r < a.T ? t0 + r : a.T - 1;
      // columns beyond H are read from within the row and not used
      const int k = k0 + idx % QS * 8 < a.H ? k0 + idx % QS * 8 : a.H - 8;
      if constexpr (SRC == kFromF32) {
        const u32x4* f = reinterpret_cast<const u32x4*>(reinterpret_cast<const float*>(a.h) + (int64_t)t * a.ld_h + k);
        hr[i][0] = f[0], hr[i][1] = f[1];
      } else {
        hr[i][0] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(a.h) + p * a.part +
                                                   (int64_t)t * a.ld_h + k);
      }
    }
  };
  auto put_h = [&](int buf) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int idx = threadIdx.x + i * THREADS;
      // (beyond the last row: the same piece of the last row again)
      const int q = idx % QS, row = idx / QS < READ * rows ? idx / QS : READ * rows - 1;
      if constexpr (SRC == kFromF32) {
        u32x4* to = hs + (buf * P * rows + row) * QS + (q ^ (row & 15));
        const uint32_t x[8] = {hr[i][0].x, hr[i][0].y, hr[i][0].z, hr[i][0].w,
                               hr[i][1].x, hr[i][1].y, hr[i][1].z, hr[i][1].w};
        uint32_t y[3][4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t lo[3], hi[3];
          split3(x[2 * k], lo);
          split3(x[2 * k + 1], hi);
#pragma unroll
          for (int p = 0; p < 3; ++p) y[p][k] = lo[p] >> 16 | (hi[p] & 0xFFFF0000u);
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) to[p * rows * QS] = u32x4{y[p][0], y[p][1], y[p][2], y[p][3]};
      } else {
        const int r = READ == 1 ? row : row % rows;
        hs[(buf * P * rows + row) * QS + (q ^ (r & 15))] = hr[i][0];
      }
    }
  };
  u32x4 w[2][CB][NV];
  Scales<KIND, CB> sc[2][NV];
  auto load_w = [&](int buf, int c) {
    const int b0 = base(c);
#pragma unroll
    for (int i = 0; i < NV; ++i) load_scales<KIND, CB>(sc[buf][i], scale[i], b0);
#pragma unroll
    for (int b = 0; b < CB; ++b)
#pragma unroll
      for (int i = 0; i < NV; ++i)
        w[buf][b][i] = *reinterpret_cast<const u32x4*>(code[i] + (b0 + b) * kBlockBytes);
  };
  f32x4 tot[MT][NV];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int i = 0; i < NV; ++i) tot[m][i] = f32x4{0.f, 0.f, 0.f, 0.f};

  // Lane (n, g) reads row n of a tile; rows beyond the last token repeat it, their results are not written.
  const int last = rows - 1;
  // `whole`: all steps of the chunk's blocks are the row's and are taken, as in every chunk but the last one
  auto take = [&](auto whole, int buf, int c) {
    const u32x4* hb = hs + buf * P * rows * QS;
    const int left = (a.H - base(c) * kBlockCols) / 32;  // steps to the row's end
    const int first = c * CB - base(c);  // of the last chunk
#pragma unroll
    for (int b = 0; b < CB; ++b) {
      if (!whole && b < first) continue;
      f32x4 sum[MT][NV];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (!whole && 4 * b + j >= left) break;
        bf16x8 A[P][MT];
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const int r = MT == 1 ? (n < last ? n : last) : m * 16 + n;
            A[p][m] = as_bf16x8(hb[(p * rows + r) * QS + ((16 * b + 4 * j + g) ^ (r & 15))]);
          }
        constexpr int per_group = KIND == kMx ? 1 : 4 / w4_groups(KIND);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const float s = step_scale<KIND, CB>(sc[buf][i], b, j);
          const bf16x8 W = as_bf16x8(w4_expand<KIND>(dword(w[buf][b][i], j), s));
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
    }
  };
  // Waits for this wave's LDS accesses, then for the other waves; loads from
  // memory stay in flight over it.
  auto meet = [&]() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

  const std::true_type yes{};
  const std::false_type no{};
  load_h(0);
  load_w(0, 0);
  put_h(0);
  load_h(1);
  load_w(1, 1);
  meet();
  int c = 0;
  for (; c + 3 < nc; c += 2) {
    put_h(1);
    load_h(c + 2);
    take(yes, 0, c);
    load_w(0, c + 2);
    meet();
    put_h(0);
    load_h(c + 3);
    take(yes, 1, c + 1);
    load_w(1, c + 3);
    meet();
  }
  // one to three chunks are left
  const int rest = nc - c;
  put_h(1);
  if (rest == 3) {
    load_h(c + 2);
    take(yes, 0, c);
    load_w(0, c + 2);
    meet();
    put_h(0);
    take(yes, 1, c + 1);
    meet();
    take(no, 0, c + 2);
  } else if (rest == 2) {
    take(yes, 0, c);
    meet();
    take(no, 1, c + 1);
  } else {
    take(no, 0, c);
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
template <int KIND, int SRC, int P, int MT, int NV, int CB, int WAVES>
static ss_status launch_one(HeadArgs& a, hipStream_t st) {
  a.tblocks = (a.T + MT * 16 - 1) / (MT * 16);
  a.vblocks = (a.V + 16 * NV * WAVES - 1) / (16 * NV * WAVES);
  a.rows = MT == 1 && a.T < 16 ? a.T : MT * 16;
  const int size = a.out_f32 ? 4 : 2;
  a.wide = (uintptr_t)a.out % (NV * size) == 0 && a.ld % NV == 0;
  const int64_t blocks = (int64_t)((a.vblocks + 7) / 8 * 8) * a.tblocks;
  if (blocks >= (1 << 26) / WAVES) return SS_ERR_UNSUPPORTED;  // 2^32 threads
  const size_t lds = (size_t)2 * P * a.rows * CB * 256;
  auto kernel = ss_head_kernel<KIND, SRC, P, MT, NV, CB, WAVES>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(WAVES * 64), lds, st, a);
  return SS_OK;
}

// CB blocks at a time where the row has as many
template <int KIND, int SRC, int P, int MT, int NV, int CB, int WAVES>
static ss_status launch_chunks(HeadArgs& a, hipStream_t st) {
  if (a.nb < CB) return launch_one<KIND, SRC, P, MT, NV, 1, WAVES>(a, st);
  return launch_one<KIND, SRC, P, MT, NV, CB, WAVES>(a, st);
}

template <int KIND>
static ss_status launch_head_f32(HeadArgs& a, bool direct, hipStream_t st) {
  if (direct) return launch_chunks<KIND, kFromF32, 3, 1, 1, 2, 8>(a, st);
  if (a.T <= 16) return launch_chunks<KIND, kFromBf16, 3, 1, 1, 2, 8>(a, st);
  return launch_one<KIND, kFromBf16, 3, 2, 2, 1, 8>(a, st);
}

template <int KIND>
static ss_status launch_head_bf16(HeadArgs& a, hipStream_t st) {
  const int tiles = (a.T + 15) / 16;
  if (tiles == 1) return launch_chunks<KIND, kFromBf16, 1, 1, 1, 4, 8>(a, st);
  const int blocks = (tiles + 3) / 4, mt = (tiles + blocks - 1) / blocks;
  if (mt == 2) return launch_chunks<KIND, kFromBf16, 1, 2, 2, 2, 8>(a, st);
  if (mt == 3) return launch_chunks<KIND, kFromBf16, 1, 3, 1, 2, 8>(a, st);
  return launch_chunks<KIND, kFromBf16, 1, 4, 2, 2, 8>(a, st);
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
  // few float32 rows are split by the product's own loads, more of them once, before it
  const bool direct = wide_rows(h, ld_h, dtype) && (dtype == SS_BF16 || T <= 16);
  if (direct) {
    a.h = h;
    a.ld_h = ld_h;
  } else {
    const int64_t n = (int64_t)T * t->H;
    const int64_t blocks = (n + 255) / 256;
    const dim3 grid((unsigned)(blocks < 4096 ? blocks : 4096));
    if (dtype == SS_F32)
      hipLaunchKernelGGL(ss_head_parts_kernel<SS_F32>, grid, dim3(256), 0, st, h, ld_h, T, t->H, (uint16_t*)ws);
    else
      hipLaunchKernelGGL(ss_head_parts_kernel<SS_BF16>, grid, dim3(256), 0, st, h, ld_h, T, t->H, (uint16_t*)ws);
    a.h = ws;
    a.ld_h = t->H;
    a.part = n;
  }
  ss_status done;
  if (dtype == SS_F32) {
    switch (kind) {
      case kInt128: done = launch_head_f32<kInt128>(a, direct, st); break;
      case kInt64: done = launch_head_f32<kInt64>(a, direct, st); break;
      case kInt32: done = launch_head_f32<kInt32>(a, direct, st); break;
      default: done = launch_head_f32<kMx>(a, direct, st); break;
    }
  } else {
    switch (kind) {
      case kInt128: done = launch_head_bf16<kInt128>(a, st); break;
      case kInt64: done = launch_head_bf16<kInt64>(a, st); break;
      case kInt32: done = launch_head_bf16<kInt32>(a, st); break;
      default: done = launch_head_bf16<kMx>(a, st); break;
    }
  }
  if (done != SS_OK) return done;
  return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_HIP;
}

}  // extern "C"
