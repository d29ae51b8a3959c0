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

#include <atomic>
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
  int rows;               // hidden rows (few), tokens of a token block (more)
  int parts;              // few: 3 where a token has four rows, its parts and one not used; else 1
  int pitch, slab_cols;   // few: 16-byte pieces of a row in LDS; columns of a slab
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

// Waits for this wave's LDS accesses, then for the other waves; loads from
// memory stay in flight over it.
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The scale of step j (32 columns) of a block whose scales are s0 and s1.
template <int KIND>
__device__ __forceinline__ float scale_of(uint32_t s0, uint32_t s1, int j) {
  if constexpr (KIND == kMx) return mx_bits(j == 3 ? s0 >> 24 : s0 >> (8 * j) & 255u);
  const int k = j / (4 / w4_groups(KIND));
  const uint32_t x = k < 2 ? s0 : s1;
  return __uint_as_float(k & 1 ? x & 0xFFFF0000u : x << 16);
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
// Up to 16 hidden rows
// --------------------------------------------------------------------------
// Bound by the table's read: V = 262144, H = 8192, T = 16 mx 217 us, 5.3 TB/s; V = 32768, H = 4096, four float32 rows 17.5 us, 4.1
// TB/s.  A workgroup of 16 waves to a CU keeps the hidden rows in LDS (all columns, or 128 KB of them
// at a time) and has an equal share of the table's tiles of 16 rows; its waves run along the rows without
// waiting for each other, eight 16-byte loads a lane in flight, the next block's asked for as soon as its register is
// free, over the ends of rows.  Where all columns fit (MULTI false), the waves share the workgroup's blocks evenly, by units of
// eight: a tile that ends up with several waves is summed through LDS, in the order of its columns.
constexpr int kFewWaves = 16, kUnit = 8;
constexpr int kSlabBytes = 128 * 1024;
constexpr int kFewTiles = 2;  // MULTI: tiles of a wave whose sums stay in registers from slab to slab

// 64 bytes a row of a tile's scales, 16 in each of a row's four lanes.
__device__ __forceinline__ u32x4 load_super(const HeadArgs& a, int tile, int n, int g, int b, int sbytes, int64_t total) {
  const int scale_row = a.nb * sbytes;
  const int v = tile * 16 + n < a.V ? tile * 16 + n : a.V - 1;
  const int64_t at = (int64_t)v * scale_row + b * sbytes + g * 16;
  u32x4 s;
  if ((int64_t)(tile * 16 + 15) * scale_row + b * sbytes + 64 <= total) {
    __builtin_memcpy(&s, __builtin_assume_aligned(a.scales + at, 2), 16);
  } else {  // at the end of the array: what lies in it
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t lo = 0u, hi = 0u;
      if (at + 4 * i + 2 <= total) lo = *reinterpret_cast<const uint16_t*>(a.scales + at + 4 * i);
      if (at + 4 * i + 4 <= total) hi = *reinterpret_cast<const uint16_t*>(a.scales + at + 4 * i + 2);
      s[i] = lo | hi << 16;
    }
  }
  return s;
}

template <int KIND, int DT, bool MULTI>
__global__ __launch_bounds__(kFewWaves * 64) void ss_head_few_kernel(HeadArgs a) {
  constexpr int SB = w4_scale_bytes(KIND), PER_SUPER = 64 / SB / kUnit;  // units that 64 bytes of scales cover
  __shared__ u32x4 slab[kSlabBytes / 16];
  __shared__ float part[MULTI ? 1 : kFewWaves][2][4][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const int tiles = (a.V + 15) / 16;
  const int first = (int)((int64_t)tiles * blockIdx.x / gridDim.x), last = (int)((int64_t)tiles * (blockIdx.x + 1) / gridDim.x);
  const int code_row = a.nb * kBlockBytes;
  const int64_t scale_total = (int64_t)a.V * a.nb * SB;
  const int r = n < a.rows ? n : a.rows - 1;  // rows beyond the last repeat it; their results are not written

  // Hidden columns [k0, k0 + cols) to LDS: piece q of row r at q ^ (r & 15), so that 16 rows lie in different banks.
  auto fill = [&](int k0, int cols) {
    const int pieces = cols / 8;
    for (int i = threadIdx.x; i < a.T * pieces; i += kFewWaves * 64) {
      const int t = i / pieces, q = i - t * pieces;
      const int64_t at = (int64_t)t * a.ld_h + k0 + q * 8;
      if constexpr (DT == SS_F32) {
        uint32_t f[8];
        __builtin_memcpy(f, __builtin_assume_aligned(reinterpret_cast<const float*>(a.h) + at, 4), 32);
        u32x4 y[3];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t lo[3], hi[3];
          split3(f[2 * k], lo);
          split3(f[2 * k + 1], hi);
#pragma unroll
          for (int p = 0; p < 3; ++p) y[p][k] = lo[p] >> 16 | (hi[p] & 0xFFFF0000u);
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) slab[(4 * t + p) * a.pitch + (q ^ ((4 * t + p) & 15))] = y[p];
      } else {
        u32x4 x;
        __builtin_memcpy(&x, __builtin_assume_aligned(reinterpret_cast<const uint16_t*>(a.h) + at, 2), 16);
        slab[t * a.pitch + (q ^ (t & 15))] = x;
      }
    }
  };

  // The codes of unit c of a tile, block by block; blocks beyond the row's last are that one again.
  struct Cursor {
    const uint8_t* row;
    int b;
  };
  auto cursor = [&](int tile, int c, int pb0) {
    const int v = tile * 16 + n < a.V ? tile * 16 + n : a.V - 1;
    return Cursor{a.codes + (int64_t)v * code_row + g * 16, pb0 + c * kUnit};
  };
  auto load = [&](const Cursor& at, int s) {
    const int b = at.b + s < a.nb ? at.b + s : a.nb - 1;
    return *reinterpret_cast<const u32x4*>(at.row + b * kBlockBytes);
  };
  u32x4 w[kUnit], sc, sc_next;

  // Units [c0, c1) of a tile, from block pb0 of the row on (the slab's first); then comes unit c2 of tile t2, nothing if t2 < 0.
  auto run = [&](int tile, int c0, int c1, int t2, int c2, int pb0, f32x4& tot) {
    for (int c = c0; c < c1; ++c) {
      const bool more = c + 1 < c1;
      const Cursor next = cursor(more || t2 < 0 ? tile : t2, more ? c + 1 : c2, pb0);
      if ((c - c0) % PER_SUPER == 0) {
        sc = sc_next;
        const bool here = c + PER_SUPER < c1;
        if (here || t2 >= 0)
          sc_next = load_super(a, here ? tile : t2, n, g, pb0 + (here ? c + PER_SUPER : c2) * kUnit, SB, scale_total);
      }
      const int piece0 = (c - c0) % PER_SUPER * (kUnit * SB / 16);
      auto unit = [&](auto whole, auto load_next) {
        const int left = (a.H - (pb0 + c * kUnit) * kBlockCols) / 32;  // steps to the row's end
        uint32_t pair = 0u;
#pragma unroll
        for (int s = 0; s < kUnit; ++s) {
          if (whole || 4 * s < left) {
            // this block's scales, from the lane that has them
            const int from = ((piece0 + s * SB / 16) * 16 + n) * 4;
            uint32_t s0, s1 = 0u;
            if constexpr (KIND == kInt128) {
              if (s % 2 == 0) pair = __builtin_amdgcn_ds_bpermute(from, sc[s / 2]);
              s0 = s % 2 ? pair >> 16 : pair;
            } else if constexpr (KIND == kInt32) {
              s0 = __builtin_amdgcn_ds_bpermute(from, sc[s % 2 * 2]);
              s1 = __builtin_amdgcn_ds_bpermute(from, sc[s % 2 * 2 + 1]);
            } else {
              s0 = __builtin_amdgcn_ds_bpermute(from, sc[s % 4]);
            }
            constexpr int per_group = KIND == kMx ? 1 : 4 / w4_groups(KIND);
            f32x4 sum = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if (whole || 4 * s + j < left) {
                const bf16x8 A = as_bf16x8(slab[r * a.pitch + (((c * kUnit + s) * 16 + 4 * j + g) ^ (r & 15))]);
                const float f = scale_of<KIND>(s0, s1, j);
                const bf16x8 W = as_bf16x8(w4_expand<KIND>(dword(w[s], j), f));
                if constexpr (KIND == kMx) {
                  tot = mfma(A, W, tot);
                } else {
                  sum = mfma(A, W, sum);
                  if ((j + 1) % per_group == 0) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) tot[k] = __builtin_fmaf(sum[k], f, tot[k]);
                    sum = f32x4{0.f, 0.f, 0.f, 0.f};
                  }
                }
              }
            }
          }
          if constexpr (decltype(load_next)::value) w[s] = load(next, s);
        }
      };
      const std::true_type yes{};
      const std::false_type no{};
      const bool whole = (pb0 + (c + 1) * kUnit) * kBlockCols <= a.H;
      if (more || t2 >= 0)
        whole ? unit(yes, yes) : unit(no, yes);
      else
        whole ? unit(yes, no) : unit(no, no);
    }
  };
  auto prime = [&](int tile, int c, int pb0) {
    const Cursor at = cursor(tile, c, pb0);
#pragma unroll
    for (int s = 0; s < kUnit; ++s) w[s] = load(at, s);
    sc_next = load_super(a, tile, n, g, pb0 + c * kUnit, SB, scale_total);
  };
  // Lane (n, g) of a tile has four rows of hidden states at vocabulary row n.
  auto store = [&](int tile, const f32x4& tot) {
    const int v = tile * 16 + n;
    if (a.parts == 3) {  // rows 4 t .. 4 t + 2 are token t's parts
      const float x[1] = {tot[0] + (tot[1] + tot[2])};
      if (g < a.T) store_cols<1>(a, g, v, x);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float x[1] = {tot[k]};
        if (g * 4 + k < a.T) store_cols<1>(a, g * 4 + k, v, x);
      }
    }
  };

  if constexpr (!MULTI) {
    const int units = (a.nb + kUnit - 1) / kUnit;  // of a tile
    const int all = (last - first) * units;
    const int u0 = all * wave / kFewWaves, u1 = all * (wave + 1) / kFewWaves;
    if (u0 < u1) prime(first + u0 / units, u0 % units, 0);
    fill(0, a.H);
    meet();
    for (int u = u0; u < u1;) {
      const int tile = u / units, c0 = u - tile * units, end = (tile + 1) * units < u1 ? (tile + 1) * units : u1;
      f32x4 tot = f32x4{0.f, 0.f, 0.f, 0.f};
      run(first + tile, c0, c0 + end - u, end < u1 ? first + tile + 1 : -1, 0, 0, tot);
      if (end - u == units) {
        store(first + tile, tot);
      } else {  // slot 0: a tile that an earlier wave began; slot 1: one that this wave began
#pragma unroll
        for (int k = 0; k < 4; ++k) part[wave][c0 == 0][k][lane] = tot[k];
      }
      u = end;
    }
    meet();
    // the wave that began a tile and did not end it adds what the next waves have of it
    const int tile = (u1 - 1) / units;
    if (u0 < u1 && u1 % units && tile * units >= u0) {
      f32x4 tot;
#pragma unroll
      for (int k = 0; k < 4; ++k) tot[k] = part[wave][1][k][lane];
      for (int o = wave + 1; o < kFewWaves; ++o) {
        const int o0 = all * o / kFewWaves, o1 = all * (o + 1) / kFewWaves;
        if (o0 >= (tile + 1) * units) break;
        if (o0 == o1) continue;
#pragma unroll
        for (int k = 0; k < 4; ++k) tot[k] += part[o][0][k][lane];
      }
      store(first + tile, tot);
    }
  } else {
    for (int t0 = first; t0 < last; t0 += kFewWaves * kFewTiles) {
      f32x4 tot[kFewTiles];
#pragma unroll
      for (int i = 0; i < kFewTiles; ++i) tot[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      const int mine = t0 + wave;
      for (int k0 = 0; k0 < a.H; k0 += a.slab_cols) {
        const int cols = a.H - k0 < a.slab_cols ? a.H - k0 : a.slab_cols, units = (cols + kUnit * kBlockCols - 1) / (kUnit * kBlockCols);
        const int pb0 = k0 / kBlockCols;
        if (mine < last) prime(mine, 0, pb0);
        meet();  // all have left the slab before
        fill(k0, cols);
        meet();
#pragma unroll
        for (int i = 0; i < kFewTiles; ++i) {
          const int tile = mine + i * kFewWaves;
          if (tile < last) {
            const bool more = i + 1 < kFewTiles && tile + kFewWaves < last;
            run(tile, 0, units, more ? tile + kFewWaves : -1, 0, pb0, tot[i]);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < kFewTiles; ++i)
        if (mine + i * kFewWaves < last) store(mine + i * kFewWaves, tot[i]);
    }
  }
}

// --------------------------------------------------------------------------
// More hidden rows
// --------------------------------------------------------------------------
constexpr int kAcross = 64;  // token blocks of a vocabulary block in one row of the grid

// SRC: where the hidden states come from, bfloat16 (P parts) or float32 split on the way (P = 3).
enum HeadSource { kFromBf16 = 0, kFromF32 = 1 };

// A workgroup has WAVES waves; each wave has NV tiles of 16 vocabulary rows and all MT tiles of 16 tokens, and takes CB blocks
// of columns (a chunk) at a time, codes of the next chunk in flight.  Up to 16 tokens it is bound by the table's read and the
// start of its workgroups (V = 32768, H = 2048, T = 1: 8.7 us, 4.0 TB/s).  Beyond, a step of 32 columns takes, for each tile of vocabulary
// rows, 7 vector instructions to expand the codes (4 for E2M1), 4 MT / (group / 32) to scale sums (none for E2M1) and a few for
// addresses, MT matrix instructions of 16 cycles, and MT / NV reads of 1 KB from LDS.  Shares of the kernel's cycles:
//   T = 64 int128, V = 131072, H = 4096 (NV = 1)  88 to 92 us, 780 to 750 TFLOP/s: vector issue 48 %, LDS 46 %, matrix units 41 %;
//     waves wait for issue 41 % of their time and for loads and barriers 41 %.
//   T = 320 mx, the same table (NV = 4)  342 us, 1000 TFLOP/s: matrix units 41 %, vector issue 29 %, LDS 13 %.  (A library's product of
//     bfloat16 matrices of these sizes: 353 us.)  int128 376 to 400, int32 457 to 473 with NV = 1.
//   T = 37 int32, V = 200003, H = 2880  117 us: vector issue 48 %, LDS 27 %, matrix units 21 %.  A sum of 32 columns is scaled as soon as
//     its products are there: the compiler puts 274 cycles of s_nop between the 388 instructions of two chunks (9 with 16 waves
//     and MT = 4, where it has other products to put there; 364 with 12).
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
  const int slot = blockIdx.x >> 3, across = a.tblocks < kAcross ? a.tblocks : kAcross;
  const int vb = (slot / across) * 8 + (blockIdx.x & 7), tb = blockIdx.y * kAcross + slot % across;
  if (vb >= a.vblocks || tb >= a.tblocks) return;
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
static void launch_one(HeadArgs& a, hipStream_t st) {
  a.tblocks = (a.T + MT * 16 - 1) / (MT * 16);
  a.vblocks = (a.V + 16 * NV * WAVES - 1) / (16 * NV * WAVES);
  a.rows = MT == 1 && a.T < 16 ? a.T : MT * 16;
  const int size = a.out_f32 ? 4 : 2;
  a.wide = (uintptr_t)a.out % (NV * size) == 0 && a.ld % NV == 0;
  const int across = a.tblocks < kAcross ? a.tblocks : kAcross;
  const dim3 grid((unsigned)((a.vblocks + 7) / 8 * 8 * across), (unsigned)((a.tblocks + kAcross - 1) / kAcross));
  const size_t lds = (size_t)2 * P * a.rows * CB * 256;
  auto kernel = ss_head_kernel<KIND, SRC, P, MT, NV, CB, WAVES>;
  hipLaunchKernelGGL(kernel, grid, dim3(WAVES * 64), lds, st, a);
}

// Compute units of the current device.
static int compute_units() {
  static std::atomic<int> known[64];
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess) return 0;
  if (dev >= 0 && dev < 64 && (n = known[dev].load(std::memory_order_relaxed)) > 0) return n;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) return 0;
  if (dev >= 0 && dev < 64) known[dev].store(n, std::memory_order_relaxed);
  return n;
}

// Whether ss_head_few_kernel takes a call of up to 16 bfloat16 or 4 float32 rows.  It has more to start with (hidden rows to LDS) and to
// end with (the last units of all waves at once, sums of split tiles) than the other kernel, and a higher rate.  Times: us, this
// kernel / the other, int128, tables that no cache holds.
//   Size: two units at least for each of its waves, a row's last, partial unit counted as one, as it is loaded.  T = 1: V = 32768, H = 2048
//     (half of that) 13.0 / 10.8, V = 49152 16.9 / 17.5, V = 65536 18.0 / 18.5, V = 131072, H = 1024 18.0 / 22.0.
// Against four float32 rows, three products each, the other kernel has nothing beyond that: 0.6 to 0.95 of its time, and the same
// for rows of one or two blocks.  Against bfloat16 rows it has two things:
//   Rows of fewer than four blocks: a unit is loaded whole.  T = 16: V = 131077, H = 128 12.0 / 7.0; V = 400000, H = 256 35 / 23, H = 384
//     31 / 26, H = 512 41 / 49.  (Half-empty second units, H = 1536: 1.00 to 1.12 of the other's time.)
//   At most one of its workgroups to a compute unit (8 tiles): one round, without a rest.  T = 16: V = 32768, H = 4096 21.3 / 17.4, V = 36869
//     25.4 / 29.4; where the rows do not fit LDS, a wave takes whole tiles and half of the waves have none: H = 8192, V = 16384 29 / 25, V =
//     32000 42 / 36, V = 50000 60 / 61; H = 65536, V = 16384 230 / 167.  Long rows that do fit are shared out evenly: H = 8192, V = 16384, T = 8 21.6 / 24.1;
//     H = 6144, V = 22533, T = 1 21.1 / 22.4, T = 8 23.8 / 23.2.  So is the time of one row: H = 4096, V = 32768 17.6 / 16.9, and 17.7 /
//     19.9 at an odd address, whence the other kernel has it copied first (T = 16: 23.7 / 21.1).
static bool few_pays(const HeadArgs& a, bool f32, int cus) {
  const int64_t tiles = (a.V + 15) / 16, units = (a.nb + kUnit - 1) / kUnit;
  if (tiles * units < (int64_t)2 * kFewWaves * cus) return false;
  if (f32) return true;
  if (a.nb < 4) return false;
  return tiles > (int64_t)8 * cus || ((a.nb >= 48 || a.T == 1) && units * kUnit * kBlockCols * a.T <= kSlabBytes / 2);
}

template <int KIND, int DT>
static void launch_few(HeadArgs& a, int cus, hipStream_t st) {
  a.parts = DT == SS_F32 ? 3 : 1;
  a.rows = DT == SS_F32 ? 4 * a.T : a.T;
  // whole units: the slab's rows end with one
  const int unit = kUnit * kBlockCols, cols = (a.nb + kUnit - 1) / kUnit * unit, fit = kSlabBytes / 2 / a.rows;
  a.slab_cols = cols <= fit ? cols : fit / unit * unit;
  a.pitch = a.slab_cols / 8;
  const int tiles = (a.V + 15) / 16;
  const dim3 grid((unsigned)(tiles < cus ? tiles : cus)), block(kFewWaves * 64);
  if (cols <= fit)
    hipLaunchKernelGGL((ss_head_few_kernel<KIND, DT, false>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((ss_head_few_kernel<KIND, DT, true>), grid, block, 0, st, a);
}

// Whether up to 16 float32 rows are split by every workgroup for itself, not by a launch of 4 us before the product.  T = 8, us, split on
// the way / before (that launch apart): V = 32768, H = 2048 int128 15 / 13, int32 16 / 14, mx 15 / 12; V = 65536, H = 4096 49 / 38, 61 / 41,
// 43 / 43; V = 212992, H = 4352 157 / 131, 203 / 145, 151 / 141.
static bool small_for_split(const HeadArgs& a, int kind, int cus) {
  return (int64_t)((a.V + 15) / 16) * a.nb < (int64_t)(kind == kMx ? 1024 : 256) * cus;
}

// direct: the hidden rows as the caller has them, else their parts or their copy.  V = 32768, H = 2048, T = 32: tiles (NV, CB, WAVES)
// (2, 1, 8) 30 us, (1, 2, 8) 20; V = 131072, H = 4096: 112 and 144.
template <int KIND>
static void launch_head_f32(HeadArgs& a, bool direct, int cus, hipStream_t st) {
  if (a.T <= 4 && few_pays(a, true, cus)) return launch_few<KIND, SS_F32>(a, cus, st);
  const bool columns = a.nb >= 2, small = (int64_t)((a.V + 15) / 16) * ((a.T + 31) / 32) <= (int64_t)8 * cus;
  if (direct && columns) return launch_one<KIND, kFromF32, 3, 1, 1, 2, 8>(a, st);
  if (direct) return launch_one<KIND, kFromF32, 3, 1, 1, 1, 8>(a, st);
  if (a.T <= 16 && columns) return launch_one<KIND, kFromBf16, 3, 1, 1, 2, 8>(a, st);
  if (a.T <= 16) return launch_one<KIND, kFromBf16, 3, 1, 1, 1, 8>(a, st);
  if (small && columns) return launch_one<KIND, kFromBf16, 3, 2, 1, 2, 8>(a, st);
  return launch_one<KIND, kFromBf16, 3, 2, 2, 1, 8>(a, st);
}

// Large tables: 16, 14 or 12 waves a workgroup, one of which a compute unit holds, by the time that the chip's rounds of
// them take, which goes with the waves and 8 more (starting, and the hidden rows' share).  Measured, us, T = 29 / 64, int128:
//   V = 131072, H = 4096 (32 tiles a compute unit)  16 waves 67 / 88, 14 waves 89, 12 waves 75
//   V = 98304, H = 4096 (24)                        59 / 76, 58 / 74, 53 / 69
//   V = 161103, H = 4736 (39.3)                     112 / 136 (mx 153), 107 / 139 (mx 133), 118 / 159 (mx 144)
// E2M1 has no sums of groups beside the row's, so that four tiles of vocabulary rows a wave fit the registers but for 332 bytes a lane that
// are put aside before and after the loop (none in it): T = 64, V = 131072 89 against 91 of 16 waves, V = 161103 226 against 133 of 14; T =
// 320, V = 131072 347 against 381.  Integers of groups of 128 and 64 spill in the loop, those of 32 put more aside: T = 320 1095, 960 and 541
// against 400, 429 and 473 of 16 waves.
template <int KIND, int MT>
static void launch_rounds(HeadArgs& a, int64_t work, int cus, hipStream_t st) {
  auto cost = [&](int tiles, int each) { return (work + (int64_t)tiles * cus - 1) / ((int64_t)tiles * cus) * each; };
  const int64_t c16 = cost(16, 24), c14 = cost(14, 22), c12 = cost(12, 20), least = c12 < c14 ? c12 : c14;
  if constexpr (KIND == kMx && MT == 4) {
    if (cost(32, 48) <= (least < c16 ? least : c16)) return launch_one<KIND, kFromBf16, 1, MT, 4, 2, 8>(a, st);
  }
  if (c16 <= least) return launch_one<KIND, kFromBf16, 1, MT, 1, 2, 16>(a, st);
  if (c14 <= c12) return launch_one<KIND, kFromBf16, 1, MT, 1, 2, 14>(a, st);
  return launch_one<KIND, kFromBf16, 1, MT, 1, 2, 12>(a, st);
}

// 33 to 48 tokens: two workgroups of 8 waves a compute unit, which leave less behind in the last round (T = 37, V = 200003: int128 98,
// mx 102; 16 waves 103, 111; V = 131072: 81, 80).  E2M1 takes two tiles of vocabulary rows a wave where that fills its
// rounds of 16 tiles to a tenth: V = 131072 79 against 88; V = 98304, one round and a half, 70 against 68.
template <int KIND>
static void launch_48(HeadArgs& a, int64_t work, int cus, hipStream_t st) {
  if constexpr (KIND == kMx) {
    const int64_t round = (int64_t)16 * cus;
    if (10 * ((work + round - 1) / round * round) <= 11 * work) return launch_one<KIND, kFromBf16, 1, 3, 2, 2, 8>(a, st);
  }
  return launch_one<KIND, kFromBf16, 1, 3, 1, 2, 8>(a, st);
}

// Tiles of 16 tokens and waves a workgroup.  The more of them, the fewer times hidden rows and codes are read; but a table that
// gives less than a workgroup to each compute unit is cut finer.  Measured, us, by (CB, WAVES):
//   V = 16384, H = 2048   T = 16: (4, 8) 8.4, (4, 4) 7.3.
//   V = 32768, H = 2048   T = 16: (4, 8) 9.6, (4, 4) 10.4.  T = 32: (4, 8) 11.4, (2, 16) 17.  T = 64: (2, 8) 15, (2, 16) 19.5.
//   V = 65536, H = 4096   T = 32: (4, 8) 37, (2, 16) 33.  T = 64: (2, 8) 55, (2, 16) 40.
template <int KIND>
static void launch_head_bf16(HeadArgs& a, int cus, hipStream_t st) {
  if (a.T <= 16 && few_pays(a, false, cus)) return launch_few<KIND, SS_BF16>(a, cus, st);
  const int tiles = (a.T + 15) / 16, blocks = (tiles + 3) / 4, mt = (tiles + blocks - 1) / blocks;
  const int64_t work = (int64_t)((a.V + 15) / 16) * ((tiles + mt - 1) / mt);  // tiles of vocabulary rows, for each token block
  if (a.nb < 4) {  // fewer blocks than a chunk
    if (mt == 1) return launch_one<KIND, kFromBf16, 1, 1, 1, 1, 8>(a, st);
    if (mt == 2) return launch_one<KIND, kFromBf16, 1, 2, 1, 1, 8>(a, st);
    if (mt == 3) return launch_one<KIND, kFromBf16, 1, 3, 1, 1, 8>(a, st);
    return launch_one<KIND, kFromBf16, 1, 4, 1, 1, 8>(a, st);
  }
  if (mt == 1) {
    if (work <= (int64_t)4 * cus) return launch_one<KIND, kFromBf16, 1, 1, 1, 4, 4>(a, st);
    return launch_one<KIND, kFromBf16, 1, 1, 1, 4, 8>(a, st);
  }
  if (mt == 3) return launch_48<KIND>(a, work, cus, st);
  if (work <= (int64_t)8 * cus) {
    if (mt == 2) return launch_one<KIND, kFromBf16, 1, 2, 1, 4, 8>(a, st);
    return launch_one<KIND, kFromBf16, 1, 4, 1, 2, 8>(a, st);
  }
  if (mt == 2) return launch_rounds<KIND, 2>(a, work, cus, st);
  return launch_rounds<KIND, 4>(a, work, cus, st);
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
  // float32 rows are split by the product's own loads where they and the table are few, else once, before it
  const int cus = compute_units();
  if (cus <= 0) return SS_ERR_HIP;
  const bool few = T <= (dtype == SS_F32 ? 4 : 16) && few_pays(a, dtype == SS_F32, cus);  // reads rows at any address
  const bool direct = few || (wide_rows(h, ld_h, dtype) && (dtype == SS_BF16 || (T <= 16 && small_for_split(a, kind, cus))));
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
  if (dtype == SS_F32) {
    switch (kind) {
      case kInt128: launch_head_f32<kInt128>(a, direct, cus, st); break;
      case kInt64: launch_head_f32<kInt64>(a, direct, cus, st); break;
      case kInt32: launch_head_f32<kInt32>(a, direct, cus, st); break;
      default: launch_head_f32<kMx>(a, direct, cus, st); break;
    }
  } else {
    switch (kind) {
      case kInt128: launch_head_bf16<kInt128>(a, cus, st); break;
      case kInt64: launch_head_bf16<kInt64>(a, cus, st); break;
      case kInt32: launch_head_bf16<kInt32>(a, cus, st); break;
      default: launch_head_bf16<kMx>(a, cus, st); break;
    }
  }
  return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_HIP;
}

}  // extern "C"
