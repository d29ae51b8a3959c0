// ss_embed.hip -- rows of the vocabulary table by token (ss_embed,
// ss_embed_w4) and the gradient of the lookup by sorted tokens (ss_embed_grad).
//
// Gradient: one launch sorts the tokens, one sums long runs in pieces, one
// writes the table's rows.
//   Sort.  Each workgroup owns a range of ids and scans all tokens: it counts
//   those below its range (where its part of the sorted list starts) and, per
//   wave and id, those in it; the second scan puts each position in its
//   place, in ascending order for each id.  No workgroup waits for another and no
//   atomics decide an order.  The scan costs (V / range) * T * 8 bytes of L2 reads,
//   against T * H * 2 or more of the sum and V * H * 2 or more of the result.
//   Sum.  A row whose run is short adds its rows of dout in order.  The list is cut at
//   multiples of kRun; of a longer run, each cut's part is summed by a
//   workgroup of its own and the row adds the parts in order.
#include <hip/hip_runtime.h>

#include "ss_w4.hpp"

namespace ss {

// ---------------------------------------------------------------------------
// Lookup
// ---------------------------------------------------------------------------
struct EmbedArgs {
  const int32_t* tokens;
  const void* table;
  const uint8_t* scales;
  void* out;
  int64_t ld, ld_out;
  float scale;
  int T, V, H, nb;
  int wide_in, wide_out;
};

constexpr int kCols = 2048;  // of a workgroup: 256 threads of eight columns

template <int DT, int ODT>
__global__ __launch_bounds__(256) void ss_embed_kernel(EmbedArgs a) {
  const int t = blockIdx.x;
  const int col = blockIdx.y * kCols + threadIdx.x * 8;
  if (col >= a.H) return;
  const int v = a.tokens[t];
  float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (v >= 0 && v < a.V) {
    row_load8<DT>(a.table, (int64_t)v * a.ld + col, a.H - col, a.wide_in, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= a.scale;
  }
  row_store8<ODT>(a.out, (int64_t)t * a.ld_out + col, a.H - col, a.wide_out, x);
}

template <int KIND, int ODT>
__global__ __launch_bounds__(256) void ss_embed_w4_kernel(EmbedArgs a) {
  const int t = blockIdx.x;
  const int o = blockIdx.y * (kCols / 8) + threadIdx.x;  // octet of the row
  const int col = o * 8;
  if (col >= a.H) return;
  const int v = a.tokens[t];
  float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (v >= 0 && v < a.V) {
    const int64_t block = (int64_t)v * a.nb + (o >> 4);
    const int ob = o & 15;
    const uint32_t word = reinterpret_cast<const uint32_t*>(a.table)[block * 16 + (ob & 3) * 4 + (ob >> 2)];
    const int64_t group = (int64_t)v * a.nb * w4_groups(KIND) + col / w4_group(KIND);
    float s;
    if constexpr (KIND == kMx)
      s = mx_scale(a.scales[group]);
    else
      s = bf16_value(reinterpret_cast<const uint16_t*>(a.scales)[group]);
    const u32x4 e = w4_expand<KIND>(word, 1.0f);  // codes: exact
    const uint32_t u[4] = {e.x, e.y, e.z, e.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // code * scale is exact in float32 (4 and 8 bits), the product is rounded once
      x[2 * i] = __uint_as_float(u[i] << 16) * s * a.scale;
      x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u) * s * a.scale;
    }
  }
  row_store8<ODT>(a.out, (int64_t)t * a.ld_out + col, a.H - col, a.wide_out, x);
}

// ---------------------------------------------------------------------------
// Gradient: the sorted list
// ---------------------------------------------------------------------------
constexpr int kRange = 256;      // ids of a sorting workgroup
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kRun = 64;         // longest run that its row adds by itself

struct GradArgs {
  const void* dout;
  const int32_t* tokens;
  void* out;
  int32_t* start;   // [V + 1] first place of each id in the list
  int32_t* perm;    // [T] positions, by id and position
  int32_t* ids;     // [T] ids of the list
  float* part;      // [cuts][2][H] sums of long runs' parts
  int64_t ld, ld_out;
  float scale;
  int T, V, H;
  int wide_in, wide_out, accumulate;
};

__global__ __launch_bounds__(kSortThreads) void ss_grad_sort_kernel(GradArgs a) {
  __shared__ int place[kSortWaves][kRange];
  __shared__ int total[kRange];
  __shared__ int below[kSortWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int v0 = blockIdx.x * kRange;
  const int v1 = v0 + kRange < a.V ? v0 + kRange : a.V;
  // each wave scans a stretch of whole 64s
  const int stretch = (((a.T + kSortWaves - 1) / kSortWaves) + 63) & ~63;
  const int64_t s0 = (int64_t)wave * stretch;
  const int begin = s0 < a.T ? (int)s0 : a.T;
  const int end = s0 + stretch < a.T ? (int)(s0 + stretch) : a.T;
  for (int i = tid; i < kSortWaves * kRange; i += kSortThreads) (&place[0][0])[i] = 0;
  __syncthreads();
  constexpr int BATCH = 8;  // 64s of tokens in flight
  auto load = [&](int t0, int (&v)[BATCH]) {
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int t = t0 + i * 64 + lane;
      const int x = a.tokens[t < end ? t : end - 1];
      v[i] = t < end ? x : -1;
    }
  };
  int under = 0;
  for (int t0 = begin; t0 < end; t0 += 64 * BATCH) {
    int v[BATCH];
    load(t0, v);
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      under += v[i] >= 0 && v[i] < v0;
      if (v[i] >= v0 && v[i] < v1) atomicAdd(&place[wave][v[i] - v0], 1);
    }
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) under += __shfl_xor(under, d);
  if (lane == 0) below[wave] = under;
  __syncthreads();
  int mine = 0;  // of id v0 + tid: its places, and each wave's first among them
  if (tid < kRange) {
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = place[w][tid];
      place[w][tid] = mine;
      mine += c;
    }
    total[tid] = mine;
  }
  __syncthreads();
  for (int d = 1; d < kRange; d <<= 1) {  // inclusive sums over the range
    int add = 0;
    if (tid < kRange && tid >= d) add = total[tid - d];
    __syncthreads();
    if (tid < kRange) total[tid] += add;
    __syncthreads();
  }
  if (tid < kRange) {
    int first = total[tid] - mine;
    for (int w = 0; w < kSortWaves; ++w) first += below[w];
    if (v0 + tid < a.V) a.start[v0 + tid] = first;
    if (v0 + tid == a.V - 1) a.start[a.V] = first + mine;
    for (int w = 0; w < kSortWaves; ++w) place[w][tid] += first;
  }
  __syncthreads();
  volatile int* mp = place[wave];
  for (int t0 = begin; t0 < end; t0 += 64 * BATCH) {
    int batch[BATCH];
    load(t0, batch);
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int v = batch[i];
      const bool in = v >= v0 && v < v1;
      uint64_t same = __ballot(in);
      if (!same) continue;
      const int id = in ? v - v0 : 0;
#pragma unroll
      for (int bit = 1; bit < kRange; bit <<= 1) {
        const uint64_t b = __ballot(in && (id & bit));
        same &= (id & bit) ? b : ~b;
      }
      if (in) {  // lanes of one id: places in lane order, the last lane moves the id on
        const int rank = __popcll(same & ((1ull << lane) - 1ull));
        const int at = mp[id] + rank;
        a.perm[at] = t0 + i * 64 + lane;
        a.ids[at] = v;
        if (rank + 1 == __popcll(same)) mp[id] = at + 1;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Gradient: sums
// ---------------------------------------------------------------------------
// A thread's columns of a tile of kCols: one octet where the table is bfloat16, two quads half a tile apart where it is
// float32, so that a wave's loads and stores are up to 16 bytes a lane and lie together.
template <int ODT>
struct Cols {
  static constexpr int kPieces = ODT == SS_F32 ? 2 : 1, kWide = 8 / kPieces;
  static __device__ int at(int piece) {
    return blockIdx.y * kCols + piece * (kCols / kPieces) + (int)threadIdx.x * kWide;
  }
};

// N columns of a row in float32, `left` of which it has.
template <int DT, int N>
__device__ __forceinline__ void cols_load(const void* p, int64_t at, int left, bool wide, float* x) {
  if constexpr (N == 8) {
    float y[8];
    row_load8<DT>(p, at, left, wide, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = y[i];
  } else if (wide && left >= 4) {
    if constexpr (DT == SS_F32) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(p) + at);
      x[0] = v[0], x[1] = v[1], x[2] = v[2], x[3] = v[3];
    } else {
      const uint2 u = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint16_t*>(p) + at);
      x[0] = __uint_as_float(u.x << 16), x[1] = __uint_as_float(u.x & 0xFFFF0000u);
      x[2] = __uint_as_float(u.y << 16), x[3] = __uint_as_float(u.y & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = 0.0f;
      if (i < left)
        x[i] = DT == SS_F32 ? reinterpret_cast<const float*>(p)[at + i] : bf16_value(reinterpret_cast<const uint16_t*>(p)[at + i]);
    }
  }
}

template <int DT, int N>
__device__ __forceinline__ void cols_store(void* p, int64_t at, int left, bool wide, const float* x) {
  if constexpr (N == 8) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i];
    row_store8<DT>(p, at, left, wide, y);
  } else if (wide && left >= 4) {
    *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(p) + at) = f32x4{x[0], x[1], x[2], x[3]};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) reinterpret_cast<float*>(p)[at + i] = x[i];
  }
}

// Adds list entries [p0, p1) of a thread's columns, in order, kDeep rows in flight.
constexpr int kDeep = 8;
template <int DT, int ODT>
__device__ __forceinline__ void add_rows(const GradArgs& a, int p0, int p1, float x[8]) {
  using C = Cols<ODT>;
  for (int p = p0; p < p1; p += kDeep) {
    float y[kDeep][8];
#pragma unroll
    for (int q = 0; q < kDeep; ++q) {
      if (p + q < p1) {
        const int64_t row = (int64_t)a.perm[p + q] * a.ld;
#pragma unroll
        for (int i = 0; i < C::kPieces; ++i)
          cols_load<DT, C::kWide>(a.dout, row + C::at(i), a.H - C::at(i), a.wide_in, y[q] + i * C::kWide);
      }
    }
#pragma unroll
    for (int q = 0; q < kDeep; ++q) {
      if (p + q < p1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] += y[q][i];
      }
    }
  }
}

// Piece `piece` of a cut's two parts, float32 rows of H columns rounded up to 4.
template <int ODT>
__device__ __forceinline__ float* part_row(const GradArgs& a, int cut, int piece) {
  return a.part + ((int64_t)cut * 2 + piece) * ((a.H + 3) & ~3);
}

template <int DT, int ODT>
__device__ __forceinline__ void sum_part(const GradArgs& a, int p0, int p1, int cut, int piece) {
  using C = Cols<ODT>;
  float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  add_rows<DT, ODT>(a, p0, p1, x);
  float* o = part_row<ODT>(a, cut, piece);
#pragma unroll
  for (int i = 0; i < 8; i += 4) {
    const int col = C::at(i / C::kWide) + i % C::kWide;
    if (col < a.H) cols_store<SS_F32, 4>(o, col, 4, true, x + i);
  }
}

// A cut of kRun entries holds parts of two long runs at most: one that began at or before
// its first entry (piece 0) and one that begins later and leaves it (piece 1).
template <int DT, int ODT>
__global__ __launch_bounds__(256) void ss_grad_parts_kernel(GradArgs a) {
  const int cut = blockIdx.x;
  const int n = a.start[a.V];
  const int p0 = cut * kRun, p1 = p0 + kRun < n ? p0 + kRun : n;
  if (p0 >= p1) return;
  const int u = a.ids[p0], u0 = a.start[u], u1 = a.start[u + 1];
  const int w = a.ids[p1 - 1], w0 = a.start[w], w1 = a.start[w + 1];
  if (u1 - u0 > kRun) sum_part<DT, ODT>(a, p0, u1 < p1 ? u1 : p1, cut, 0);
  if (w != u && w1 - w0 > kRun) sum_part<DT, ODT>(a, w0, p1, cut, 1);
}

constexpr int kRows = 8;  // of a workgroup: what it takes to start one is spread over them

template <int DT, int ODT>
__global__ __launch_bounds__(256) void ss_grad_rows_kernel(GradArgs a) {
  using C = Cols<ODT>;
  const int v0 = blockIdx.x * kRows;
  int start[kRows + 1];
#pragma unroll
  for (int r = 0; r <= kRows; ++r) start[r] = a.start[v0 + r < a.V ? v0 + r : a.V];
  if (!a.accumulate) {
    const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      if (start[r] != start[r + 1] || v0 + r >= a.V) continue;
#pragma unroll
      for (int i = 0; i < C::kPieces; ++i)
        cols_store<ODT, C::kWide>(a.out, (int64_t)(v0 + r) * a.ld_out + C::at(i), a.H - C::at(i), a.wide_out, zero);
    }
  }
#pragma unroll 1
  for (int r = 0; r < kRows; ++r) {
    const int v = v0 + r;
    if (v >= a.V) break;
    const int p0 = a.start[v], p1 = a.start[v + 1];
    if (p0 == p1) continue;
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (p1 - p0 <= kRun) {
      add_rows<DT, ODT>(a, p0, p1, x);
    } else {
      for (int cut = p0 / kRun; cut * kRun < p1; ++cut) {
        const float* q = part_row<ODT>(a, cut, p0 > cut * kRun);
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
          const int col = C::at(i / C::kWide) + i % C::kWide;
          float y[4] = {0.f, 0.f, 0.f, 0.f};
          if (col < a.H) cols_load<SS_F32, 4>(q, col, 4, true, y);
#pragma unroll
          for (int k = 0; k < 4; ++k) x[i + k] += y[k];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= a.scale;
#pragma unroll
    for (int i = 0; i < C::kPieces; ++i) {
      const int64_t at = (int64_t)v * a.ld_out + C::at(i);
      const int left = a.H - C::at(i);
      if (a.accumulate) {
        float y[8];
        cols_load<ODT, C::kWide>(a.out, at, left, a.wide_out, y);
#pragma unroll
        for (int k = 0; k < C::kWide; ++k) x[i * C::kWide + k] += y[k];
      }
      cols_store<ODT, C::kWide>(a.out, at, left, a.wide_out, x + i * C::kWide);
    }
  }
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
static bool is_type(int dt) { return dt == SS_F32 || dt == SS_BF16; }
static size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

struct GradLayout {
  size_t start, perm, ids, part, total;
};
static bool grad_layout(int T, int V, int H, GradLayout* l) {
  if (T < 0 || T > SS_MAX_T || V < 1 || V > SS_MAX_V || H < 1 || H > SS_MAX_H) return false;
  size_t o = 0;
  l->start = o, o = align256(o + ((size_t)V + 1) * 4);
  l->perm = o, o = align256(o + (size_t)T * 4);
  l->ids = o, o = align256(o + (size_t)T * 4);
  l->part = o, o = align256(o + (size_t)((T + kRun - 1) / kRun) * 2 * ((H + 3) & ~3) * 4);
  l->total = o;
  return true;
}

template <int DT, int ODT>
static void launch_sums(const GradArgs& a, unsigned tiles, hipStream_t st) {
  if (a.T > kRun) {
    const dim3 grid((unsigned)((a.T + kRun - 1) / kRun), tiles);
    hipLaunchKernelGGL((ss_grad_parts_kernel<DT, ODT>), grid, dim3(256), 0, st, a);
  }
  const dim3 grid((unsigned)((a.V + kRows - 1) / kRows), tiles);
  hipLaunchKernelGGL((ss_grad_rows_kernel<DT, ODT>), grid, dim3(256), 0, st, a);
}

template <int KIND>
static void launch_embed_w4(const EmbedArgs& a, int odt, dim3 grid, hipStream_t st) {
  if (odt == SS_F32)
    hipLaunchKernelGGL((ss_embed_w4_kernel<KIND, SS_F32>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((ss_embed_w4_kernel<KIND, SS_BF16>), grid, dim3(256), 0, st, a);
}

}  // namespace ss

using namespace ss;

extern "C" {

ss_status ss_embed(const int32_t* tokens, int T, const void* table, int dtype, int V, int H, int64_t ld, float scale,
                   void* out, int out_dtype, int64_t ld_out, void* stream) {
  if (!is_type(dtype) || !is_type(out_dtype) || T < 0 || T > SS_MAX_T || V < 1 || V > SS_MAX_V || H < 1 || H > SS_MAX_H)
    return SS_ERR_INVALID_ARG;
  if (T == 0) return SS_OK;
  if (!tokens || !table || !out || ld < H || ld_out < H) return SS_ERR_INVALID_ARG;
  EmbedArgs a = {};
  a.tokens = tokens;
  a.table = table;
  a.out = out;
  a.ld = ld;
  a.ld_out = ld_out;
  a.scale = scale;
  a.T = T;
  a.V = V;
  a.H = H;
  a.wide_in = wide_rows(table, ld, dtype);
  a.wide_out = wide_rows(out, ld_out, out_dtype);
  const dim3 grid((unsigned)T, (unsigned)((H + kCols - 1) / kCols));
  const hipStream_t st = (hipStream_t)stream;
  if (dtype == SS_F32 && out_dtype == SS_F32)
    hipLaunchKernelGGL((ss_embed_kernel<SS_F32, SS_F32>), grid, dim3(256), 0, st, a);
  else if (dtype == SS_F32)
    hipLaunchKernelGGL((ss_embed_kernel<SS_F32, SS_BF16>), grid, dim3(256), 0, st, a);
  else if (out_dtype == SS_F32)
    hipLaunchKernelGGL((ss_embed_kernel<SS_BF16, SS_F32>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((ss_embed_kernel<SS_BF16, SS_BF16>), grid, dim3(256), 0, st, a);
  return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_HIP;
}

ss_status ss_embed_w4(const int32_t* tokens, int T, const ss_w4* t, float scale, void* out, int out_dtype,
                      int64_t ld_out, void* stream) {
  if (!t || !is_type(out_dtype) || T < 0 || T > SS_MAX_T) return SS_ERR_INVALID_ARG;
  const int kind = w4_kind(t);
  if (kind < 0) return SS_ERR_INVALID_ARG;
  if (T == 0) return SS_OK;
  if (!tokens || !out || !w4_aligned(t->codes) || !w4_aligned(t->scales) || ld_out < t->H) return SS_ERR_INVALID_ARG;
  EmbedArgs a = {};
  a.tokens = tokens;
  a.table = t->codes;
  a.scales = reinterpret_cast<const uint8_t*>(t->scales);
  a.out = out;
  a.ld_out = ld_out;
  a.scale = scale;
  a.T = T;
  a.V = t->V;
  a.H = t->H;
  a.nb = w4_blocks(t->H);
  a.wide_out = wide_rows(out, ld_out, out_dtype);
  const dim3 grid((unsigned)T, (unsigned)((t->H + kCols - 1) / kCols));
  const hipStream_t st = (hipStream_t)stream;
  switch (kind) {
    case kInt128: launch_embed_w4<kInt128>(a, out_dtype, grid, st); break;
    case kInt64: launch_embed_w4<kInt64>(a, out_dtype, grid, st); break;
    case kInt32: launch_embed_w4<kInt32>(a, out_dtype, grid, st); break;
    default: launch_embed_w4<kMx>(a, out_dtype, grid, st); break;
  }
  return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_HIP;
}

size_t ss_embed_grad_bytes(int T, int V, int H) {
  GradLayout l;
  return grad_layout(T, V, H, &l) ? l.total : 0;
}

ss_status ss_embed_grad(const void* dout, int dtype, int T, int64_t ld, const int32_t* tokens, int V, int H,
                        float scale, void* dtable, int out_dtype, int64_t ld_out, int accumulate, void* ws,
                        size_t ws_bytes, void* stream) {
  GradLayout l;
  if (!is_type(dtype) || !is_type(out_dtype) || !grad_layout(T, V, H, &l)) return SS_ERR_INVALID_ARG;
  if (!dtable || !ws || ld_out < H || (T > 0 && (!dout || !tokens || ld < H))) return SS_ERR_INVALID_ARG;
  if (ws_bytes < l.total || ((uintptr_t)ws & 15u)) return SS_ERR_WORKSPACE;
  unsigned char* w = reinterpret_cast<unsigned char*>(ws);
  GradArgs a = {};
  a.dout = dout;
  a.tokens = tokens;
  a.out = dtable;
  a.start = reinterpret_cast<int32_t*>(w + l.start);
  a.perm = reinterpret_cast<int32_t*>(w + l.perm);
  a.ids = reinterpret_cast<int32_t*>(w + l.ids);
  a.part = reinterpret_cast<float*>(w + l.part);
  a.ld = ld;
  a.ld_out = ld_out;
  a.scale = scale;
  a.T = T;
  a.V = V;
  a.H = H;
  a.wide_in = T > 0 && wide_rows(dout, ld, dtype);
  a.wide_out = wide_rows(dtable, ld_out, out_dtype);
  a.accumulate = accumulate;
  const hipStream_t st = (hipStream_t)stream;
  const unsigned tiles = (unsigned)((H + kCols - 1) / kCols);
  hipLaunchKernelGGL(ss_grad_sort_kernel, dim3((unsigned)((V + kRange - 1) / kRange)), dim3(kSortThreads), 0, st, a);
  if (dtype == SS_F32)
    out_dtype == SS_F32 ? launch_sums<SS_F32, SS_F32>(a, tiles, st) : launch_sums<SS_F32, SS_BF16>(a, tiles, st);
  else
    out_dtype == SS_F32 ? launch_sums<SS_BF16, SS_F32>(a, tiles, st) : launch_sums<SS_BF16, SS_BF16>(a, tiles, st);
  return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_HIP;
}

}  // extern "C"
