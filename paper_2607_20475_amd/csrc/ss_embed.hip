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
constexpr int kRun = 128;        // longest run that its row adds by itself

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
  int under = 0;
  for (int t = begin + lane; t < end; t += 64) {
    const int v = a.tokens[t];
    under += v >= 0 && v < v0;
    if (v >= v0 && v < v1) atomicAdd(&place[wave][v - v0], 1);
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
  for (int t0 = begin; t0 < end; t0 += 64) {
    const int t = t0 + lane;
    const int v = t < end ? a.tokens[t] : -1;
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
      a.perm[at] = t;
      a.ids[at] = v;
      if (rank + 1 == __popcll(same)) mp[id] = at + 1;
    }
  }
}

// ---------------------------------------------------------------------------
// Gradient: sums
// ---------------------------------------------------------------------------
// Adds list entries [p0, p1) of eight columns, in order, four rows in flight.
template <int DT>
__device__ __forceinline__ void add_rows(const GradArgs& a, int p0, int p1, int col, float x[8]) {
  const int left = a.H - col;
  int p = p0;
  for (; p + 4 <= p1; p += 4) {
    float y[4][8];
#pragma unroll
    for (int q = 0; q < 4; ++q) row_load8<DT>(a.dout, (int64_t)a.perm[p + q] * a.ld + col, left, a.wide_in, y[q]);
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] += y[q][i];
  }
  for (; p < p1; ++p) {
    float y[8];
    row_load8<DT>(a.dout, (int64_t)a.perm[p] * a.ld + col, left, a.wide_in, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] += y[i];
  }
}

__device__ __forceinline__ void put_part(const GradArgs& a, int cut, int piece, int col, const float x[8]) {
  float* o = a.part + ((int64_t)cut * 2 + piece) * a.H + col;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (col + i < a.H) o[i] = x[i];
}

// A cut of kRun entries holds parts of two long runs at most: one that began at or before
// its first entry (piece 0) and one that begins later and leaves it (piece 1).
template <int DT>
__global__ __launch_bounds__(256) void ss_grad_parts_kernel(GradArgs a) {
  const int cut = blockIdx.x, col = blockIdx.y * kCols + threadIdx.x * 8;
  const int n = a.start[a.V];
  const int p0 = cut * kRun, p1 = p0 + kRun < n ? p0 + kRun : n;
  if (p0 >= p1 || col >= a.H) return;
  const int u = a.ids[p0], u0 = a.start[u], u1 = a.start[u + 1];
  const int w = a.ids[p1 - 1], w0 = a.start[w], w1 = a.start[w + 1];
  if (u1 - u0 > kRun) {
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    add_rows<DT>(a, p0, u1 < p1 ? u1 : p1, col, x);
    put_part(a, cut, 0, col, x);
  }
  if (w != u && w1 - w0 > kRun) {
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    add_rows<DT>(a, w0, p1, col, x);
    put_part(a, cut, 1, col, x);
  }
}

template <int DT, int ODT>
__global__ __launch_bounds__(256) void ss_grad_rows_kernel(GradArgs a) {
  const int v = blockIdx.x;
  const int col = blockIdx.y * kCols + threadIdx.x * 8;
  if (col >= a.H) return;
  const int p0 = a.start[v], p1 = a.start[v + 1];
  if (a.accumulate && p0 == p1) return;
  float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (p1 - p0 <= kRun) {
    add_rows<DT>(a, p0, p1, col, x);
  } else {
    for (int cut = p0 / kRun; cut * kRun < p1; ++cut) {
      const float* q = a.part + ((int64_t)cut * 2 + (p0 > cut * kRun)) * a.H + col;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (col + i < a.H) x[i] += q[i];
    }
  }
  const int64_t at = (int64_t)v * a.ld_out + col;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] *= a.scale;
  if (a.accumulate) {
    float y[8];
    row_load8<ODT>(a.out, at, a.H - col, a.wide_out, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] += y[i];
  }
  row_store8<ODT>(a.out, at, a.H - col, a.wide_out, x);
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
  l->part = o, o = align256(o + (size_t)((T + kRun - 1) / kRun) * 2 * H * 4);
  l->total = o;
  return true;
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
  if (T > kRun) {
    const dim3 grid((unsigned)((T + kRun - 1) / kRun), tiles);
    if (dtype == SS_F32)
      hipLaunchKernelGGL(ss_grad_parts_kernel<SS_F32>, grid, dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL(ss_grad_parts_kernel<SS_BF16>, grid, dim3(256), 0, st, a);
  }
  const dim3 grid((unsigned)V, tiles);
  if (dtype == SS_F32 && out_dtype == SS_F32)
    hipLaunchKernelGGL((ss_grad_rows_kernel<SS_F32, SS_F32>), grid, dim3(256), 0, st, a);
  else if (dtype == SS_F32)
    hipLaunchKernelGGL((ss_grad_rows_kernel<SS_F32, SS_BF16>), grid, dim3(256), 0, st, a);
  else if (out_dtype == SS_F32)
    hipLaunchKernelGGL((ss_grad_rows_kernel<SS_BF16, SS_F32>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((ss_grad_rows_kernel<SS_BF16, SS_BF16>), grid, dim3(256), 0, st, a);
  return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_HIP;
}

}  // extern "C"
