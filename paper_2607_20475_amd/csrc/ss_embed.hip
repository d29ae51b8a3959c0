// ss_embed.hip -- rows of the vocabulary table by token (ss_embed,
// ss_embed_w4) and the gradient of the lookup by sorted tokens (ss_embed_grad).
//
// Gradient: one launch sorts the tokens, one writes the table's rows but those of
// long runs, which it sums in parts, one joins these parts.  Bound by memory: V * H
// written, T * H read.
//   Sort.  Each workgroup owns a range of ids and scans all tokens: it counts
//   those below its range (where its part of the sorted list starts) and, per
//   wave and id, those in it; the second scan puts each position in its
//   place, in ascending order for each id.  No workgroup waits for another and no
//   atomics decide an order.  The scans read (V / range) * T * 4 bytes from L2, twice that
//   above 16384 tokens, which a wave's registers do not hold from one to the other,
//   against T * H * 2 or more of the sum and V * H * 2 or more of the result: 6 us at V =
//   32768, T = 2048 (of 65 in all, H = 2048, float32), 19 at V = 131072, T = 16384 (of 455, below).
//   When accumulating, only named rows are written, and the sort and the chain of three
//   launches weigh more: 23 us at T = 2048 (985 rows of H = 2048 float32, 31 MB), 129 at T = 16384
//   (6305 of H = 4096, 327 MB), 16 at T = 64, V = 131072.
//   Sum.  A row whose run is short adds its rows of dout in order.  The list is cut at
//   multiples of kRun; of a longer run, each cut's part is summed by a
//   workgroup of its own and a last launch adds the parts in order (5 and 9 us).
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

// Each octet of columns is read once, expanded, scaled and written once: bound by memory, and by the launch where there are few
// tokens.  A workgroup has a token's 2048 columns, 16 bytes of bfloat16 a thread.  H = 4096, bfloat16 out: 8192 tokens from a 4-bit
// table 15.8 us (5.2 TB/s of codes read and rows written), 320 from a bfloat16 one 2.9 us.
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
constexpr int kFewLanes = 8;
constexpr int kRun = 32;         // longest run that its row adds by itself

struct GradArgs {
  const void* dout;
  const int32_t* tokens;
  void* out;
  int32_t* start;   // [V + 1] first place of each id in the list
  int4* list;       // [T] by id and position: the position, the id, its run's first and last place + 1
  float* part;      // [cuts][2][H] sums of long runs' parts
  int64_t ld, ld_out;
  float scale;
  int T, V, H;
  int wide_in, wide_out, accumulate;
  uint32_t blocks;                     // workgroups that have something to do
  uint32_t tiles, wtiles, cuts, heads;  // column tiles, one and kWide; cuts of the list; groups of kHeads entries
  uint32_t strips;                     // waves' pieces of 1 KB of a row
};

__global__ __launch_bounds__(kSortThreads) void ss_grad_sort_kernel(GradArgs a) {
  __shared__ int place[kSortWaves][kRange];
  __shared__ int run[kRange][2];
  __shared__ int total[kRange / 64];
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
  constexpr int BATCH = 16;  // 64s of tokens in flight
  int batch[BATCH];
  auto load = [&](int t0) {
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int t = t0 + i * 64 + lane;
      const int x = a.tokens[t < end ? t : end - 1];
      batch[i] = t < end ? x : -1;
    }
  };
  int under = 0;
  for (int t0 = begin; t0 < end; t0 += 64 * BATCH) {
    load(t0);
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      under += batch[i] >= 0 && batch[i] < v0;
      if (batch[i] >= v0 && batch[i] < v1) atomicAdd(&place[wave][batch[i] - v0], 1);
    }
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) under += __shfl_xor(under, d);
  if (lane == 0) below[wave] = under;
  __syncthreads();
  int mine = 0, upto = 0;  // of id v0 + tid: its places; of it and its wave's ids before it
  if (tid < kRange) {
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) mine += place[w][tid];
    upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(upto, d);
      if (lane >= d) upto += o;
    }
    if (lane == 63) total[wave] = upto;
  }
  __syncthreads();
  if (tid < kRange) {
    int first = upto - mine;
    for (int w = 0; w < wave; ++w) first += total[w];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) first += below[w];
    if (v0 + tid < a.V) a.start[v0 + tid] = first;
    if (v0 + tid == a.V - 1) a.start[a.V] = first + mine;
    run[tid][0] = first, run[tid][1] = first + mine;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {  // each wave's first place of the id
      const int c = place[w][tid];
      place[w][tid] = first;
      first += c;
    }
  }
  __syncthreads();
  volatile int* mp = place[wave];
  for (int t0 = begin; t0 < end; t0 += 64 * BATCH) {
    if (end - begin > 64 * BATCH) load(t0);  // else the first scan's are still there
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int v = batch[i];
      const bool in = v >= v0 && v < v1;
      uint64_t same = __ballot(in);
      if (!same) continue;
      const int id = in ? v - v0 : 0;
      // the lanes of each lane's id: few lanes id by id, many bit by bit
      if (__popcll(same) <= kFewLanes) {
        for (uint64_t todo = same; todo;) {
          const int one = __builtin_amdgcn_readlane(id, __ffsll((unsigned long long)todo) - 1);
          const uint64_t m = __ballot(in && id == one);
          if (id == one) same = m;
          todo &= ~m;
        }
      } else {
#pragma unroll
        for (int bit = 1; bit < kRange; bit <<= 1) {
          const uint64_t b = __ballot(in && (id & bit));
          same &= (id & bit) ? b : ~b;
        }
      }
      if (in) {  // lanes of one id: places in lane order, the last lane moves the id on
        const int rank = __popcll(same & ((1ull << lane) - 1ull));
        const int at = mp[id] + rank;
        a.list[at] = make_int4(t0 + i * 64 + lane, v, run[id][0], run[id][1]);
        if (rank + 1 == __popcll(same)) mp[id] = at + 1;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Gradient: sums
// ---------------------------------------------------------------------------
// A thread has 16 bytes of the table: N = 4 columns of float32 or 8 of bfloat16, of a tile of 256 N.
template <int ODT>
struct Cols {
  static constexpr int N = ODT == SS_F32 ? 4 : 8, kTile = 256 * N;
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

// Adds D list entries from p on, all in flight at once: W pieces of N columns, a tile apart, from col on.
template <int DT, int N, int W, int D>
__device__ __forceinline__ void add_some(const GradArgs& a, int p, int col, float (&x)[W][N]) {
  int t[D];
  float y[D][W][N];
#pragma unroll
  for (int q = 0; q < D; ++q) t[q] = a.list[p + q].x;
#pragma unroll
  for (int q = 0; q < D; ++q)
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const int c = col + w * 256 * N;
      cols_load<DT, N>(a.dout, (int64_t)t[q] * a.ld + c, a.H - c, a.wide_in, y[q][w]);
    }
#pragma unroll
  for (int q = 0; q < D; ++q)
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int i = 0; i < N; ++i) x[w][i] += y[q][w][i];
}

// Adds list entries [p0, p1), in order.
template <int DT, int N, int W>
__device__ __forceinline__ void add_rows(const GradArgs& a, int p0, int p1, int col, float (&x)[W][N]) {
  constexpr int D = (W == 1 ? 64 : 16) / N;
#pragma unroll
  for (int w = 0; w < W; ++w)
#pragma unroll
    for (int i = 0; i < N; ++i) x[w][i] = 0.0f;
  int p = p0;
  for (; p + D <= p1; p += D) add_some<DT, N, W, D>(a, p, col, x);
  if constexpr (D > 8)
    if (p + 8 <= p1) add_some<DT, N, W, 8>(a, p, col, x), p += 8;
  if constexpr (D > 4)
    if (p + 4 <= p1) add_some<DT, N, W, 4>(a, p, col, x), p += 4;
  if constexpr (D > 2)
    if (p + 2 <= p1) add_some<DT, N, W, 2>(a, p, col, x), p += 2;
  if (p < p1) add_some<DT, N, W, 1>(a, p, col, x);
}

// Writes a row's sum, scaled and rounded, or adds it to the row.
template <int ODT, int N>
__device__ __forceinline__ void put_row(const GradArgs& a, int v, int col, float x[N]) {
  const int64_t at = (int64_t)v * a.ld_out + col;
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] *= a.scale;
  if (a.accumulate) {
    float y[N];
    cols_load<ODT, N>(a.out, at, a.H - col, a.wide_out, y);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] += y[i];
  }
  cols_store<ODT, N>(a.out, at, a.H - col, a.wide_out, x);
}

// The two pieces of a cut, float32 rows of H columns rounded up to 8.
__device__ __forceinline__ float* part_row(const GradArgs& a, int cut, int piece) {
  return a.part + ((int64_t)cut * 2 + piece) * ((a.H + 7) & ~7);
}

template <int DT, int N>
__device__ __forceinline__ void sum_part(const GradArgs& a, int p0, int p1, int cut, int piece, int col) {
  float x[1][N];
  add_rows<DT, N, 1>(a, p0, p1, col, x);
  cols_store<SS_F32, N>(part_row(a, cut, piece), col, N, true, x[0]);
}

// Three kinds of workgroups in one launch:
//   parts   of long runs.  A cut of kRun entries holds parts of two such runs at most, one that began at or before
//           its first entry (piece 0) and one that begins later and leaves it (piece 1).
//   runs    the rows of the short runs that begin among kHeads entries.  The list, not the table, is
//           shared out: wherever its rows lie, the runs go to all parts of the chip.
//   zeros   the rows without a run, in the order of memory, kPieces pieces of 1 KB to a wave (none when accumulating).  V = 112616,
//           H = 2816, float32, T = 97: 230 us (5.5 TB/s; pieces of 4 KB to a workgroup, the row's last not full: 248).
// The first two start first, the zeros' stores follow: dealt out in turn with them, loads and stores that lie apart slow the
// stores in order down (583 us at the following size).  16384 tokens by Zipf's law, bfloat16 to float32, V = 131072, H = 4096
// (2.27 GB), with sort and join: 459 us; pieces 1, 2 and 8 618, 476 and 462
// (the 112616 rows: 235 of 4, 285, 225 and 240); runs up to 16 and 64 entries short 458 and 457 (T = 2048, V =
// 32768, H = 2048, float32: 68 of 32, 68 and 75; T = 16384, accumulating: 129 of 32, 122 and 152).  One entry a workgroup puts runs of
// equal lengths on few XCDs (2000 runs of 8: 648 against 464).
constexpr int kHeads = 3, kPieces = 4, kWide = 2;

template <int DT, int ODT>
__global__ __launch_bounds__(256) void ss_grad_rows_kernel(GradArgs a) {
  constexpr int N = Cols<ODT>::N, TILE = Cols<ODT>::kTile;
  uint32_t b = blockIdx.x + blockIdx.y * gridDim.x;
  if (b >= a.blocks) return;
  if (b < a.cuts * a.tiles) {
    const int cut = (int)(b / a.tiles), col = (int)(b % a.tiles) * TILE + (int)threadIdx.x * N;
    const int n = a.start[a.V];
    const int p0 = cut * kRun, p1 = p0 + kRun < n ? p0 + kRun : n;
    if (p0 >= p1 || col >= a.H) return;
    const int4 u = a.list[p0], w = a.list[p1 - 1];
    if (u.w - u.z > kRun) sum_part<DT, N>(a, p0, u.w < p1 ? u.w : p1, cut, 0, col);
    if (w.y != u.y && w.w - w.z > kRun) sum_part<DT, N>(a, w.z, p1, cut, 1, col);
    return;
  }
  b -= a.cuts * a.tiles;
  if (b < a.heads * a.wtiles) {
    const int h = (int)(b / a.wtiles) * kHeads, col = (int)(b % a.wtiles) * (kWide * TILE) + (int)threadIdx.x * N;
    const int n = a.start[a.V];
    int4 e[kHeads];
#pragma unroll
    for (int k = 0; k < kHeads; ++k) e[k] = a.list[h + k < a.T ? h + k : a.T - 1];
#pragma unroll
    for (int k = 0; k < kHeads; ++k) {
      // not in the list, not a run's first entry, or a long run's
      if (h + k >= n || e[k].z != h + k || e[k].w - e[k].z > kRun) continue;
      float x[kWide][N];
      add_rows<DT, N, kWide>(a, e[k].z, e[k].w, col, x);
#pragma unroll
      for (int w = 0; w < kWide; ++w) put_row<ODT, N>(a, e[k].y, col + w * TILE, x[w]);
    }
    return;
  }
  b -= a.heads * a.wtiles;
  const float zero[N] = {};
  const uint32_t first = b * (4 * kPieces) + (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t v[kPieces];
  bool none[kPieces];
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    v[k] = (first + 4 * k) / a.strips;
    none[k] = v[k] < (uint32_t)a.V && a.start[v[k]] == a.start[v[k] + 1];
  }
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    const int col = (int)(first + 4 * k - v[k] * a.strips) * (64 * N) + (int)(threadIdx.x & 63) * N;
    if (none[k]) cols_store<ODT, N>(a.out, (int64_t)v[k] * a.ld_out + col, a.H - col, a.wide_out, zero);
  }
}

// The rows of long runs: the workgroup of the cut that such a run begins in adds its parts; each wave a quarter of them,
// in order, and the quarters in order.
template <int ODT>
__global__ __launch_bounds__(256) void ss_grad_join_kernel(GradArgs a) {
  constexpr int N = Cols<ODT>::N, D = 64 / N;
  __shared__ float sums[4][64][N];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int cut = blockIdx.x, col = blockIdx.y * (64 * N) + lane * N;
  const int n = a.start[a.V];
  const int p0 = cut * kRun, p1 = p0 + kRun < n ? p0 + kRun : n;
  if (p0 >= p1) return;
  const int4 e = a.list[p1 - 1];
  if (e.z < p0 || e.w - e.z <= kRun) return;
  float x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = 0.0f;
  const int parts = (e.w - 1) / kRun + 1 - cut, from = parts * wave / 4, to = parts * (wave + 1) / 4;
  if (col < a.H) {
    for (int c = from; c < to; c += D) {
      float y[D][N];
#pragma unroll
      for (int q = 0; q < D; ++q) {
        const int k = c + q < to ? c + q : to - 1;
        cols_load<SS_F32, N>(part_row(a, cut + k, k == 0 && e.z > p0), col, N, true, y[q]);
      }
#pragma unroll
      for (int q = 0; q < D; ++q)
        if (c + q < to) {
#pragma unroll
          for (int i = 0; i < N; ++i) x[i] += y[q][i];
        }
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) sums[wave][lane][i] = x[i];
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int w = 1; w < 4; ++w)
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] += sums[w][lane][i];
  put_row<ODT, N>(a, e.y, col, x);
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
static bool is_type(int dt) { return dt == SS_F32 || dt == SS_BF16; }
static size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

struct GradLayout {
  size_t start, list, part, total;
};
static bool grad_layout(int T, int V, int H, GradLayout* l) {
  if (T < 0 || T > SS_MAX_T || V < 1 || V > SS_MAX_V || H < 1 || H > SS_MAX_H) return false;
  size_t o = 0;
  l->start = o, o = align256(o + ((size_t)V + 1) * 4);
  l->list = o, o = align256(o + (size_t)T * 16);
  l->part = o, o = align256(o + (size_t)((T + kRun - 1) / kRun) * 2 * ((H + 7) & ~7) * 4);
  l->total = o;
  return true;
}

template <int DT, int ODT>
static void launch_sums(GradArgs& a, hipStream_t st) {
  a.tiles = (uint32_t)((a.H + Cols<ODT>::kTile - 1) / Cols<ODT>::kTile);
  // A row of three pieces is dealt out as four, the last one empty, so that a workgroup's four waves have a row: V = 182836, H =
  // 1280, bfloat16, T = 1000 103 us against 110 in threes.  Two pieces stay two: V = 300000, H = 640, T = 97 80 us against 145 in fours.
  a.strips = (uint32_t)((a.H + 64 * Cols<ODT>::N - 1) / (64 * Cols<ODT>::N));
  if (a.strips == 3) a.strips = 4;
  a.cuts = a.T > kRun ? (uint32_t)((a.T + kRun - 1) / kRun) : 0u;
  a.heads = (uint32_t)((a.T + kHeads - 1) / kHeads);
  a.wtiles = (a.tiles + kWide - 1) / kWide;
  const uint32_t zeros = a.accumulate ? 0u : ((uint32_t)a.V * a.strips + 4 * kPieces - 1) / (4 * kPieces), most = 1u << 16;
  a.blocks = a.cuts * a.tiles + a.heads * a.wtiles + zeros;
  if (a.blocks == 0) return;
  // in rows of 2^16: a launch has fewer than 2^32 threads in one direction
  const dim3 grid(a.blocks < most ? a.blocks : most, (a.blocks + most - 1) / most);
  hipLaunchKernelGGL((ss_grad_rows_kernel<DT, ODT>), grid, dim3(256), 0, st, a);
  if (a.cuts) hipLaunchKernelGGL(ss_grad_join_kernel<ODT>, dim3(a.cuts, (unsigned)((a.H + 64 * Cols<ODT>::N - 1) / (64 * Cols<ODT>::N))), dim3(256), 0, st, a);
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
  a.list = reinterpret_cast<int4*>(w + l.list);
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
  hipLaunchKernelGGL(ss_grad_sort_kernel, dim3((unsigned)((V + kRange - 1) / kRange)), dim3(kSortThreads), 0, st, a);
  if (dtype == SS_F32)
    out_dtype == SS_F32 ? launch_sums<SS_F32, SS_F32>(a, st) : launch_sums<SS_F32, SS_BF16>(a, st);
  else
    out_dtype == SS_F32 ? launch_sums<SS_BF16, SS_F32>(a, st) : launch_sums<SS_BF16, SS_BF16>(a, st);
  return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_HIP;
}

}  // extern "C"
