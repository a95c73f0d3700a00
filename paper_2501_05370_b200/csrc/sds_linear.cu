// Linear layer with its epilogue, forward and backward, on the tensor cores.
//
//   forward   z = x W^T + b + table[step], y = act(z) + residual          (x [rows, k], W [n, k])
//   backward  dz = dy act'(z), dx = dz W, dW = dz^T x, db = sum_rows dz, dtable[s] = sum_{rows with step s} dz
//   (a row whose step is outside the table is NaN forward, and zeros in dz)
//
// The products are those of sds_tiles.cuh: persistent tiles for batches, weights split over clusters for few rows. Bias, table
// rows, activation and residual are applied to the accumulator, before its one rounding, so y is written once and z never.
// For the backward pass the forward one keeps act'(z) as a float: in 16 bits it would add an error to every gradient as large as that
// gradient's own rounding, and one a thousand times larger to a float db (2e-4 of it, against 2e-7).
//
// Backward: one pass over dy writes dz as operand and adds the columns for db (in float, of the unrounded dz); dx and dW
// are one launch. The table's gradient is a sum over rows in the order of their steps: the rows of each step are listed
// once (ascending), then every warp adds a slice of that list, of equal length whatever the steps are; runs that
// cross slices are joined in order. No atomics: same bits on every run.
#include "sds_tiles.cuh"

namespace sds {

namespace {

// ---------------------------------------------------------------------------------------------
// dz and the bias gradient
// ---------------------------------------------------------------------------------------------

// Kernels of this file start beside the end of the one in front, and wait for it before they read or write anything. (They let the next
// one go before that wait: it has to be one that waits in full as well, as every first kernel of a call does.) Their loads are plain
// ones: the compiler may move read-only loads ahead of the wait.
__device__ __forceinline__ void start_behind_prior_kernel() {
  launch_dependents();
  wait_for_prior_kernel();
}

struct DzArgs {
  const void* dy;                                 // [rows, n] of tdy, rows lddy elements apart
  const float* factor;                            // [rows, ldz], NULL = ones
  uint16_t* dz;                                   // [rows, ldz] of the operands' type, NULL = not wanted
  float* part;                                    // [gridDim.y][n] column sums
  void* db;                                       // NULL = not wanted; where the chunks of rows are one cluster the sums go here at once
  const int* step;                                // [rows], NULL = no table: rows whose step is outside it count as zeros
  int64_t lddy, ldz;
  int tdy, tdb, rows, n, steps, f16;
  int cluster;                                    // chunks of rows in a cluster (1: the sums go to part, unless there is but one)
};

constexpr int kDzThreads = 256, kDzWarps = kDzThreads / 32, kDzCols = 256;

__device__ __forceinline__ void store_typed(void* p, int type, size_t i, float v) {
  if (type == SDS_F32) static_cast<float*>(p)[i] = v;
  else static_cast<uint16_t*>(p)[i] = round16(v, type == SDS_F16);
}

// Eight columns of a row of dy and of its factors, as they lie in memory. Where dy's rows are not whole 16-byte pieces (WHOLE = false), the
// pieces that hold the columns are read, as far as the row goes, and shifted into place: the row's shift is the same for all lanes.
// (The factors' rows are padded to whole pieces, as dz's are.)
template <bool F32, bool WHOLE> struct DzRow { uint4 y[(F32 ? 2 : 1) + (WHOLE ? 0 : 1)], f[2]; };
template <bool F32, bool WHOLE, class A>
__device__ __forceinline__ void dz_request(DzRow<F32, WHOLE>& r, const A& a, int64_t row, int c0) {
  constexpr int kSize = F32 ? 4 : 2, kPieces = (F32 ? 2 : 1) + (WHOLE ? 0 : 1);
  const char* y = static_cast<const char*>(a.dy) + ((size_t)row * a.lddy + c0) * kSize;
  if (WHOLE) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) r.y[i] = *(reinterpret_cast<const uint4*>(y) + i);
  } else {
    const uintptr_t first = reinterpret_cast<uintptr_t>(y) & ~(uintptr_t)15;
    const uintptr_t last = reinterpret_cast<uintptr_t>(y) + (uintptr_t)(min(8, a.n - c0) * kSize - 1);
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      r.y[i] = first + 16 * i <= last ? *(reinterpret_cast<const uint4*>(first) + i) : make_uint4(0u, 0u, 0u, 0u);
  }
  if (a.factor)
#pragma unroll
    for (int i = 0; i < 2; ++i) r.f[i] = *(reinterpret_cast<const uint4*>(a.factor + (size_t)row * a.ldz + c0) + i);
}
template <bool F32, bool WHOLE, class A>
__device__ __forceinline__ void dz_values(const DzRow<F32, WHOLE>& r, const A& a, int64_t row, int c0, float (&v)[8]) {
  constexpr int kSize = F32 ? 4 : 2, kPieces = (F32 ? 2 : 1) + (WHOLE ? 0 : 1), kWords = F32 ? 8 : 4;
  uint32_t w[4 * kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) { w[4 * i] = r.y[i].x; w[4 * i + 1] = r.y[i].y; w[4 * i + 2] = r.y[i].z; w[4 * i + 3] = r.y[i].w; }
  if (!WHOLE) {
    const uint32_t shift = (uint32_t)(reinterpret_cast<uintptr_t>(a.dy) + ((size_t)row * a.lddy + c0) * kSize) & 15u;
#pragma unroll
    for (int i = 0; i < 4 * kPieces - 2; ++i) w[i] = shift & 8u ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 4 * kPieces - 3; ++i) w[i] = shift & 4u ? w[i + 1] : w[i];
    if (!F32)
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], (shift & 2u) * 8u);
  }
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    if (F32) {
      v[i] = __uint_as_float(w[i]);
    } else {
      const float2 t = unpack16x2(w[i], a.f16);
      v[(2 * i) % 8] = t.x; v[(2 * i + 1) % 8] = t.y;
    }
  }
  if (a.factor) {
    const uint32_t f[8] = {r.f[0].x, r.f[0].y, r.f[0].z, r.f[0].w, r.f[1].x, r.f[1].y, r.f[1].z, r.f[1].w};
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] *= __uint_as_float(f[u]);
  }
}
// a row whose step is outside the table: neither its dy nor its act' (NaN) counts
__device__ __forceinline__ void no_row(float (&v)[8]) {
#pragma unroll
  for (int u = 0; u < 8; ++u) v[u] = 0.f;
}
template <class A>
__device__ __forceinline__ void dz_store(const A& a, int64_t row, int c0, const float (&v)[8]) {      // (columns beyond n are padding)
  *reinterpret_cast<uint4*>(a.dz + (size_t)row * a.ldz + c0) =
      make_uint4(pack16(v[0], v[1], a.f16), pack16(v[2], v[3], a.f16), pack16(v[4], v[5], a.f16), pack16(v[6], v[7], a.f16));
}

// A lane takes eight neighbouring columns of every eighth row of its chunk, four rows requested ahead. Bound by memory: db alone of
// 8192 x 2048 bf16 behind SiLU 16.5 us (101 MB of dy and act', 6.1 TB/s); 256 x 4096 6.4 us, a launch and the exchange of its sums.
template <bool F32, bool WHOLE>
__global__ void __launch_bounds__(kDzThreads) k_linear_dz(const DzArgs a) {
  __shared__ float sums[kDzWarps][kDzCols];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c0 = blockIdx.x * kDzCols + lane * 8;
  float sum[8] = {};
  start_behind_prior_kernel();
  const int64_t stride = (int64_t)gridDim.y * kDzWarps, first = (int64_t)blockIdx.y * kDzWarps + warp;
  if (c0 < a.n) {
    constexpr int kAhead = 4;
    DzRow<F32, WHOLE> ahead[kAhead];
    int steps_ahead[kAhead] = {};
    const auto request = [&](int i, int64_t row) {
      dz_request(ahead[i], a, row, c0);
      if (a.step) steps_ahead[i] = a.step[row];
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (first + i * stride < a.rows) request(i, first + i * stride);
    for (int64_t base = first; base < a.rows; base += kAhead * stride) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int64_t row = base + i * stride, next = row + kAhead * stride;
        if (row >= a.rows) break;
        float v[8];
        dz_values(ahead[i], a, row, c0, v);
        if (a.step && (steps_ahead[i] < 0 || steps_ahead[i] >= a.steps)) no_row(v);
        if (next < a.rows) request(i, next);
#pragma unroll
        for (int u = 0; u < 8; ++u) sum[u] += v[u];
        if (a.dz) dz_store(a, row, c0, v);
      }
    }
  }
  if (!a.db) return;
  *reinterpret_cast<float4*>(&sums[warp][lane * 8]) = make_float4(sum[0], sum[1], sum[2], sum[3]);
  *reinterpret_cast<float4*>(&sums[warp][lane * 8 + 4]) = make_float4(sum[4], sum[5], sum[6], sum[7]);
  __syncthreads();
  const int c = blockIdx.x * kDzCols + threadIdx.x;
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < kDzWarps; ++w) s += sums[w][threadIdx.x];
  if (a.cluster > 1) {                            // the first CTA of the cluster adds the others' sums
    sums[0][threadIdx.x] = s;                     // (of this thread's column alone)
    cluster_sync_all();
    if (blockIdx.y == 0) {
      const uint32_t mine = smem_u32(&sums[0][threadIdx.x]);
      for (int r = 1; r < a.cluster; ++r) {
        float other;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(other) : "r"(map_to_cta(mine, (uint32_t)r)) : "memory");
        s += other;
      }
    }
    cluster_sync_all();                           // no CTA leaves while its sums may still be read
  }
  if (c >= a.n || (a.cluster > 1 && blockIdx.y > 0)) return;
  if ((int)gridDim.y == a.cluster) store_typed(a.db, a.tdb, c, s);
  else a.part[(size_t)blockIdx.y * a.n + c] = s;
}

// The chunks' column sums, added in order: 32 columns of a CTA, a warp every eighth chunk. Latency: 128 chunks of 2048 columns 5.7 us
// alone, about 1.5 beside the end of the kernel in front.
__global__ void __launch_bounds__(256) k_linear_db(const float* part, int chunks, int n, void* db, int tdb) {
  __shared__ float sums[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  start_behind_prior_kernel();
  float s = 0.f;
  if (c < n)
#pragma unroll 8
    for (int i = warp; i < chunks; i += 8) s += part[(size_t)i * n + c];
  sums[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < n) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) t += sums[w][lane];
    store_typed(db, tdb, c, t);
  }
}

// Chunks of rows: four rows for every warp, until there are two CTAs for each SM (which hold 96 KB of requests between them).
int dz_chunks(int64_t rows, int32_t n) {
  const int64_t cols = (n + kDzCols - 1) / kDzCols;
  return (int)std::max<int64_t>(1, std::min<int64_t>((rows + 4 * kDzWarps - 1) / (4 * kDzWarps), 2 * 148 / cols));
}

// ---------------------------------------------------------------------------------------------
// the table's gradient
// ---------------------------------------------------------------------------------------------

struct TableArgs {
  const int* step;                                // [rows]
  int* begin;                                     // [steps + 1] where a step's rows begin in the list
  int* list;                                      // [rows] rows in the order of their steps, those outside the table in the end
  int* list_step;                                 // [rows] the steps, in the same order (`steps` outside the table)
  const void* dy; const float* factor;            // as in DzArgs
  uint16_t* dz;                                   // as in DzArgs
  float* db_part;                                 // [table_parts][n] column sums, NULL = not wanted
  float* part;                                    // [slices][2][n] sums of runs that cross a slice's begin, its end
  uint16_t* dtable;                               // [steps, n] of the operands' type
  int64_t lddy, ldz;
  int tdy, rows, n, steps, f16;
  int slice;                                      // list entries of a warp of k_table_sum: 32 (one in each lane) at most
  int whole_out;                                  // rows of dtable are whole 16-byte pieces
};

constexpr int kListThreads = 512, kListWarps = kListThreads / 32;

// One CTA per step, and one for rows outside the table: how many rows have smaller steps, then its own rows in ascending order, a warp for
// every sixteenth of the rows. Every CTA reads all of `step`, twice, from L2 and L1: 250 steps over 8192 rows are 8 MB (8.6 us alone: a
// few waits for memory one behind the other).
__global__ void __launch_bounds__(kListThreads) k_table_list(const TableArgs a) {
  __shared__ int less[kListWarps], same[kListWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, s = blockIdx.x;
  const int64_t share = ((int64_t)a.rows + kListThreads - 1) / kListThreads * 32;
  const int64_t r0 = warp * share, r1 = min((int64_t)a.rows, r0 + share);
  constexpr int kAhead = 8;
  start_behind_prior_kernel();
  const auto step_at = [&](int64_t r) {           // -1 behind the last row
    if (r >= r1) return -1;
    const int v = a.step[r];
    return v >= 0 && v < a.steps ? v : a.steps;
  };
  int nless = 0, nsame = 0;
  for (int64_t r = r0 + lane; r < r1; r += 32 * kAhead) {
    int v[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) v[i] = step_at(r + 32 * i);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      nless += v[i] >= 0 && v[i] < s;
      nsame += v[i] == s;
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    nless += __shfl_xor_sync(0xffffffffu, nless, o);
    nsame += __shfl_xor_sync(0xffffffffu, nsame, o);
  }
  if (lane == 0) { less[warp] = nless; same[warp] = nsame; }
  __syncthreads();
  int base = 0, at = 0;
  for (int w = 0; w < kListWarps; ++w) {
    base += less[w];
    if (w < warp) at += same[w];
  }
  if (threadIdx.x == 0) a.begin[s] = base;
  if (nsame == 0) return;
  at += base;
  for (int64_t r = r0; r < r1; r += 32 * kAhead) {
    int v[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) v[i] = step_at(r + 32 * i + lane);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const uint32_t votes = __ballot_sync(0xffffffffu, v[i] == s);
      if (v[i] == s) {
        const int to = at + __popc(votes & ((1u << lane) - 1u));
        a.list[to] = (int)(r + 32 * i + lane);
        a.list_step[to] = s;
      }
      at += __popc(votes);
    }
  }
}

constexpr int kTableThreads = 128, kTableWarps = kTableThreads / 32;

// The same pass as k_linear_dz with the rows in the order of the list (dy and its factors are read once for all three results). A warp
// adds the rows of a slice over 256 columns, four rows requested ahead. A run of one step that begins and ends in the slice
// is a finished row of the gradient; the others are parts for k_table_join. 8192 x 2048 bf16, 250 steps: 30 us alone (101 MB read, 34
// written, 4.5 TB/s: rows in the list's order are short requests), against 16.5 and a pass of its own over dz.
template <bool F32, bool WHOLE>
__global__ void __launch_bounds__(kTableThreads) k_table_sum(const TableArgs a) {
  __shared__ float sums[kTableWarps][256];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int cols = (a.n + 255) / 256, strip = (int)(blockIdx.x % cols), part = (int)(blockIdx.x / cols);   // (parts may pass 65535)
  const int64_t sl = (int64_t)part * kTableWarps + warp;
  const int total = a.rows, i0 = (int)min((int64_t)total, sl * a.slice), count = min(a.slice, total - i0);   // (0: behind the last row)
  start_behind_prior_kernel();
  const int c0 = strip * 256 + lane * 8;
  const bool live = c0 < a.n;
  const int my_row = lane < count ? a.list[i0 + lane] : 0, my_step = lane < count ? a.list_step[i0 + lane] : -1;
  const int step_before = i0 > 0 ? a.list_step[i0 - 1] : -1, step_after = i0 + count < total ? a.list_step[i0 + count] : -1;
  float sum[8] = {}, all[8] = {};
  const auto flush = [&](int s, bool whole) {     // the run of step s that ends here
#pragma unroll
    for (int u = 0; u < 8; ++u) all[u] += sum[u];
    if (s == a.steps || !live) {                  // outside the table
    } else if (whole) {
      uint16_t* out = a.dtable + (size_t)s * a.n + c0;
      if (a.whole_out) {
        *reinterpret_cast<uint4*>(out) = make_uint4(pack16(sum[0], sum[1], a.f16), pack16(sum[2], sum[3], a.f16),
                                                    pack16(sum[4], sum[5], a.f16), pack16(sum[6], sum[7], a.f16));
      } else {
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (c0 + u < a.n) out[u] = round16(sum[u], a.f16);
      }
    } else {
      float* out = a.part + ((size_t)sl * 2 + (s == step_before ? 0 : 1)) * a.ldz + c0;
      *reinterpret_cast<float4*>(out) = make_float4(sum[0], sum[1], sum[2], sum[3]);
      *reinterpret_cast<float4*>(out + 4) = make_float4(sum[4], sum[5], sum[6], sum[7]);
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) sum[u] = 0.f;
  };
  constexpr int kAhead = 4;
  DzRow<F32, WHOLE> ahead[kAhead];
  int step = __shfl_sync(0xffffffffu, my_step, 0);
#pragma unroll
  for (int k = 0; k < kAhead; ++k) {
    const int row = __shfl_sync(0xffffffffu, my_row, k);
    if (live && k < count) dz_request(ahead[k], a, row, c0);
  }
  for (int i = 0; i < count; i += kAhead) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (i + k >= count) break;
      const int s = __shfl_sync(0xffffffffu, my_step, i + k), row = __shfl_sync(0xffffffffu, my_row, i + k);
      const int next = __shfl_sync(0xffffffffu, my_row, (i + k + kAhead) & 31);
      if (s != step) {
        flush(step, step != step_before);
        step = s;
      }
      if (live) {
        float v[8];
        dz_values(ahead[k], a, row, c0, v);
        if (s == a.steps) no_row(v);
        if (i + k + kAhead < count) dz_request(ahead[k], a, next, c0);
#pragma unroll
        for (int u = 0; u < 8; ++u) sum[u] += v[u];
        if (a.dz) dz_store(a, row, c0, v);
      }
    }
  }
  if (count > 0) flush(step, step != step_before && step != step_after);
  if (!a.db_part) return;
  *reinterpret_cast<float4*>(&sums[warp][lane * 8]) = make_float4(all[0], all[1], all[2], all[3]);
  *reinterpret_cast<float4*>(&sums[warp][lane * 8 + 4]) = make_float4(all[4], all[5], all[6], all[7]);
  __syncthreads();
#pragma unroll
  for (int u = 0; u < 256 / kTableThreads; ++u) {
    const int x = threadIdx.x + u * kTableThreads, c = strip * 256 + x;
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kTableWarps; ++w) t += sums[w][x];
    if (c < a.n) a.db_part[(size_t)part * a.n + c] = t;
  }
}

// The sums of a run that crosses slices, and zeros for a step without rows. A CTA takes one step and 256 / W columns, a warp of W for
// the same columns every W-th slice: W = 1 where there are CTAs enough, else 8 (few steps have long runs).
template <int W>
__global__ void __launch_bounds__(256) k_table_join(const TableArgs a) {
  __shared__ float sums[W][256 / W];
  const int s = blockIdx.y, x = threadIdx.x % (256 / W), w = threadIdx.x / (256 / W), c = blockIdx.x * (256 / W) + x;
  start_behind_prior_kernel();
  const int from = a.begin[s], end = a.begin[s + 1];
  const int first = from / a.slice, last = (end - 1) / a.slice;
  if (from < end && first == last) return;        // written by the slice's warp
  float sum = 0.f;
  if (from < end && c < a.n) {
    if (w == 0) sum = a.part[((size_t)first * 2 + 1) * a.ldz + c];
#pragma unroll 8
    for (int i = first + 1 + w; i <= last; i += W) sum += a.part[(size_t)i * 2 * a.ldz + c];
  }
  if (W > 1) {
    sums[w][x] = sum;
    __syncthreads();
    if (w > 0) return;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) sum += sums[i][x];
  }
  if (c < a.n) a.dtable[(size_t)s * a.n + c] = round16(sum, a.f16);
}

// Entries of a slice: as many as leave 24 warps for every SM, between 8 and 32 (a warp's rows wait for memory one behind the other).
int table_slice(int64_t rows, int32_t n) {
  const int64_t cols = (n + 255) / 256;
  int s = 32;
  while (s > 8 && rows * cols < (int64_t)s * 24 * 148) s /= 2;
  return s;
}
int64_t table_slices(int64_t rows, int32_t n) { return (rows + table_slice(rows, n) - 1) / table_slice(rows, n); }
int64_t table_parts(int64_t rows, int32_t n) { return (table_slices(rows, n) + kTableWarps - 1) / kTableWarps; }

inline size_t round_up(size_t v, size_t to) { return (v + to - 1) / to * to; }
inline bool whole(const void* p, int64_t ld, size_t bytes) {      // rows of whole 16-byte pieces
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (size_t)ld * bytes % 16 == 0;
}

// us that tiles take: single CTAs on 128 x 128 (0.15 a step of K, 0.18 where they fill the chip), pairs on 256 x 256
// above one tile an SM, and 5 to 7.5 for the launch, the first loads and the last epilogue.
double tiles_time(int64_t small, int64_t wide, int nkb) {
  if (small <= 148) return 5.2 + nkb * (0.15 + 0.03 * (double)small / 148.0);
  return 7.5 + (double)((wide + 73) / 74) * nkb * 0.27;
}

// The form of a product of `rows` tokens and N output columns: the few-row form's CTAs along K and tokens of a block, or tiles (splits = 0).
// Up to 64 tokens half a tile of rows would be empty: always the few-row form. Above, the shorter estimate: a step of K takes the few-row
// form 0.27 us while each CTA has an SM of its own (three stages of its half of the SM's memory are in flight), 0.39 and a later start where
// two share one; clusters of eight fill no more than 96 SMs singly. 256 x 2048 x 2048: tiles 10.0 us, four CTAs along K 8.8, eight 12.4;
// 512 x 1024 x 4096 tiles 8.2, one CTA 13.0; 256 x 8192 x 640 tiles 23.5, eight 11.2; 512 x 8192 x 2048 24.3, two 24.6, four 22.4.
// `floats`: a float result, whose sums may not be longer than a CTA's accumulators take (kFewRowSteps each): more CTAs along K, or smaller
// blocks of tokens, which have more accumulators (128 x 65536 x 512: 48 us in blocks of 32, 238 as tiles), or tiles.
struct LinearForm { int splits, tokens; };
LinearForm linear_form(int64_t rows, int N, int nkb, bool floats = false) {
  const int64_t tiles = (N + 127) / 128, small = (rows + 127) / 128 * tiles;
  const auto fits = [&](int s, int bn) { return !floats || (nkb + s - 1) / s <= split_accumulators(bn, kLinear) * kFewRowSteps; };
  if (rows <= 64) {
    for (int bn = split_tokens((int)rows); bn >= 16; bn /= 2) {
      int s = split_count((int)rows, (int)tiles, nkb);
      while (s < 8 && !fits(s, bn)) s *= 2;
      if (fits(s, bn)) return {s, bn};
    }
    return {0, 0};
  }
  double least = tiles_time(small, tiles_of(rows, N, 256, 256), nkb);
  LinearForm best{0, 0};
  for (int bn = 128; bn >= 16; bn /= 2) {
    const int64_t tok = (rows + bn - 1) / bn;
    if (tok > 65535) break;                       // (blocks of tokens are the grid's second dimension)
    for (int s = 1; s <= 8; s *= 2) {
      if (s > 1 && nkb / s < 4) break;
      if (!fits(s, bn)) continue;
      const int64_t ctas = tiles * tok * s;
      const int len = (nkb + s - 1) / s;
      const double time = ctas > (s == 8 ? 96 : 148) ? 9.5 + (double)((ctas + 295) / 296) * len * 0.39 : 6.5 + len * 0.27;
      if (time < least) { least = time; best = {s, bn}; }
    }
    if (fits(8, bn)) break;                       // (smaller blocks read the weights more often)
  }
  return best;
}

// Parts into which dW's contraction over the rows is cut (see gradient_parts of the feed-forward block).
int linear_parts(int64_t rows, int32_t k, int32_t n) {
  const bool dx_tiles = linear_form(rows, k, steps(n)).splits == 0;
  const int kr = steps((int)rows), kx = dx_tiles ? steps(n) : 0;
  const int64_t small = tiles_of(n, k, 128, 128), wide = tiles_of(n, k, 256, 256);
  const int64_t xs = dx_tiles ? tiles_of(rows, k, 128, 128) : 0, xw = dx_tiles ? tiles_of(rows, k, 256, 256) : 0;
  const auto time = [&](int parts) {
    const int len = (kr + parts - 1) / parts;
    const double join = parts > 1 ? 4.0 + (double)parts * k * n * 8.0 / 4e6 : 0.0;
    if (xs + small * parts <= 148) return 5.2 + 0.18 * std::max(kx, len) + join;
    const double full = ((double)xw * kx + (double)wide * parts * len) / 74.0;
    return 7.5 + 0.27 * std::max(full + 0.5 * std::min(kx ? kx : len, len), (double)std::max(kx, len)) + join;
  };
  int best = 1;
  double least = time(1);
  for (int parts = 2; parts <= 64 && kr / parts >= 4; ++parts)
    if (time(parts) < least) { least = time(parts); best = parts; }
  return best;
}

size_t part_floats(int64_t m, int64_t n, int parts) {
  return parts > 1 ? round_up((size_t)m, 32) * round_up((size_t)n, 32) * (size_t)parts : 0;
}

}  // namespace

cudaError_t linear_gave_up(int* role, cudaStream_t st) {
  *role = 0;
  const int none = 0;
  cudaError_t e = cudaMemcpyFromSymbolAsync(role, gave_up_word, sizeof(int), 0, cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess || *role == 0) return e;
  e = cudaMemcpyToSymbolAsync(gave_up_word, &none, sizeof(int), 0, cudaMemcpyHostToDevice, st);
  return e == cudaSuccess ? cudaStreamSynchronize(st) : e;
}

size_t linear_factor_bytes(int64_t rows, int32_t n) { return (size_t)rows * round_up(n, 8) * 4; }

LinearWorkspace linear_workspace(int64_t rows, int32_t k, int32_t n, int32_t nsteps, bool has_table) {
  LinearWorkspace w{};
  size_t at = 256;                                // the status word
  const auto take = [&](size_t bytes) { const size_t o = at; at = round_up(at + bytes, 256); return o; };
  w.dz = take((size_t)rows * round_up(n, 8) * 2);
  w.db = take(rows > 0 ? (size_t)std::max<int64_t>(dz_chunks(rows, n), has_table ? table_parts(rows, n) : 0) * n * 4 : 0);
  w.dw = take(rows > 0 ? part_floats(n, k, linear_parts(rows, k, n)) * 4 : 0);
  w.begin = take(has_table ? ((size_t)nsteps + 1) * 4 : 0);
  w.list = take(has_table ? (size_t)rows * 8 : 0);
  w.table = take(has_table ? (size_t)table_slices(rows, n) * 2 * round_up(n, 8) * 4 : 0);
  w.bytes = at;
  return w;
}

namespace {

template <int EPI>
cudaError_t forward(const LinearArgs& a, const FfnArgs& f, const LinearEpilogue& e, cudaStream_t st) {
  const LinearForm form = linear_form(a.rows, a.n, steps(a.k), a.ty == SDS_F32);
  if (form.splits > 0) {
    SplitSpec s{};
    s.w[0] = {a.w, a.k}; s.t[0] = {a.x, a.ldx};
    s.nseg = 1; s.N = a.n; s.K = a.k; s.out = a.y; s.ldo = a.ldy;
    return launch_split<EPI>(f, s, nullptr, true, st, &e, form.splits, form.tokens);
  }
  ProductSpec s{};
  s.a[0] = {a.x, a.ldx}; s.b[0] = {a.w, a.k};
  s.nseg = 1; s.M = a.rows; s.N = a.n; s.K = a.k; s.out = a.y; s.ldo = a.ldy;
  // The epilogue has more to do than the feed-forward block's: eight warps. Four and eight: 8192 x 2048 x 2048 with SiLU, bias and table
  // 59.1 and 56.7 us, with GELU 70.5 and 57.7, 1037 x 1000 x 2731 with GELU 30.2 and 23.9; 16384 x 8192 x 2048 354.9 and 357.7, with
  // bias and GELU 378.8 and 373.5.
  if (a.ty == SDS_F32 && steps(a.k) > kSumSteps) return launch_tiles<EPI, false, false, 16, true>(f, &s, 1, true, st, nullptr, nullptr, false, &e);
  return launch_tiles<EPI, false, false, 8>(f, &s, 1, true, st, nullptr, nullptr, false, &e);
}

}  // namespace

cudaError_t launch_linear(const LinearArgs& a, cudaStream_t st) {
  if (a.rows <= 0) return cudaMemsetAsync(a.err, 0, sizeof(int), st);
  LinearEpilogue e{};
  e.bias = a.bias; e.tbias = a.tbias;
  e.table = static_cast<const uint16_t*>(a.table); e.step = a.step; e.steps = a.steps;
  e.residual = a.residual; e.ldr = a.ldr;
  e.ty = a.ty;
  e.factor = a.act == SDS_ACT_NONE ? nullptr : a.factor;
  e.ldf = (int64_t)round_up(a.n, 8);
  const size_t size = a.ty == SDS_F32 ? 4 : 2;
  const bool wide = a.n % 8 == 0 && whole(a.y, a.ldy, size) && (!a.residual || whole(a.residual, a.ldr, size)) &&
                    (!a.table || whole(a.table, a.n, 2));
  FfnArgs f{};
  f.rows = a.rows; f.f16 = a.f16; f.act = a.act; f.err = a.err;
  return wide ? forward<kLinear>(a, f, e, st) : forward<kLinearNarrow>(a, f, e, st);
}

namespace {

template <class K, class... Args>
cudaError_t start(K kernel, dim3 grid, int threads, int cluster_y, cudaStream_t st, const Args&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  launch_attributes(attr, 1);
  attr[0].val.clusterDim.y = (unsigned)cluster_y;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

cudaError_t launch_dz(const DzArgs& d, bool whole_dy, int chunks, cudaStream_t st) {
  const dim3 grid((d.n + kDzCols - 1) / kDzCols, chunks);
  const auto go = [&](auto kernel) { return start(kernel, grid, kDzThreads, d.cluster, st, d); };
  if (d.tdy == SDS_F32) return whole_dy ? go(k_linear_dz<true, true>) : go(k_linear_dz<true, false>);
  return whole_dy ? go(k_linear_dz<false, true>) : go(k_linear_dz<false, false>);
}

cudaError_t launch_join(const float* part, uint16_t* out, int M, int N, int parts, int f16, cudaStream_t st) {
  FfnJoinArgs join{};
  join.np = 1; join.parts = parts; join.f16 = f16;
  join.p[0].part = part; join.p[0].out = out; join.p[0].M = M; join.p[0].N = N;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)((int64_t)((M + 31) / 32) * ((N + 31) / 32)));
  cfg.blockDim = dim3(kJoinThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  launch_attributes(attr, 1);
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, k_ffn_join, join);
}

cudaError_t launch_table(const TableArgs& t, bool whole_dy, cudaStream_t st) {
  cudaError_t e = start(k_table_list, dim3(t.steps + 1), kListThreads, 1, st, t);
  if (e != cudaSuccess) return e;
  const int cols = (t.n + 255) / 256;
  const dim3 grid((unsigned)(cols * table_parts(t.rows, t.n)));
  const auto go = [&](auto kernel) { return start(kernel, grid, kTableThreads, 1, st, t); };
  if (t.tdy == SDS_F32) e = whole_dy ? go(k_table_sum<true, true>) : go(k_table_sum<true, false>);
  else e = whole_dy ? go(k_table_sum<false, true>) : go(k_table_sum<false, false>);
  if (e != cudaSuccess) return e;
  return (int64_t)cols * t.steps >= 4 * 148 ? start(k_table_join<1>, dim3(cols, t.steps), 256, 1, st, t)
                                            : start(k_table_join<8>, dim3((t.n + 31) / 32, t.steps), 256, 1, st, t);
}

}  // namespace

cudaError_t launch_linear_backward(const LinearArgs& a, cudaStream_t st) {
  cudaError_t e = cudaSuccess;
  const size_t sb = a.tbias == SDS_F32 ? 4 : 2;
  if (a.rows <= 0) {                              // empty sums: the parameters' gradients are zeros
    if ((e = cudaMemsetAsync(a.err, 0, sizeof(int), st)) != cudaSuccess) return e;
    if (a.dw && (e = cudaMemsetAsync(a.dw, 0, (size_t)a.n * a.k * 2, st)) != cudaSuccess) return e;
    if (a.db && (e = cudaMemsetAsync(a.db, 0, (size_t)a.n * sb, st)) != cudaSuccess) return e;
    if (a.dtable && (e = cudaMemsetAsync(a.dtable, 0, (size_t)a.steps * a.n * 2, st)) != cudaSuccess) return e;
    return cudaSuccess;
  }
  char* ws = reinterpret_cast<char*>(a.err);
  const LinearWorkspace at = linear_workspace(a.rows, a.k, a.n, a.steps, a.dtable != nullptr);
  const float* factor = a.act == SDS_ACT_NONE ? nullptr : a.factor;
  const int64_t ldz = (int64_t)round_up(a.n, 8);
  const size_t sy = a.ty == SDS_F32 ? 4 : 2;
  const bool whole_dy = a.n % 8 == 0 && whole(a.dy, a.lddy, sy);
  const bool products = a.dx || a.dw;
  // without an activation dy itself is the operand, where its rows are ones that the tensor maps take (and none may have to be left out)
  const bool direct = !factor && !a.table && a.ty != SDS_F32 && whole(a.dy, a.lddy, 2);
  uint16_t* to_dz = products && !direct ? reinterpret_cast<uint16_t*>(ws + at.dz) : nullptr;
  float* db_part = reinterpret_cast<float*>(ws + at.db);
  int64_t db_parts = 0;                           // whose sums are still to be added
  if (a.dtable) {
    TableArgs t{};
    t.step = a.step;
    t.begin = reinterpret_cast<int*>(ws + at.begin); t.list = reinterpret_cast<int*>(ws + at.list);
    t.list_step = t.list + a.rows;
    t.part = reinterpret_cast<float*>(ws + at.table);
    t.dy = a.dy; t.lddy = a.lddy; t.tdy = a.ty; t.factor = factor; t.ldz = ldz;
    t.dz = to_dz; t.db_part = a.db ? db_part : nullptr;
    t.dtable = static_cast<uint16_t*>(a.dtable);
    t.rows = a.rows; t.n = a.n; t.steps = a.steps; t.f16 = a.f16;
    t.slice = table_slice(a.rows, a.n);
    t.whole_out = a.n % 8 == 0 && whole(a.dtable, a.n, 2);
    if ((e = launch_table(t, whole_dy, st)) != cudaSuccess) return e;
    db_parts = a.db ? table_parts(a.rows, a.n) : 0;
  } else if (to_dz || a.db) {
    DzArgs d{};
    d.dy = a.dy; d.lddy = a.lddy; d.tdy = a.ty;
    d.factor = factor; d.ldz = ldz; d.f16 = a.f16;
    d.dz = to_dz;
    d.step = a.table ? a.step : nullptr; d.steps = a.steps;
    d.part = db_part; d.db = a.db; d.tdb = a.tbias;
    d.rows = a.rows; d.n = a.n;
    const int chunks = dz_chunks(a.rows, a.n);
    d.cluster = a.db && chunks <= 8 ? chunks : 1;
    if ((e = launch_dz(d, whole_dy, chunks, st)) != cudaSuccess) return e;
    db_parts = a.db && chunks > d.cluster ? chunks : 0;
  }
  if (db_parts > 0 &&
      (e = start(k_linear_db, dim3((a.n + 31) / 32), 256, 1, st, (const float*)db_part, (int)db_parts, a.n, a.db, a.tbias)) != cudaSuccess)
    return e;
  if (!products) return cudaMemsetAsync(a.err, 0, sizeof(int), st);
  const Mat dz = direct ? Mat{a.dy, a.lddy} : Mat{ws + at.dz, ldz};
  FfnArgs f{};
  f.rows = a.rows; f.f16 = a.f16; f.err = a.err;
  ProductSpec w[2];
  int n = 0;
  bool first = true, beside = false;
  const LinearForm dx_form = a.dx ? linear_form(a.rows, a.k, steps(a.n)) : LinearForm{0, 0};
  if (dx_form.splits > 0) {
    SplitSpec s{};
    s.w[0] = {a.w, a.k}; s.t[0] = dz;
    s.nseg = 1; s.w_mn = true; s.N = a.k; s.K = a.n; s.out = a.dx; s.ldo = a.lddx;
    if ((e = launch_split<kFfnOut>(f, s, nullptr, first, st, nullptr, dx_form.splits, dx_form.tokens)) != cudaSuccess) return e;
    first = false;
    beside = true;                                // (dW does not read dx)
  } else if (a.dx) {
    ProductSpec s{};
    s.a[0] = dz; s.b[0] = {a.w, a.k};
    s.nseg = 1; s.M = a.rows; s.N = a.k; s.K = a.n; s.out = a.dx; s.ldo = a.lddx;
    w[n++] = s;
  }
  if (a.dw) {
    ProductSpec s{};
    s.a[0] = dz; s.b[0] = {a.x, a.ldx};
    s.nseg = 1; s.a_mn = true; s.M = a.n; s.N = a.k; s.K = a.rows; s.out = a.dw; s.ldo = a.k;
    s.parts = linear_parts(a.rows, a.k, a.n); s.part = reinterpret_cast<float*>(ws + at.dw);
    w[n++] = s;
  }
  if (n == 0) return cudaSuccess;
  const int parts = a.dw ? linear_parts(a.rows, a.k, a.n) : 1;
  if (parts == 1) return launch_tiles<kFfnOut, true>(f, w, n, first, st, nullptr, nullptr, beside);
  if ((e = launch_tiles<kFfnOut, true, true>(f, w, n, first, st, nullptr, nullptr, beside)) != cudaSuccess) return e;
  return launch_join(reinterpret_cast<float*>(ws + at.dw), static_cast<uint16_t*>(a.dw), a.n, a.k, parts, a.f16, st);
}

}  // namespace sds
