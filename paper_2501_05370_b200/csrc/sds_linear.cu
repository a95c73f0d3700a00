// Linear layer with its epilogue, forward and backward, on the tensor cores.
//
//   forward   z = x W^T + b + table[step], y = act(z) + residual          (x [rows, k], W [n, k])
//   backward  dz = dy act'(z), dx = dz W, dW = dz^T x, db = sum_rows dz, dtable[s] = sum_{rows with step s} dz
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

struct DzArgs {
  const void* dy;                                 // [rows, n] of tdy, rows lddy elements apart
  const float* factor;                            // [rows, ldz], NULL = ones
  uint16_t* dz;                                   // [rows, ldz] of the operands' type, NULL = not wanted
  float* part;                                    // [gridDim.y][n] column sums, NULL = not wanted
  void* db;                                       // with a single chunk of rows the sums go here at once
  int64_t lddy, ldz;
  int tdy, tdb, rows, n, f16;
};

constexpr int kDzThreads = 256, kDzWarps = kDzThreads / 32, kDzCols = 256;

__device__ __forceinline__ void store_typed(void* p, int type, size_t i, float v) {
  if (type == SDS_F32) static_cast<float*>(p)[i] = v;
  else static_cast<uint16_t*>(p)[i] = round16(v, type == SDS_F16);
}

// eight columns of a row of dy and of its factors, as they lie in memory
template <bool F32> struct DzRow { uint4 y[F32 ? 2 : 1], f[2]; };
template <bool F32, class A>
__device__ __forceinline__ void dz_request(DzRow<F32>& r, const A& a, int64_t row, int c0) {
  const char* y = static_cast<const char*>(a.dy) + ((size_t)row * a.lddy + c0) * (F32 ? 4 : 2);
#pragma unroll
  for (int i = 0; i < (F32 ? 2 : 1); ++i) r.y[i] = __ldg(reinterpret_cast<const uint4*>(y) + i);
  if (a.factor)
#pragma unroll
    for (int i = 0; i < 2; ++i) r.f[i] = __ldg(reinterpret_cast<const uint4*>(a.factor + (size_t)row * a.ldz + c0) + i);
}
template <bool F32, class A>
__device__ __forceinline__ void dz_values(const DzRow<F32>& r, const A& a, float (&v)[8]) {
  if (F32) {
    const uint32_t w[8] = {r.y[0].x, r.y[0].y, r.y[0].z, r.y[0].w, r.y[F32].x, r.y[F32].y, r.y[F32].z, r.y[F32].w};
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = __uint_as_float(w[u]);
  } else {
    const uint32_t w[4] = {r.y[0].x, r.y[0].y, r.y[0].z, r.y[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 t = unpack16x2(w[i], a.f16);
      v[2 * i] = t.x; v[2 * i + 1] = t.y;
    }
  }
  if (a.factor) {
    const uint32_t w[8] = {r.f[0].x, r.f[0].y, r.f[0].z, r.f[0].w, r.f[1].x, r.f[1].y, r.f[1].z, r.f[1].w};
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] *= __uint_as_float(w[u]);
  }
}
// the same for columns 32 apart, one by one
template <class A>
__device__ __forceinline__ void dz_scalar(const A& a, int64_t row, int c0, float (&v)[8]) {
  float f[8];
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const int c = c0 + u * 32;
    v[u] = c < a.n ? load_typed(a.dy, a.tdy, (size_t)row * a.lddy + c) : 0.f;
    f[u] = a.factor && c < a.n ? a.factor[(size_t)row * a.ldz + c] : 1.f;
  }
#pragma unroll
  for (int u = 0; u < 8; ++u) v[u] *= f[u];
}

// A lane takes eight columns of every eighth row of its chunk (VEC: neighbours, in 16-byte accesses; else 32 columns apart), four rows
// requested ahead. Bound by memory.
template <bool F32, bool VEC>
__global__ void __launch_bounds__(kDzThreads) k_linear_dz(const DzArgs a) {
  __shared__ float sums[kDzWarps][kDzCols];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c0 = blockIdx.x * kDzCols + (VEC ? lane * 8 : lane);
  float sum[8] = {};
  const int64_t stride = (int64_t)gridDim.y * kDzWarps, first = (int64_t)blockIdx.y * kDzWarps + warp;
  if (VEC && c0 < a.n) {
    constexpr int kAhead = 4;
    DzRow<F32> ahead[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (first + i * stride < a.rows) dz_request(ahead[i], a, first + i * stride, c0);
    for (int64_t base = first; base < a.rows; base += kAhead * stride) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int64_t row = base + i * stride, next = row + kAhead * stride;
        if (row >= a.rows) break;
        float v[8];
        dz_values(ahead[i], a, v);
        if (next < a.rows) dz_request(ahead[i], a, next, c0);
#pragma unroll
        for (int u = 0; u < 8; ++u) sum[u] += v[u];
        if (a.dz)
          *reinterpret_cast<uint4*>(a.dz + (size_t)row * a.ldz + c0) =
              make_uint4(pack16(v[0], v[1], a.f16), pack16(v[2], v[3], a.f16), pack16(v[4], v[5], a.f16), pack16(v[6], v[7], a.f16));
      }
    }
  } else if (!VEC) {
#pragma unroll 2
    for (int64_t row = first; row < a.rows; row += stride) {
      float v[8];
      dz_scalar(a, row, c0, v);
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        sum[u] += v[u];
        if (a.dz && c0 + u * 32 < a.n) a.dz[(size_t)row * a.ldz + c0 + u * 32] = round16(v[u], a.f16);
      }
    }
  }
  if (!a.part) return;
  if (VEC) {
    *reinterpret_cast<float4*>(&sums[warp][lane * 8]) = make_float4(sum[0], sum[1], sum[2], sum[3]);
    *reinterpret_cast<float4*>(&sums[warp][lane * 8 + 4]) = make_float4(sum[4], sum[5], sum[6], sum[7]);
  } else {
#pragma unroll
    for (int u = 0; u < 8; ++u) sums[warp][lane + u * 32] = sum[u];
  }
  __syncthreads();
  const int c = blockIdx.x * kDzCols + threadIdx.x;
  if (c >= a.n) return;
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < kDzWarps; ++w) s += sums[w][threadIdx.x];
  if (gridDim.y == 1) store_typed(a.db, a.tdb, c, s);
  else a.part[(size_t)blockIdx.y * a.n + c] = s;
}

// The chunks' column sums, added in order: 32 columns of a CTA, a warp every eighth chunk.
__global__ void __launch_bounds__(256) k_linear_db(const float* part, int chunks, int n, void* db, int tdb) {
  __shared__ float sums[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (c < n)
#pragma unroll 4
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
  int* list;                                      // [rows] rows in the order of their steps; those outside the table are left out
  int* list_step;                                 // [rows] the steps, in the same order
  const void* dy; const float* factor;            // as in DzArgs
  float* part;                                    // [slices][2][n] sums of runs that cross a slice's begin, its end
  uint16_t* dtable;                               // [steps, n] of the operands' type
  int64_t lddy, ldz;
  int tdy, rows, n, steps, f16;
};

constexpr int kListThreads = 512, kListWarps = kListThreads / 32;
constexpr int kSlice = 32;                        // list entries of a warp of k_table_sum: one in each lane

// One CTA per step: how many rows have smaller steps, then its own rows in ascending order, a warp for every sixteenth of the rows. Every
// CTA reads all of `step`, twice, from L2 and L1: 250 steps over 8192 rows are 8 MB.
__global__ void __launch_bounds__(kListThreads) k_table_list(const TableArgs a) {
  __shared__ int less[kListWarps], same[kListWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, s = blockIdx.x;
  const int64_t share = ((int64_t)a.rows + kListThreads - 1) / kListThreads * 32;
  const int64_t r0 = warp * share, r1 = min((int64_t)a.rows, r0 + share);
  constexpr int kAhead = 8;
  int nless = 0, nsame = 0;
  for (int64_t r = r0 + lane; r < r1; r += 32 * kAhead) {
    int v[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) v[i] = r + 32 * i < r1 ? __ldg(a.step + r + 32 * i) : -1;
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
  int base = 0, at = 0, all = 0;
  for (int w = 0; w < kListWarps; ++w) {
    base += less[w];
    if (w < warp) at += same[w];
    all += same[w];
  }
  if (threadIdx.x == 0) {
    a.begin[s] = base;
    if (s == a.steps - 1) a.begin[a.steps] = base + all;
  }
  if (nsame == 0) return;
  at += base;
  for (int64_t r = r0; r < r1; r += 32 * kAhead) {
    int v[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) v[i] = r + 32 * i + lane < r1 ? __ldg(a.step + r + 32 * i + lane) : -1;
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

// A warp adds the rows of a slice of the list over 256 columns (VEC: eight neighbours per lane), four rows requested ahead. A run of one
// step that begins and ends in the slice is a finished row of the gradient; the others are parts for k_table_join.
template <bool F32, bool VEC>
__global__ void __launch_bounds__(kTableThreads) k_table_sum(const TableArgs a) {
  const int lane = threadIdx.x & 31;
  const int64_t sl = (int64_t)blockIdx.y * kTableWarps + (threadIdx.x >> 5);
  const int total = a.begin[a.steps];
  if (sl * kSlice >= total) return;
  const int i0 = (int)(sl * kSlice), count = min(kSlice, total - i0);
  const int c0 = blockIdx.x * 256 + (VEC ? lane * 8 : lane);
  const bool live = c0 < a.n;
  constexpr int kStep = VEC ? 1 : 32;
  const int my_row = lane < count ? __ldg(a.list + i0 + lane) : 0, my_step = lane < count ? __ldg(a.list_step + i0 + lane) : -1;
  const int step_before = i0 > 0 ? __ldg(a.list_step + i0 - 1) : -1, step_after = i0 + count < total ? __ldg(a.list_step + i0 + count) : -1;
  float sum[8] = {};
  const auto flush = [&](int s, bool whole) {     // the run of step s that ends here
    if (whole) {
      uint16_t* out = a.dtable + (size_t)s * a.n + c0;
      if (VEC) {
        if (live)
          *reinterpret_cast<uint4*>(out) = make_uint4(pack16(sum[0], sum[1], a.f16), pack16(sum[2], sum[3], a.f16),
                                                      pack16(sum[4], sum[5], a.f16), pack16(sum[6], sum[7], a.f16));
      } else {
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (c0 + u * kStep < a.n) out[u * kStep] = round16(sum[u], a.f16);
      }
    } else {
      float* out = a.part + ((size_t)sl * 2 + (s == step_before ? 0 : 1)) * a.n + c0;
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (c0 + u * kStep < a.n) out[u * kStep] = sum[u];
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) sum[u] = 0.f;
  };
  constexpr int kAhead = 4;
  DzRow<F32> ahead[kAhead];
  int first_row[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k) first_row[k] = __shfl_sync(0xffffffffu, my_row, min(k, count - 1));
  if (VEC && live)
#pragma unroll
    for (int k = 0; k < kAhead; ++k) dz_request(ahead[k], a, first_row[k], c0);
  int step = __shfl_sync(0xffffffffu, my_step, 0);
  for (int i = 0; i < kSlice; i += kAhead) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (i + k >= count) break;
      const int s = __shfl_sync(0xffffffffu, my_step, i + k), row = __shfl_sync(0xffffffffu, my_row, i + k);
      const int next = __shfl_sync(0xffffffffu, my_row, min(i + k + kAhead, count - 1));
      if (s != step) {
        flush(step, step != step_before);
        step = s;
      }
      float v[8];
      if (VEC) {
        if (live) {
          dz_values(ahead[k], a, v);
          if (i + k + kAhead < count) dz_request(ahead[k], a, next, c0);
#pragma unroll
          for (int u = 0; u < 8; ++u) sum[u] += v[u];
        }
      } else {
        dz_scalar(a, row, c0, v);
#pragma unroll
        for (int u = 0; u < 8; ++u) sum[u] += v[u];
      }
    }
  }
  flush(step, step != step_before && step != step_after);
}

// The sums of a run that crosses slices, and zeros for a step without rows. A CTA takes one step and 256 / W columns, a warp of W for
// the same columns every W-th slice: W = 1 where there are CTAs enough, else 8 (few steps have long runs).
template <int W>
__global__ void __launch_bounds__(256) k_table_join(const TableArgs a) {
  __shared__ float sums[W][256 / W];
  const int s = blockIdx.y, x = threadIdx.x % (256 / W), w = threadIdx.x / (256 / W), c = blockIdx.x * (256 / W) + x;
  const int from = a.begin[s], end = a.begin[s + 1];
  const int first = from / kSlice, last = (end - 1) / kSlice;
  if (from < end && first == last) return;        // written by the slice's warp
  float sum = 0.f;
  if (from < end && c < a.n) {
    if (w == 0) sum = a.part[((size_t)first * 2 + 1) * a.n + c];
#pragma unroll 8
    for (int i = first + 1 + w; i <= last; i += W) sum += a.part[(size_t)i * 2 * a.n + c];
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

int64_t table_slices(int64_t rows) { return (rows + kSlice - 1) / kSlice; }

inline size_t round_up(size_t v, size_t to) { return (v + to - 1) / to * to; }
inline bool whole(const void* p, int64_t ld, size_t bytes) {      // rows of whole 16-byte pieces
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (size_t)ld * bytes % 16 == 0;
}

// Parts into which dW's contraction over the rows is cut (see gradient_parts of the feed-forward block).
int linear_parts(int64_t rows, int32_t k, int32_t n) {
  const bool dx_tiles = !prefer_split<kFfnOut>((int)rows, k, steps(n));
  const int kr = steps((int)rows), kx = dx_tiles ? steps(n) : 0;
  const int64_t small = tiles_of(n, k, 128, 128), wide = tiles_of(n, k, 256, 256);
  const int64_t xs = dx_tiles ? tiles_of(rows, k, 128, 128) : 0, xw = dx_tiles ? tiles_of(rows, k, 256, 256) : 0;
  const auto time = [&](int parts) {
    const int len = (kr + parts - 1) / parts;
    const double join = parts > 1 ? 4.0 + (double)parts * k * n * 8.0 / 4e6 : 0.0;
    if (xs + small * parts <= 148) return 0.35 * std::max(kx, len) + 2.0 + join;
    const double full = ((double)xw * kx + (double)wide * parts * len) / 74.0;
    return 0.3 * std::max(full + 0.5 * std::min(kx ? kx : len, len), (double)std::max(kx, len)) + 4.0 + join;
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
  w.db = take(rows > 0 ? (size_t)dz_chunks(rows, n) * n * 4 : 0);
  w.dw = take(rows > 0 ? part_floats(n, k, linear_parts(rows, k, n)) * 4 : 0);
  w.begin = take(has_table ? ((size_t)nsteps + 1) * 4 : 0);
  w.list = take(has_table ? (size_t)rows * 8 : 0);
  w.table = take(has_table ? (size_t)table_slices(rows) * 2 * n * 4 : 0);
  w.bytes = at;
  return w;
}

namespace {

template <int EPI>
cudaError_t forward(const LinearArgs& a, const FfnArgs& f, const LinearEpilogue& e, cudaStream_t st) {
  if (prefer_split<EPI>(a.rows, a.n, steps(a.k))) {
    SplitSpec s{};
    s.w[0] = {a.w, a.k}; s.t[0] = {a.x, a.ldx};
    s.nseg = 1; s.N = a.n; s.K = a.k; s.out = a.y; s.ldo = a.ldy;
    return launch_split<EPI>(f, s, nullptr, true, st, &e);
  }
  ProductSpec s{};
  s.a[0] = {a.x, a.ldx}; s.b[0] = {a.w, a.k};
  s.nseg = 1; s.M = a.rows; s.N = a.n; s.K = a.k; s.out = a.y; s.ldo = a.ldy;
  // The epilogue has more to do than the feed-forward block's, and a tile of few steps ends sooner: eight warps up to 64 steps of K,
  // four beyond. Four and eight: 8192 x 2048 x 2048 with SiLU, bias and table 75.8 and 68.5 us, with GELU 87.6 and 72.2, 1037 x 1000 x 2731
  // with GELU 30.9 and 25.6; 16384 x 8192 x 2048 392 and 405, with a float residual 474 and 486.
  if (steps(a.k) <= 64) return launch_tiles<EPI, false, false, 8>(f, &s, 1, true, st, nullptr, nullptr, false, &e);
  return launch_tiles<EPI, false>(f, &s, 1, true, st, nullptr, nullptr, false, &e);
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

cudaError_t launch_dz(const DzArgs& d, bool vec, int chunks, cudaStream_t st) {
  const dim3 grid((d.n + kDzCols - 1) / kDzCols, chunks);
  if (d.tdy == SDS_F32) {
    if (vec) k_linear_dz<true, true><<<grid, kDzThreads, 0, st>>>(d);
    else k_linear_dz<true, false><<<grid, kDzThreads, 0, st>>>(d);
  } else {
    if (vec) k_linear_dz<false, true><<<grid, kDzThreads, 0, st>>>(d);
    else k_linear_dz<false, false><<<grid, kDzThreads, 0, st>>>(d);
  }
  return cudaGetLastError();
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

cudaError_t launch_table(const TableArgs& t, bool vec, cudaStream_t st) {
  k_table_list<<<t.steps, kListThreads, 0, st>>>(t);
  const int cols = (t.n + 255) / 256;
  const dim3 grid(cols, (unsigned)((table_slices(t.rows) + kTableWarps - 1) / kTableWarps));
  if (t.tdy == SDS_F32) {
    if (vec) k_table_sum<true, true><<<grid, kTableThreads, 0, st>>>(t);
    else k_table_sum<true, false><<<grid, kTableThreads, 0, st>>>(t);
  } else {
    if (vec) k_table_sum<false, true><<<grid, kTableThreads, 0, st>>>(t);
    else k_table_sum<false, false><<<grid, kTableThreads, 0, st>>>(t);
  }
  if ((int64_t)cols * t.steps >= 4 * 148) k_table_join<1><<<dim3(cols, t.steps), 256, 0, st>>>(t);
  else k_table_join<8><<<dim3((t.n + 31) / 32, t.steps), 256, 0, st>>>(t);
  return cudaGetLastError();
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
  const bool vec = a.n % 8 == 0 && whole(a.dy, a.lddy, sy);
  const bool products = a.dx || a.dw;
  // without an activation dy itself is the operand, where its rows are ones that the tensor maps take
  const bool direct = !factor && a.ty != SDS_F32 && whole(a.dy, a.lddy, 2);
  if ((products && !direct) || a.db) {
    DzArgs d{};
    d.dy = a.dy; d.lddy = a.lddy; d.tdy = a.ty;
    d.factor = factor; d.ldz = ldz; d.f16 = a.f16;
    d.dz = products && !direct ? reinterpret_cast<uint16_t*>(ws + at.dz) : nullptr;
    d.part = a.db ? reinterpret_cast<float*>(ws + at.db) : nullptr;
    d.db = a.db; d.tdb = a.tbias;
    d.rows = a.rows; d.n = a.n;
    const int chunks = dz_chunks(a.rows, a.n);
    if ((e = launch_dz(d, vec, chunks, st)) != cudaSuccess) return e;
    if (a.db && chunks > 1) {
      k_linear_db<<<(a.n + 31) / 32, 256, 0, st>>>(d.part, chunks, a.n, a.db, a.tbias);
      if ((e = cudaGetLastError()) != cudaSuccess) return e;
    }
  }
  if (a.dtable) {
    TableArgs t{};
    t.step = a.step;
    t.begin = reinterpret_cast<int*>(ws + at.begin); t.list = reinterpret_cast<int*>(ws + at.list);
    t.list_step = t.list + a.rows;
    t.part = reinterpret_cast<float*>(ws + at.table);
    t.dy = a.dy; t.lddy = a.lddy; t.tdy = a.ty; t.factor = factor; t.ldz = ldz;
    t.dtable = static_cast<uint16_t*>(a.dtable);
    t.rows = a.rows; t.n = a.n; t.steps = a.steps; t.f16 = a.f16;
    if ((e = launch_table(t, vec, st)) != cudaSuccess) return e;
  }
  if (!products) return cudaMemsetAsync(a.err, 0, sizeof(int), st);
  const Mat dz = direct ? Mat{a.dy, a.lddy} : Mat{ws + at.dz, ldz};
  FfnArgs f{};
  f.rows = a.rows; f.f16 = a.f16; f.err = a.err;
  ProductSpec w[2];
  int n = 0;
  bool first = true, beside = false;
  if (a.dx && prefer_split<kFfnOut>(a.rows, a.k, steps(a.n))) {
    SplitSpec s{};
    s.w[0] = {a.w, a.k}; s.t[0] = dz;
    s.nseg = 1; s.w_mn = true; s.N = a.k; s.K = a.n; s.out = a.dx; s.ldo = a.lddx;
    if ((e = launch_split<kFfnOut>(f, s, nullptr, first, st)) != cudaSuccess) return e;
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
