// Linear layer with its epilogue, forward and backward, on the tensor cores.
//
//   forward   z = x W^T + b + table[step], y = act(z) + residual          (x [rows, k], W [n, k])
//   backward  dz = dy act'(z), dx = dz W, dW = dz^T x, db = sum_rows dz, dtable[s] = sum_{rows with step s} dz
//
// The products are those of sds_tiles.cuh: persistent tiles for batches, weights split over clusters for few rows. Bias, table
// rows, activation and residual are applied to the accumulator, before its one rounding, so y is written once and z never.
// For the backward pass the forward one keeps act'(z) as f16 (2 bytes per output): its values lie in [-0.2, 1.2], so that
// the rounding is at most 2^-11 relative, against 2^-8 of dz as a bf16 operand of the products that follow (f16: the same size).
// Keeping z itself would take as many bytes and the activation again; keeping a float would make a training step of
// small k wait for memory.
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
  const uint16_t* factor;                         // [rows, ldz] f16, NULL = ones
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

// A lane takes eight columns of every eighth row of its chunk (VEC: neighbours, in 16-byte accesses; else 32 columns apart).
// Memory bound: 8192 x 2048 bf16 with its factors.
template <bool F32, bool VEC>
__global__ void __launch_bounds__(kDzThreads) k_linear_dz(const DzArgs a) {
  __shared__ float sums[kDzWarps][kDzCols];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c0 = blockIdx.x * kDzCols + (VEC ? lane * 8 : lane);
  constexpr int kStep = VEC ? 1 : 32;             // between a lane's columns
  float sum[8] = {};
  const int stride = (int)gridDim.y * kDzWarps;
  const auto load = [&](int row, float (&v)[8], float (&f)[8]) {
    if (VEC) {
      const bool in = c0 < a.n;
      if (F32) {
        const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(a.dy) + (size_t)row * a.lddy + c0);
        const float4 lo = in ? __ldg(p) : make_float4(0.f, 0.f, 0.f, 0.f), hi = in ? __ldg(p + 1) : make_float4(0.f, 0.f, 0.f, 0.f);
        v[0] = lo.x; v[1] = lo.y; v[2] = lo.z; v[3] = lo.w; v[4] = hi.x; v[5] = hi.y; v[6] = hi.z; v[7] = hi.w;
      } else {
        const uint4 w = in ? __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.dy) + (size_t)row * a.lddy + c0))
                           : make_uint4(0u, 0u, 0u, 0u);
        const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 t = unpack16x2(q[i], a.f16);
          v[2 * i] = t.x; v[2 * i + 1] = t.y;
        }
      }
      if (a.factor) {
        const uint4 w = in ? __ldg(reinterpret_cast<const uint4*>(a.factor + (size_t)row * a.ldz + c0)) : make_uint4(0u, 0u, 0u, 0u);
        const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 t = unpack16x2(q[i], 1);
          f[2 * i] = t.x; f[2 * i + 1] = t.y;
        }
      }
    } else {
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int c = c0 + u * kStep;
        v[u] = c < a.n ? load_typed(a.dy, a.tdy, (size_t)row * a.lddy + c) : 0.f;
        if (a.factor) f[u] = c < a.n ? unpack16(a.factor[(size_t)row * a.ldz + c], 1) : 0.f;
      }
    }
  };
  const auto take = [&](int row, float (&v)[8], const float (&f)[8]) {
    if (a.factor)
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] *= f[u];
#pragma unroll
    for (int u = 0; u < 8; ++u) sum[u] += v[u];
    if (!a.dz) return;
    if (VEC) {
      if (c0 < a.n)
        *reinterpret_cast<uint4*>(a.dz + (size_t)row * a.ldz + c0) =
            make_uint4(pack16(v[0], v[1], a.f16), pack16(v[2], v[3], a.f16), pack16(v[4], v[5], a.f16), pack16(v[6], v[7], a.f16));
    } else {
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (c0 + u * kStep < a.n) a.dz[(size_t)row * a.ldz + c0 + u * kStep] = round16(v[u], a.f16);
    }
  };
  constexpr int kAhead = 4;                       // rows requested before the first is used
  for (int row = blockIdx.y * kDzWarps + warp; row < a.rows;) {
    float v[kAhead][8], f[kAhead][8];
    if (row <= a.rows - 1 - (kAhead - 1) * stride) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) load(row + i * stride, v[i], f[i]);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) take(row + i * stride, v[i], f[i]);
      if (row > a.rows - 1 - kAhead * stride) break;              // (before the sum below could pass 2^31)
      row += kAhead * stride;
    } else {
      load(row, v[0], f[0]);
      take(row, v[0], f[0]);
      if (row > a.rows - 1 - stride) break;
      row += stride;
    }
  }
  if (!a.part) return;
#pragma unroll
  for (int u = 0; u < 8; ++u) sums[warp][VEC ? lane * 8 + u : lane + u * 32] = sum[u];
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

// Chunks of rows: four rows for every warp, until there are eight CTAs for each SM.
int dz_chunks(int64_t rows, int32_t n) {
  const int64_t cols = (n + kDzCols - 1) / kDzCols;
  return (int)std::max<int64_t>(1, std::min<int64_t>((rows + 4 * kDzWarps - 1) / (4 * kDzWarps), (8 * 148 + cols - 1) / cols));
}

// ---------------------------------------------------------------------------------------------
// the table's gradient
// ---------------------------------------------------------------------------------------------

struct TableArgs {
  const int* step;                                // [rows]
  int* begin;                                     // [steps + 1] where a step's rows begin in the list
  int* list;                                      // [rows] rows in the order of their steps; those outside the table are left out
  const void* dy; const uint16_t* factor;         // as in DzArgs
  float* part;                                    // [slices][2][n] sums of runs that cross a slice's begin, its end
  uint16_t* dtable;                               // [steps, n] of the operands' type
  int64_t lddy, ldz;
  int tdy, rows, n, steps, f16;
  int slice, slices;                              // list entries of a warp; warps' worth of the longest list
};

constexpr int kListThreads = 256;

// One CTA per step: how many rows have smaller steps, then its own rows in ascending order. Every CTA reads all of `step`,
// twice, from L2: 250 steps over 8192 rows are 16 MB.
__global__ void __launch_bounds__(kListThreads) k_table_list(const TableArgs a) {
  __shared__ int below[kListThreads / 32], counts[kListThreads / 32];
  __shared__ int base;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, s = blockIdx.x;
  int less = 0;
  for (int64_t r = threadIdx.x; r < a.rows; r += kListThreads) {
    const int v = __ldg(a.step + r);
    less += v >= 0 && v < s;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) less += __shfl_xor_sync(0xffffffffu, less, o);
  if (lane == 0) below[warp] = less;
  __syncthreads();
  if (threadIdx.x == 0) {
    int t = 0;
    for (int w = 0; w < kListThreads / 32; ++w) t += below[w];
    base = t;
    a.begin[s] = t;
  }
  __syncthreads();
  int at = base;
  for (int64_t r0 = 0; r0 < a.rows; r0 += kListThreads) {
    const int64_t r = r0 + threadIdx.x;
    const bool mine = r < a.rows && __ldg(a.step + r) == s;
    const uint32_t votes = __ballot_sync(0xffffffffu, mine);
    if (lane == 0) counts[warp] = __popc(votes);
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kListThreads / 32; ++w) {
      if (w < warp) before += counts[w];
      all += counts[w];
    }
    if (mine) a.list[at + before + __popc(votes & ((1u << lane) - 1u))] = (int)r;
    at += all;
    __syncthreads();
  }
  if (s == a.steps - 1 && threadIdx.x == 0) a.begin[a.steps] = at;
}

// the last step that begins at or before entry i of the list (i < its length, so that step has rows)
__device__ __forceinline__ int step_of(const int* begin, int steps, int i) {
  int lo = 0, hi = steps;                         // begin[lo] <= i < begin[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (begin[mid] <= i) lo = mid; else hi = mid;
  }
  return lo;
}

constexpr int kTableThreads = 128, kTableWarps = kTableThreads / 32;

// A warp adds `slice` entries of the list over 256 columns (VEC: eight neighbours per lane). A run of one step that lies inside
// the slice is a finished row of the gradient; the others are parts for k_table_join.
template <bool F32, bool VEC>
__global__ void __launch_bounds__(kTableThreads) k_table_sum(const TableArgs a) {
  const int lane = threadIdx.x & 31;
  const int64_t sl = (int64_t)blockIdx.y * kTableWarps + (threadIdx.x >> 5);
  const int total = a.begin[a.steps];
  if (sl * a.slice >= total) return;
  const int i0 = (int)(sl * a.slice), i1 = (int)min((int64_t)total, (sl + 1) * a.slice);
  const int c0 = blockIdx.x * 256 + (VEC ? lane * 8 : lane);
  constexpr int kStep = VEC ? 1 : 32;
  float sum[8] = {};
  int s = step_of(a.begin, a.steps, i0);
  int from = a.begin[s], end = a.begin[s + 1];
  const auto flush = [&]() {
    if (from >= i0 && end <= i1) {
      uint16_t* out = a.dtable + (size_t)s * a.n;
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (c0 + u * kStep < a.n) out[c0 + u * kStep] = round16(sum[u], a.f16);
    } else {
      float* out = a.part + ((size_t)sl * 2 + (from >= i0 ? 1 : 0)) * a.n;
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (c0 + u * kStep < a.n) out[c0 + u * kStep] = sum[u];
    }
  };
  constexpr int kAhead = 4;
  for (int i = i0; i < i1; i += kAhead) {
    float v[kAhead][8];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (i + k >= i1) break;
      const int row = __ldg(a.list + i + k);
      if (VEC) {
        float f[8];
        const bool in = c0 < a.n;
        if (F32) {
          const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(a.dy) + (size_t)row * a.lddy + c0);
          const float4 lo = in ? __ldg(p) : make_float4(0.f, 0.f, 0.f, 0.f), hi = in ? __ldg(p + 1) : make_float4(0.f, 0.f, 0.f, 0.f);
          v[k][0] = lo.x; v[k][1] = lo.y; v[k][2] = lo.z; v[k][3] = lo.w; v[k][4] = hi.x; v[k][5] = hi.y; v[k][6] = hi.z; v[k][7] = hi.w;
        } else {
          const uint4 w = in ? __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.dy) + (size_t)row * a.lddy + c0))
                             : make_uint4(0u, 0u, 0u, 0u);
          const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const float2 t = unpack16x2(q[u], a.f16);
            v[k][2 * u] = t.x; v[k][2 * u + 1] = t.y;
          }
        }
        if (a.factor) {
          const uint4 w = in ? __ldg(reinterpret_cast<const uint4*>(a.factor + (size_t)row * a.ldz + c0)) : make_uint4(0u, 0u, 0u, 0u);
          const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const float2 t = unpack16x2(q[u], 1);
            f[2 * u] = t.x; f[2 * u + 1] = t.y;
          }
#pragma unroll
          for (int u = 0; u < 8; ++u) v[k][u] *= f[u];
        }
      } else {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int c = c0 + u * kStep;
          v[k][u] = c < a.n ? load_typed(a.dy, a.tdy, (size_t)row * a.lddy + c) : 0.f;
          if (a.factor && c < a.n) v[k][u] *= unpack16(a.factor[(size_t)row * a.ldz + c], 1);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (i + k >= i1) break;
      if (i + k >= end) {                         // the next step that has rows
        flush();
#pragma unroll
        for (int u = 0; u < 8; ++u) sum[u] = 0.f;
        do { ++s; end = a.begin[s + 1]; } while (end <= i + k);
        from = a.begin[s];
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) sum[u] += v[k][u];
    }
  }
  flush();
}

// One CTA per step and 256 columns: zeros for a step without rows, the sums of a run that crosses slices.
__global__ void __launch_bounds__(256) k_table_join(const TableArgs a) {
  const int s = blockIdx.y, c = blockIdx.x * 256 + threadIdx.x;
  const int from = a.begin[s], end = a.begin[s + 1];
  if (c >= a.n) return;
  float sum = 0.f;
  if (from < end) {
    const int first = from / a.slice, last = (end - 1) / a.slice;
    if (first == last) return;                    // written by the slice's warp
    sum = a.part[((size_t)first * 2 + 1) * a.n + c];
#pragma unroll 4
    for (int i = first + 1; i <= last; ++i) sum += a.part[(size_t)i * 2 * a.n + c];
  }
  a.dtable[(size_t)s * a.n + c] = round16(sum, a.f16);
}

// List entries of a warp: 32, or more where that makes over four times as many warps as the machine holds.
int table_slice(int64_t rows, int32_t n) {
  const int64_t cols = (n + 255) / 256, most = 4 * 148 * 48;
  return (int)std::max<int64_t>(32, (rows * cols + most - 1) / most);
}
int64_t table_slices(int64_t rows, int32_t n) {
  const int s = table_slice(rows, n);
  return (rows + s - 1) / s;
}

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

size_t linear_factor_bytes(int64_t rows, int32_t n) { return (size_t)rows * round_up(n, 8) * 2; }

LinearWorkspace linear_workspace(int64_t rows, int32_t k, int32_t n, int32_t nsteps, bool has_table) {
  LinearWorkspace w{};
  size_t at = 256;                                // the status word
  const auto take = [&](size_t bytes) { const size_t o = at; at = round_up(at + bytes, 256); return o; };
  w.dz = take(linear_factor_bytes(rows, n));
  w.db = take(rows > 0 ? (size_t)dz_chunks(rows, n) * n * 4 : 0);
  w.dw = take(rows > 0 ? part_floats(n, k, linear_parts(rows, k, n)) * 4 : 0);
  w.begin = take(has_table ? ((size_t)nsteps + 1) * 4 : 0);
  w.list = take(has_table ? (size_t)rows * 4 : 0);
  w.table = take(has_table && rows > 0 ? (size_t)table_slices(rows, n) * 2 * n * 4 : 0);
  w.bytes = at;
  return w;
}

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
  e.wide = (size_t)a.n * size % 16 == 0 && whole(a.y, a.ldy, size) && (!a.residual || whole(a.residual, a.ldr, size));
  e.table_wide = a.n % 8 == 0 && whole(a.table, a.n, 2);
  FfnArgs f{};
  f.rows = a.rows; f.f16 = a.f16; f.act = a.act; f.err = a.err;
  if (prefer_split<kLinear>(a.rows, a.n, steps(a.k))) {
    SplitSpec s{};
    s.w[0] = {a.w, a.k}; s.t[0] = {a.x, a.ldx};
    s.nseg = 1; s.N = a.n; s.K = a.k; s.out = a.y; s.ldo = a.ldy;
    return launch_split<kLinear>(f, s, nullptr, true, st, &e);
  }
  ProductSpec s{};
  s.a[0] = {a.x, a.ldx}; s.b[0] = {a.w, a.k};
  s.nseg = 1; s.M = a.rows; s.N = a.n; s.K = a.k; s.out = a.y; s.ldo = a.ldy;
  return launch_tiles<kLinear, false>(f, &s, 1, true, st, nullptr, nullptr, false, &e);
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
  const dim3 grid(cols, (t.slices + kTableWarps - 1) / kTableWarps);
  if (t.tdy == SDS_F32) {
    if (vec) k_table_sum<true, true><<<grid, kTableThreads, 0, st>>>(t);
    else k_table_sum<true, false><<<grid, kTableThreads, 0, st>>>(t);
  } else {
    if (vec) k_table_sum<false, true><<<grid, kTableThreads, 0, st>>>(t);
    else k_table_sum<false, false><<<grid, kTableThreads, 0, st>>>(t);
  }
  k_table_join<<<dim3(cols, t.steps), 256, 0, st>>>(t);
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
  const uint16_t* factor = a.act == SDS_ACT_NONE ? nullptr : a.factor;
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
    t.part = reinterpret_cast<float*>(ws + at.table);
    t.dy = a.dy; t.lddy = a.lddy; t.tdy = a.ty; t.factor = factor; t.ldz = ldz;
    t.dtable = static_cast<uint16_t*>(a.dtable);
    t.rows = a.rows; t.n = a.n; t.steps = a.steps; t.f16 = a.f16;
    t.slice = table_slice(a.rows, a.n); t.slices = (int)table_slices(a.rows, a.n);
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
