// Dropout: y = D x + residual with D = 0 or 1 / (1 - p), forward and (on dy) backward.
//
// D is a function of (seed, step, row, column) through the library's generator and is never stored: the backward pass draws it
// again. One block of Philox-4x32-10 decides eight neighbouring columns of a row with 16 bits each, so p is a multiple of 2^-16
// (1 / (1 - p) is that of the rounded p: the mean is kept exactly). 32 bits per column would take twice the blocks, and the
// generator would bound the kernel: it makes 1.7e12 words a second here, and memory moves 1.6e12 16-bit elements in and out.
#include "sds_residual.cuh"

namespace sds {

namespace {

constexpr int kDropThreads = 256;

// A thread takes blocks of eight columns of the whole array, in steps of the grid, two requested at a time. Bound by memory: 16384 x 2048
// bf16 onto a float residual 50 us (336 MB, 6.7 TB/s), its gradient from float to bf16 36 (201 MB, 5.6 TB/s).
template <class TX, class TY>
__global__ void __launch_bounds__(kDropThreads, 3) k_dropout(const DropoutCall a, int64_t nb) {
  start_after_prior_kernel();
  const bool drops = a.drop.threshold != 0;
  const uint32_t dstep = drops ? dropout_step(a.drop) : 0u;
  const float2 scale = both(drops ? a.drop.scale : 1.0f);
  const int64_t stride = (int64_t)gridDim.x * kDropThreads, first = (int64_t)blockIdx.x * kDropThreads + threadIdx.x;
  const int64_t srow = stride / nb, sblock = stride % nb;
  int64_t row = first / nb, block = first % nb;
  constexpr int kAhead = 2;
  while (row < a.rows) {
    int64_t rows[kAhead], blocks[kAhead];
    Raw<TX> xr[kAhead];
    Raw<TY> rr[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      rows[i] = row;
      blocks[i] = block;
      if (row < a.rows) {
        xr[i].load(static_cast<const TX*>(a.x) + (size_t)row * a.ldx + block * kBlock);
        if (a.residual) rr[i].load(static_cast<const TY*>(a.residual) + (size_t)row * a.ldr + block * kBlock);
      }
      row += srow;
      block += sblock;
      if (block >= nb) { block -= nb; ++row; }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (rows[i] >= a.rows) break;
      float2 x[P], y[P];
      words_to(xr[i].q, x, TX{});
      Kept kept;
      if (drops) kept = kept_block(a.drop, dstep, a.drop.row0 + (uint64_t)rows[i], (uint32_t)blocks[i]);
      if (a.residual) {
        words_to(rr[i].q, y, TY{});
#pragma unroll
        for (int k = 0; k < P; ++k) add_branch(y[k], scale, x[k], drops, kept, k);
      } else {
#pragma unroll
        for (int k = 0; k < P; ++k) y[k] = drops ? select_kept(mul2(scale, x[k]), kept, k) : x[k];
      }
      store_words(static_cast<TY*>(a.y) + (size_t)rows[i] * a.ldy + blocks[i] * kBlock, y);
    }
  }
}

// Rows that are not whole pieces: a warp takes 256 columns of a row, a lane every 32nd of them, so that accesses are neighbours.
// 33500 x 1001 bf16 49 us (134 MB, 2.7 TB/s): 16-bit loads and stores, and issue.
template <class TX, class TY>
__global__ void __launch_bounds__(kDropThreads) k_dropout_narrow(const DropoutCall a, int64_t groups) {
  start_after_prior_kernel();
  const bool drops = a.drop.threshold != 0;
  const uint32_t dstep = drops ? dropout_step(a.drop) : 0u;
  const float scale = drops ? a.drop.scale : 1.0f;
  const int lane = threadIdx.x & 31;
  const int64_t stride = (int64_t)gridDim.x * (kDropThreads / 32), total = a.rows * groups;
  for (int64_t unit = (int64_t)blockIdx.x * (kDropThreads / 32) + (threadIdx.x >> 5); unit < total; unit += stride) {
    const int64_t row = unit / groups;
    Columns<32, 1, false> col(lane, a.d);
    col.c0 += (int)(unit - row * groups) * 32 * kBlock;
    float2 x[P], y[P];
    load_scalar(static_cast<const TX*>(a.x) + (size_t)row * a.ldx, col, x);
    if (a.residual) {
      load_scalar(static_cast<const TY*>(a.residual) + (size_t)row * a.ldr, col, y);
    } else {
#pragma unroll
      for (int i = 0; i < P; ++i) y[i] = both(0.f);
    }
    Kept kept;
    if (drops) kept = kept_columns(a.drop, dstep, (int)row, col, lane);
#pragma unroll
    for (int i = 0; i < P; ++i) add_branch(y[i], both(scale), x[i], drops, kept, i);
    store_row(static_cast<TY*>(a.y) + (size_t)row * a.ldy, col, true, y);
  }
}

template <class TX, class TY>
cudaError_t dropout_k(const DropoutCall& a, cudaStream_t st) {
  static std::atomic<int> cache[kRowDevices];
  int resident = 0;
  const cudaError_t e = row_resident(k_dropout<TX, TY>, cache, kDropThreads, 0, 1, &resident);
  if (e != cudaSuccess) return e;
  const int64_t nb = a.d / kBlock, ctas = (a.rows * nb + kDropThreads - 1) / kDropThreads;
  return row_launch(k_dropout<TX, TY>, dim3((unsigned)std::min<int64_t>(ctas, resident)), kDropThreads, 0, 1, st, a, nb);
}
template <class TX, class TY>
cudaError_t dropout_narrow_k(const DropoutCall& a, cudaStream_t st) {
  static std::atomic<int> cache[kRowDevices];
  int resident = 0;
  const cudaError_t e = row_resident(k_dropout_narrow<TX, TY>, cache, kDropThreads, 0, 1, &resident);
  if (e != cudaSuccess) return e;
  const int64_t groups = (a.d + 32 * kBlock - 1) / (32 * kBlock), ctas = (a.rows * groups + kDropThreads / 32 - 1) / (kDropThreads / 32);
  return row_launch(k_dropout_narrow<TX, TY>, dim3((unsigned)std::min<int64_t>(ctas, resident)), kDropThreads, 0, 1, st, a, groups);
}

template <class TX, class TY>
cudaError_t dropout_t(const DropoutCall& a, cudaStream_t st) {
  const bool vec = a.d % 8 == 0 && pieces8(a.x, a.ldx, a.tx) && pieces8(a.y, a.ldy, a.ty) &&
                   (!a.residual || pieces8(a.residual, a.ldr, a.ty));
  return vec ? dropout_k<TX, TY>(a, st) : dropout_narrow_k<TX, TY>(a, st);
}

}  // namespace

cudaError_t launch_dropout(const DropoutCall& a, cudaStream_t st) {
  if (a.rows <= 0) return cudaSuccess;
  if (a.tx == SDS_F32 && a.ty == SDS_F32) return dropout_t<float, float>(a, st);
  if (a.tx == SDS_F32 && a.ty == SDS_BF16) return dropout_t<float, Bf16>(a, st);
  if (a.tx == SDS_F32) return dropout_t<float, F16>(a, st);
  if (a.tx == SDS_BF16) return a.ty == SDS_F32 ? dropout_t<Bf16, float>(a, st) : dropout_t<Bf16, Bf16>(a, st);
  return a.ty == SDS_F32 ? dropout_t<F16, float>(a, st) : dropout_t<F16, F16>(a, st);
}

}  // namespace sds
