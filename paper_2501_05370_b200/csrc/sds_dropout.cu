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

// A thread takes blocks of eight columns of the whole array in steps of the grid. VEC: 16-byte accesses.
template <class TX, class TY, bool VEC>
__global__ void __launch_bounds__(kDropThreads) k_dropout(const DropoutCall a, int64_t nb) {
  start_after_prior_kernel();
  const bool drops = a.drop.threshold != 0;
  const uint32_t dstep = drops ? dropout_step(a.drop) : 0u;
  const int64_t stride = (int64_t)gridDim.x * kDropThreads, first = (int64_t)blockIdx.x * kDropThreads + threadIdx.x;
  const int64_t srow = stride / nb, sblock = stride % nb;
  int64_t row = first / nb, block = first % nb;
  const auto advance = [&]() {
    row += srow;
    block += sblock;
    if (block >= nb) { block -= nb; ++row; }
  };
  constexpr int kAhead = VEC ? 4 : 1;             // blocks requested before the first is used
  while (row < a.rows) {
    int64_t rows[kAhead], blocks[kAhead];
    float2 x[kAhead][P], res[kAhead][P];
    Raw<TX> xr[kAhead];
    Raw<TY> rr[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      rows[i] = row;
      blocks[i] = block;
      if (row < a.rows) {
        const TX* px = static_cast<const TX*>(a.x) + (size_t)row * a.ldx + block * kBlock;
        const TY* pr = static_cast<const TY*>(a.residual) + (size_t)row * a.ldr + block * kBlock;
        if (VEC) {
          xr[i].load(px);
          if (a.residual) rr[i].load(pr);
        } else {
          const int live = (int)min((int64_t)kBlock, a.d - block * kBlock);
#pragma unroll
          for (int e = 0; e < kBlock; ++e) {
            element(x[i], e) = e < live ? Conv<TX>::get(px[e]) : 0.f;
            element(res[i], e) = a.residual && e < live ? Conv<TY>::get(pr[e]) : 0.f;
          }
        }
      }
      advance();
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (rows[i] >= a.rows) break;
      if (VEC) {
        words_to(xr[i].q, x[i], TX{});
        if (a.residual) words_to(rr[i].q, res[i], TY{});
      }
      Kept kept;
      if (drops) kept = kept_block(a.drop, dstep, a.drop.row0 + (uint64_t)rows[i], (uint32_t)blocks[i]);
      const float2 scale = both(drops ? a.drop.scale : 1.0f);
#pragma unroll
      for (int k = 0; k < P; ++k) {
        if (a.residual) {
          add_branch(res[i][k], scale, x[i][k], drops, kept, k);
          x[i][k] = res[i][k];
        } else if (drops) {
          x[i][k] = select_kept(mul2(scale, x[i][k]), kept, k);
        }
      }
      TY* py = static_cast<TY*>(a.y) + (size_t)rows[i] * a.ldy + blocks[i] * kBlock;
      if (VEC) {
        store_words(py, x[i]);
      } else {
        const int live = (int)min((int64_t)kBlock, a.d - blocks[i] * kBlock);
#pragma unroll
        for (int e = 0; e < kBlock; ++e)
          if (e < live) py[e] = Conv<TY>::put(element(x[i], e));
      }
    }
  }
}

template <class TX, class TY, bool VEC>
cudaError_t dropout_k(const DropoutCall& a, cudaStream_t st) {
  static std::atomic<int> cache[kRowDevices];
  int resident = 0;
  const cudaError_t e = row_resident(k_dropout<TX, TY, VEC>, cache, kDropThreads, 0, 1, &resident);
  if (e != cudaSuccess) return e;
  const int64_t nb = (a.d + kBlock - 1) / kBlock, ctas = (a.rows * nb + kDropThreads - 1) / kDropThreads;
  return row_launch(k_dropout<TX, TY, VEC>, dim3((unsigned)std::min<int64_t>(ctas, resident)), kDropThreads, 0, 1, st, a, nb);
}

template <class TX, class TY>
cudaError_t dropout_t(const DropoutCall& a, cudaStream_t st) {
  const bool vec = a.d % 8 == 0 && pieces8(a.x, a.ldx, a.tx) && pieces8(a.y, a.ldy, a.ty) &&
                   (!a.residual || pieces8(a.residual, a.ldr, a.ty));
  return vec ? dropout_k<TX, TY, true>(a, st) : dropout_k<TX, TY, false>(a, st);
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
