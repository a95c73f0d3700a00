// Residual norm: how a backward call deals out its rows, the kernels that add the workers' sums, and the choice of the row kernels.
#include "sds_residual.cuh"

namespace sds {

namespace {

// groups of threads that run at once in a backward launch: 512 threads per SM
int most_workers(int d) { return kRowSms * 512 / residual_threads(d); }

// COLS columns of a CTA, a thread one of them of every PARTS-th worker. Bound by latency: as many parts as leave every SM one CTA of
// 1024 threads, and short CTAs for wide rows. Backward of 1021 x 1001 float (511 workers): <8, 128> 16.0 us, <16, 64> 16.5, <16, 16> 22.3;
// 20000 x 64 23.0, 33.2, 116; 64 x 2048 8.4, 7.1, 7.1; 16384 x 2048 126.7, 124.3, 128.5; 300 x 5000 30.0, 27.2, 24.7; 1 x 10056 18.8, 12.9, 8.7.
// One group (kSumAll): the plain sums give every gradient; else they are weighted already, and the groups' own gradients were written
// before.
template <int COLS, int PARTS>
__global__ void __launch_bounds__(COLS * PARTS) k_residual_join(const ResidualNormArgs a) {
  __shared__ float sums[3][PARTS * COLS], total[3][COLS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = threadIdx.x % COLS, d = a.d;
  const int c = blockIdx.x * COLS + col;
  start_after_prior_kernel();
  float s[3] = {0.f, 0.f, 0.f};
  if (c < d) {
#pragma unroll 4
    for (int64_t i = threadIdx.x / COLS; i < a.workers; i += PARTS) {
      const float* from = a.part + (size_t)i * 3 * d + c;
      s[0] += from[0];
      s[1] += from[d];
      s[2] += from[2 * (size_t)d];
    }
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) sums[k][threadIdx.x] = s[k];
  __syncthreads();
  if (warp < 3) {
    float v = 0.f;
#pragma unroll 8
    for (int i = 0; i < PARTS * COLS / 32; ++i) v += sums[warp][i * 32 + lane];
#pragma unroll
    for (int at = COLS; at < 32; at *= 2) v += __shfl_xor_sync(0xffffffffu, v, at);
    if (lane < COLS) total[warp][lane] = v;
  }
  __syncthreads();
  if (threadIdx.x >= COLS || c >= d) return;
  const float A = total[0][col], B = total[1][col], C = total[2][col];
  if (a.mode != kSumAll) {
    if (a.dw) store_any(a.dw, a.tw, c, A);
    if (a.db) store_any(a.db, a.tw, c, B);
    if (a.dwp) store_any(a.dwp, a.tw, c, C);
    return;
  }
  const float w = a.w ? load_any(a.w, a.tw, c) : 1.f, b = a.b ? load_any(a.b, a.tw, c) : 0.f, wp = a.wp ? load_any(a.wp, a.tw, c) : 1.f;
  const float f = 1.0f + (a.scale ? load_any(a.scale, a.tc, c) : 0.f), gate = a.gate ? load_any(a.gate, a.tc, c) : 1.f;
  if (a.dw) store_any(a.dw, a.tw, c, f * A);
  if (a.db) store_any(a.db, a.tw, c, f * B);
  if (a.dwp) store_any(a.dwp, a.tw, c, gate * C);
  if (a.dshift) store_any(a.dshift, a.tc, c, B);
  if (a.dscale) store_any(a.dscale, a.tc, c, fmaf(w, A, b * B));
  if (a.dgate) store_any(a.dgate, a.tc, c, wp * C);
}

// Groups whose rows several workers had: one for each border between two workers, where it is the first border in its group. A CTA takes
// 32 columns of it, a warp every eighth part.
__global__ void __launch_bounds__(256) k_residual_join_groups(const ResidualNormArgs a, int strips) {
  __shared__ float sums[3][8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, d = a.d;
  const int first = (int)(blockIdx.x / strips), c = (int)(blockIdx.x % strips) * 32 + lane;
  const int64_t border = (int64_t)(first + 1) * a.share;
  const int group = (int)(border / a.per);
  start_after_prior_kernel();
  if (border % a.per == 0 || (int64_t)group * a.per / a.share != first) return;
  const int last = (int)(((int64_t)(group + 1) * a.per - 1) / a.share);
  float s[3] = {0.f, 0.f, 0.f};
  if (c < d) {
#pragma unroll 4
    for (int i = first + warp; i <= last; i += 8) {
      const float* from = a.group_part + ((size_t)i * 2 + (i == first ? 1 : 0)) * 3 * d + c;
      s[0] += from[0];
      s[1] += from[d];
      s[2] += from[2 * (size_t)d];
    }
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) sums[k][warp][lane] = s[k];
  __syncthreads();
  if (warp != 0 || c >= d) return;
  float t[3] = {0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < 3; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) t[k] += sums[k][i][lane];
  const float w = a.w ? load_any(a.w, a.tw, c) : 1.f, b = a.b ? load_any(a.b, a.tw, c) : 0.f, wp = a.wp ? load_any(a.wp, a.tw, c) : 1.f;
  if (a.dshift) store_any(a.dshift, a.tc, (size_t)group * a.lddshift + c, t[1]);
  if (a.dscale) store_any(a.dscale, a.tc, (size_t)group * a.lddscale + c, fmaf(w, t[0], b * t[1]));
  if (a.dgate) store_any(a.dgate, a.tc, (size_t)group * a.lddgate + c, wp * t[2]);
}

cudaError_t launch_rows(ResidualNormArgs& a, bool vec, bool backward, cudaStream_t st) {
  if (a.tr == SDS_BF16) return residual_bf16(a, vec, backward, st);
  if (a.tr == SDS_F16) return residual_f16(a, vec, backward, st);
  if (a.th == SDS_BF16) return residual_f32_bf16(a, vec, backward, st);
  if (a.th == SDS_F16) return residual_f32_f16(a, vec, backward, st);
  return residual_f32(a, vec, backward, st);
}

bool whole(const void* p, int64_t ld, int type) { return !p || pieces8(p, ld, type); }
bool whole_vectors(const ResidualNormArgs& a) {
  return a.d % 8 == 0 && whole(a.w, 0, a.tw) && whole(a.b, 0, a.tw) && whole(a.wp, 0, a.tw) && whole(a.gate, a.ldgate, a.tc) &&
         whole(a.scale, a.ldscale, a.tc) && whole(a.shift, a.ldshift, a.tc);
}

}  // namespace

void residual_norm_plan(ResidualNormArgs* a, size_t* part_floats, size_t* group_floats) {
  const bool wanted = a->dgate || a->dscale || a->dshift, conditioned = wanted || a->gate || a->scale || a->shift;
  a->mode = a->groups == 1 || !conditioned ? kSumAll : a->per > 1 && wanted ? kSumGroups : kSumWeighted;
  a->workers = std::min(a->rows, most_workers(a->d));
  *part_floats = (size_t)a->workers * 3 * (size_t)a->d;
  *group_floats = a->mode == kSumGroups ? 2 * *part_floats : 0;
}

cudaError_t launch_residual_norm(const ResidualNormArgs& a, cudaStream_t st) {
  if (a.rows <= 0) return cudaSuccess;
  const bool vec = whole_vectors(a) && whole(a.r, a.ldr, a.tr) && whole(a.h, a.ldh, a.th) && whole(a.n, a.ldn, a.th) &&
                   (!a.h || whole(a.out, a.ldo, a.tr));
  ResidualNormArgs g = a;
  return launch_rows(g, vec, false, st);
}

cudaError_t launch_residual_norm_backward(const ResidualNormArgs& a, cudaStream_t st) {
  cudaError_t e = cudaSuccess;
  if (a.rows <= 0) {                              // empty sums
    const size_t sw = a.tw == SDS_F32 ? 4 : 2, sc = a.tc == SDS_F32 ? 4 : 2;
    for (void* p : {a.dw, a.db, a.dwp})
      if (p && (e = cudaMemsetAsync(p, 0, (size_t)a.d * sw, st)) != cudaSuccess) return e;
    const struct { void* p; int64_t ld; } cond[3] = {{a.dgate, a.lddgate}, {a.dscale, a.lddscale}, {a.dshift, a.lddshift}};
    for (const auto& c : cond)
      if (c.p && a.groups > 0 &&
          (e = cudaMemset2DAsync(c.p, (size_t)c.ld * sc, 0, (size_t)a.d * sc, (size_t)a.groups, st)) != cudaSuccess)
        return e;
    return cudaSuccess;
  }
  const bool vec = whole_vectors(a) && whole(a.r, a.ldr, a.tr) && whole(a.h, a.ldh, a.th) && whole(a.dn, a.lddn, a.th) &&
                   whole(a.dr, a.lddr, a.tr) && whole(a.dr_in, a.lddr_in, a.tr) && whole(a.dh, a.lddh, a.th) &&
                   whole(a.dgate, a.lddgate, a.tc) && whole(a.dscale, a.lddscale, a.tc) && whole(a.dshift, a.lddshift, a.tc);
  ResidualNormArgs g = a;
  if ((e = launch_rows(g, vec, true, st)) != cudaSuccess) return e;
  const int strips = (a.d + 31) / 32;
  if (a.mode == kSumGroups && g.workers > 1 && g.share % g.per != 0 &&      // (else no group crosses workers)
      (e = row_launch(k_residual_join_groups, dim3((unsigned)((g.workers - 1) * strips)), 256, 0, 1, st, g, strips)) != cudaSuccess)
    return e;
  const bool any = a.dw || a.db || a.dwp || (a.mode == kSumAll && (a.dgate || a.dscale || a.dshift));
  if (!any) return cudaSuccess;
  const auto join = [&](auto kernel, int cols, int parts) {
    return row_launch(kernel, dim3((unsigned)((a.d + cols - 1) / cols)), cols * parts, 0, 1, st, g);
  };
  if (a.d <= 8 * kRowSms) return join(k_residual_join<8, 128>, 8, 128);
  return a.d <= 16 * kRowSms ? join(k_residual_join<16, 64>, 16, 64) : join(k_residual_join<16, 16>, 16, 16);
}

}  // namespace sds
