// Layer norm over rows, forward and backward.
//
//   mean = sum x / d, var = sum (x - mean)^2 / d, rstd = 1 / sqrt(var + eps), xhat = (x - mean) rstd
//   y  = xhat w + b
//   dx = rstd (w dy - <w dy> - xhat <w dy xhat>)      (<.> = mean over the row)
//   dw = sum_rows dy xhat,   db = sum_rows dy
//
// Both directions are bound by memory: one read of every input, one write of every output. A group of threads
// holds a row in registers (E elements per thread) between the pass that sums and the pass that writes, and
// walks over rows with the weights in registers, so that they are read once per group and not once per row.
// The next row is requested before the current one is reduced.
//
// The mean is rounded to 32 bits, which for rows far from zero is an error that every element shares. The second
// reduction therefore also sums x - mean (exact differences) and the remainder c0 is taken off every element; the
// backward pass does the same in its one reduction.
//
// Gradients of the weights: a CTA keeps the sums of its columns in registers over all rows it visits and stores
// them once; a second kernel adds the CTAs' sums in a fixed order (no atomics: same bits on every run).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "../../include/sds.h"
#include "sds_layers.h"

namespace sds {

namespace {

struct Bf16 { uint16_t v; };
struct F16 { uint16_t v; };

template <class T> struct Conv;
template <> struct Conv<float> {
  __device__ static float get(float v) { return v; }
  __device__ static float put(float v) { return v; }
};
template <> struct Conv<Bf16> {
  __device__ static float get(Bf16 v) { return __uint_as_float((uint32_t)v.v << 16); }
  __device__ static Bf16 put(float v) { return Bf16{__bfloat16_as_ushort(__float2bfloat16_rn(v))}; }
};
template <> struct Conv<F16> {
  __device__ static float get(F16 v) { return __half2float(__ushort_as_half(v.v)); }
  __device__ static F16 put(float v) { return F16{__half_as_ushort(__float2half_rn(v))}; }
};

// V consecutive elements as one access of sizeof(T) * V bytes
template <class T, int V> struct alignas(sizeof(T) * V) Pack { T v[V]; };

// a column vector of any of the three types, read once per thread group
__device__ __forceinline__ float load_any(const void* p, int type, size_t i) {
  if (type == SDS_F32) return static_cast<const float*>(p)[i];
  if (type == SDS_BF16) return Conv<Bf16>::get(static_cast<const Bf16*>(p)[i]);
  return Conv<F16>::get(static_cast<const F16*>(p)[i]);
}
__device__ __forceinline__ void store_any(void* p, int type, size_t i, float v) {
  if (type == SDS_F32) static_cast<float*>(p)[i] = v;
  else if (type == SDS_BF16) static_cast<Bf16*>(p)[i] = Conv<Bf16>::put(v);
  else static_cast<F16*>(p)[i] = Conv<F16>::put(v);
}

// sum of N values over the TPR threads of a row's group, the result in every thread. `slot`: shared memory of the
// group, N * (TPR / 32) floats, not reused before the group's next barrier.
template <int TPR, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float* slot, int t, int bar) {
  constexpr int W = TPR < 32 ? TPR : 32;
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1)
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] += __shfl_xor_sync(0xffffffffu, v[n], o);
  if (TPR > 32) {
    constexpr int NW = TPR > 32 ? TPR / 32 : 1;
    if ((t & 31) == 0)
#pragma unroll
      for (int n = 0; n < N; ++n) slot[n * NW + (t >> 5)] = v[n];
    asm volatile("bar.sync %0, %1;" ::"r"(bar), "r"(TPR) : "memory");
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float s = slot[n * NW + ((t & 31) & (NW - 1))];
#pragma unroll
      for (int o = NW / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      v[n] = s;
    }
  }
}

// threads of a row's group and elements per thread; groups of up to 128 threads share a CTA of 256
template <int TPR> constexpr int norm_cta = TPR < 256 ? 256 : TPR;

template <class TX, class TY, int TPR, int E, bool VEC, bool RES>
__global__ void __launch_bounds__(norm_cta<TPR>) k_norm(const NormArgs a) {
  constexpr int RPC = norm_cta<TPR> / TPR;                    // rows of a CTA at a time
  constexpr int V = VEC ? (sizeof(TX) == 4 ? 4 : 8) : 1;
  constexpr int NV = E / V;
  constexpr int NW = TPR > 32 ? TPR / 32 : 1;
  __shared__ float slots[RPC * 3 * NW];
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  float* slot = slots + sub * 3 * NW;
  const int rows = a.nrows_dev ? min(*a.nrows_dev, a.rows) : a.rows;
  const int d = a.d;
  const float inv_d = 1.0f / (float)d;
  using PX = Pack<TX, V>;
  using PY = Pack<TY, V>;
  float w[E], b[E];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int u = 0; u < V; ++u) {
      const int c = (i * TPR + t) * V + u;
      w[i * V + u] = (a.w && c < d) ? load_any(a.w, a.tw, c) : 1.0f;
      b[i * V + u] = (a.b && c < d) ? load_any(a.b, a.tw, c) : 0.0f;
    }
  PX nxt[NV];
  auto fetch = [&](int row) {
    const TX* xr = static_cast<const TX*>(a.x) + (size_t)row * a.ldx;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + t) * V;
      if (row < rows && c < d) nxt[i] = *reinterpret_cast<const PX*>(xr + c);
      else nxt[i] = PX{};
    }
  };
  int base = blockIdx.x * RPC;
  if (base < rows) fetch(base + sub);
  for (; base < rows; base += gridDim.x * RPC) {
    const int row = base + sub;
    const bool live = row < rows;
    float x[E];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int u = 0; u < V; ++u) x[i * V + u] = Conv<TX>::get(nxt[i].v[u]);
    if (RES && live) {                                          // x + temb[k], kept as the residual stream
      const uint16_t* te = a.temb ? a.temb + (size_t)__ldg(a.rowk + row) * d : nullptr;
      float* rr = a.res + (size_t)row * d;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * V;
        if (c < d) {
          Pack<float, V> o;
          if (te) {
            const Pack<Bf16, V> e = *reinterpret_cast<const Pack<Bf16, V>*>(te + c);
#pragma unroll
            for (int u = 0; u < V; ++u) x[i * V + u] += Conv<Bf16>::get(e.v[u]);
          }
#pragma unroll
          for (int u = 0; u < V; ++u) o.v[u] = x[i * V + u];
          *reinterpret_cast<Pack<float, V>*>(rr + c) = o;
        }
      }
    }
    fetch(row + gridDim.x * RPC);
    float s[1] = {0.f};
#pragma unroll
    for (int e = 0; e < E; ++e) s[0] += x[e];                   // (elements past d hold zeros)
    group_sum<TPR, 1>(s, slot, t, 1 + sub);
    const float mean = __fmul_rn(s[0], inv_d);                  // (a rounded number: the same one with and without statistics)
    float q[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const bool in = (i * TPR + t) * V < d;
#pragma unroll
      for (int u = 0; u < V; ++u) {
        const float c = x[i * V + u] - mean;
        x[i * V + u] = c;
        if (in) { q[0] += c; q[1] = fmaf(c, c, q[1]); }
      }
    }
    group_sum<TPR, 2>(q, slot + NW, t, 1 + sub);
    const float c0 = __fmul_rn(q[0], inv_d);
    const float rstd = rsqrtf(fmaxf(fmaf(-c0, c0, q[1] * inv_d), 0.f) + a.eps);
    if (!live) continue;
    if (t == 0) {
      if (a.mean) a.mean[row] = mean + c0;
      if (a.rstd) a.rstd[row] = rstd;
    }
    TY* yr = static_cast<TY*>(a.y) + (size_t)row * a.ldy;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + t) * V;
      if (c < d) {
        PY o;
#pragma unroll
        for (int u = 0; u < V; ++u) o.v[u] = Conv<TY>::put(fmaf((x[i * V + u] - c0) * rstd, w[i * V + u], b[i * V + u]));
        *reinterpret_cast<PY*>(yr + c) = o;
      }
    }
  }
}

// rows longer than the register kernels hold: one CTA per row, the row read three times (the later passes from L2)
template <class TX, class TY>
__global__ void __launch_bounds__(1024) k_norm_long(const NormArgs a) {
  __shared__ float slot[96];
  const int t = threadIdx.x;
  const double inv_d = 1.0 / (double)a.d;
  for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const TX* xr = static_cast<const TX*>(a.x) + (size_t)row * a.ldx;
    float s[1] = {0.f};
    for (int c = t; c < a.d; c += 1024) s[0] += Conv<TX>::get(xr[c]);
    group_sum<1024, 1>(s, slot, t, 1);
    const float mean = (float)(s[0] * inv_d);
    float q[2] = {0.f, 0.f};
    for (int c = t; c < a.d; c += 1024) {
      const float v = Conv<TX>::get(xr[c]) - mean;
      q[0] += v;
      q[1] = fmaf(v, v, q[1]);
    }
    group_sum<1024, 2>(q, slot + 32, t, 1);
    const float c0 = (float)(q[0] * inv_d);
    const float rstd = rsqrtf(fmaxf(fmaf(-c0, c0, (float)(q[1] * inv_d)), 0.f) + a.eps);
    if (t == 0) {
      if (a.mean) a.mean[row] = mean + c0;
      if (a.rstd) a.rstd[row] = rstd;
    }
    TY* yr = static_cast<TY*>(a.y) + (size_t)row * a.ldy;
    for (int c = t; c < a.d; c += 1024) {
      const float w = a.w ? load_any(a.w, a.tw, c) : 1.0f, b = a.b ? load_any(a.b, a.tw, c) : 0.0f;
      yr[c] = Conv<TY>::put(fmaf((Conv<TX>::get(xr[c]) - mean - c0) * rstd, w, b));
    }
  }
}

// Backward. SMEM: the CTA's weight-gradient sums live in shared memory (rows so long that a thread holds 16
// elements: x, dy and two sums of 16 would not fit the 64 registers a thread of 1024 has), else in registers.
template <class TX, class TY, int TPR, int E, bool VEC, bool SMEM>
__global__ void __launch_bounds__(norm_cta<TPR>) k_norm_bwd(const NormArgs a) {
  constexpr int CTA = norm_cta<TPR>, RPC = CTA / TPR;
  constexpr int V = VEC ? (sizeof(TX) == 4 ? 4 : 8) : 1;
  constexpr int NV = E / V;
  constexpr int NW = TPR > 32 ? TPR / 32 : 1;
  constexpr int AE = SMEM ? 1 : E;
  extern __shared__ float acc_s[];                              // SMEM: [2][TPR * E]; else [RPC][2][TPR * E] if RPC > 1
  __shared__ float slots[2 * RPC * 3 * NW];
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const int rows = a.rows, d = a.d;
  const float inv_d = 1.0f / (float)d;
  const bool want_w = a.dw || a.db;
  using PX = Pack<TX, V>;
  using PY = Pack<TY, V>;
  float w[AE], dw[AE], db[AE];
#pragma unroll
  for (int e = 0; e < AE; ++e) { w[e] = 1.0f; dw[e] = db[e] = 0.f; }
  if (!SMEM) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int u = 0; u < V; ++u) {
        const int c = (i * TPR + t) * V + u;
        if (a.w && c < d) w[(i * V + u) % AE] = load_any(a.w, a.tw, c);
      }
  } else {
    for (int i = t; i < 2 * TPR * E; i += CTA) acc_s[i] = 0.f;
    __syncthreads();
  }
  PX xn[NV];
  PY yn[NV];
  float mean_n = 0.f, rstd_n = 0.f;
  auto fetch = [&](int row) {
    const TX* xr = static_cast<const TX*>(a.x) + (size_t)row * a.ldx;
    const TY* yr = static_cast<const TY*>(a.dy) + (size_t)row * a.lddy;
    const bool in = row < rows;
    mean_n = in ? __ldg(a.mean + row) : 0.f;
    rstd_n = in ? __ldg(a.rstd + row) : 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + t) * V;
      if (in && c < d) {
        xn[i] = *reinterpret_cast<const PX*>(xr + c);
        yn[i] = *reinterpret_cast<const PY*>(yr + c);
      } else {
        xn[i] = PX{};
        yn[i] = PY{};
      }
    }
  };
  int base = blockIdx.x * RPC, flip = 0;
  if (base < rows) fetch(base + sub);
  for (; base < rows; base += gridDim.x * RPC, flip ^= 1) {
    const int row = base + sub;
    const bool live = row < rows;
    const float mean = mean_n, rstd = rstd_n;
    PX xp[NV];
    PY yp[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) { xp[i] = xn[i]; yp[i] = yn[i]; }
    if (!SMEM) fetch(row + gridDim.x * RPC);
    float q[3] = {0.f, 0.f, 0.f};                               // sums of x - mean, w dy, w dy (x - mean)
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + t) * V;
      if (c < d) {
#pragma unroll
        for (int u = 0; u < V; ++u) {
          const float xc = Conv<TX>::get(xp[i].v[u]) - mean;
          const float we = SMEM ? (a.w ? load_any(a.w, a.tw, c + u) : 1.0f) : w[(i * V + u) % AE];
          const float g = Conv<TY>::get(yp[i].v[u]) * we;
          q[0] += xc;
          q[1] += g;
          q[2] = fmaf(g, xc, q[2]);
        }
      }
    }
    group_sum<TPR, 3>(q, slots + (flip * RPC + sub) * 3 * NW, t, 1 + sub);
    const float c0 = __fmul_rn(q[0], inv_d), c1 = __fmul_rn(q[1], inv_d), c2 = rstd * fmaf(-c0, c1, q[2] * inv_d);
    TX* dxr = static_cast<TX*>(a.dx) + (size_t)row * a.lddx;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + t) * V;
      if (live && c < d) {
        PX o;
#pragma unroll
        for (int u = 0; u < V; ++u) {
          const float xhat = (Conv<TX>::get(xp[i].v[u]) - mean - c0) * rstd;
          const float dy = Conv<TY>::get(yp[i].v[u]);
          const float we = SMEM ? (a.w ? load_any(a.w, a.tw, c + u) : 1.0f) : w[(i * V + u) % AE];
          o.v[u] = Conv<TX>::put(rstd * (fmaf(dy, we, -c1) - xhat * c2));
          if (SMEM) {
            acc_s[c + u] = fmaf(dy, xhat, acc_s[c + u]);
            acc_s[TPR * E + c + u] += dy;
          } else {
            dw[(i * V + u) % AE] = fmaf(dy, xhat, dw[(i * V + u) % AE]);
            db[(i * V + u) % AE] += dy;
          }
        }
        if (a.dx) *reinterpret_cast<PX*>(dxr + c) = o;
      }
    }
    if (SMEM) fetch(row + gridDim.x * RPC);
  }
  if (!want_w) return;
  float* part = a.part + (size_t)blockIdx.x * 2 * d;
  if (SMEM) {
    __syncthreads();                                            // (columns are stored in another order than they were summed)
    for (int c = t; c < d; c += CTA) { part[c] = acc_s[c]; part[d + c] = acc_s[TPR * E + c]; }
  } else if (RPC == 1) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int u = 0; u < V; ++u) {
        const int c = (i * TPR + t) * V + u;
        if (c < d) { part[c] = dw[(i * V + u) % AE]; part[d + c] = db[(i * V + u) % AE]; }
      }
  } else {                                                      // the CTA's row groups, added in order
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int u = 0; u < V; ++u) {
        const int c = (i * TPR + t) * V + u;
        acc_s[(sub * 2 + 0) * TPR * E + c] = dw[(i * V + u) % AE];
        acc_s[(sub * 2 + 1) * TPR * E + c] = db[(i * V + u) % AE];
      }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * TPR * E; c += CTA) {
      const int which = c / (TPR * E), col = c % (TPR * E);
      float s = 0.f;
      for (int g = 0; g < RPC; ++g) s += acc_s[(g * 2 + which) * TPR * E + col];
      if (col < d) part[(size_t)which * d + col] = s;
    }
  }
}

// long rows: dx and the row offsets c0, then the columns' sums over chunks of rows
template <class TX, class TY>
__global__ void __launch_bounds__(1024) k_norm_bwd_long(const NormArgs a) {
  __shared__ float slots[2][96];
  const int t = threadIdx.x;
  const double inv_d = 1.0 / (double)a.d;
  int flip = 0;
  for (int row = blockIdx.x; row < a.rows; row += gridDim.x, flip ^= 1) {
    const TX* xr = static_cast<const TX*>(a.x) + (size_t)row * a.ldx;
    const TY* yr = static_cast<const TY*>(a.dy) + (size_t)row * a.lddy;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float q[3] = {0.f, 0.f, 0.f};
    for (int c = t; c < a.d; c += 1024) {
      const float xc = Conv<TX>::get(xr[c]) - mean;
      const float g = Conv<TY>::get(yr[c]) * (a.w ? load_any(a.w, a.tw, c) : 1.0f);
      q[0] += xc;
      q[1] += g;
      q[2] = fmaf(g, xc, q[2]);
    }
    group_sum<1024, 3>(q, slots[flip], t, 1);
    const float c0 = (float)(q[0] * inv_d), c1 = (float)(q[1] * inv_d);
    const float c2 = rstd * fmaf(-c0, c1, (float)(q[2] * inv_d));
    if (t == 0) a.shift[row] = c0;
    if (!a.dx) continue;
    TX* dxr = static_cast<TX*>(a.dx) + (size_t)row * a.lddx;
    for (int c = t; c < a.d; c += 1024) {
      const float xhat = (Conv<TX>::get(xr[c]) - mean - c0) * rstd;
      const float g = Conv<TY>::get(yr[c]) * (a.w ? load_any(a.w, a.tw, c) : 1.0f);
      dxr[c] = Conv<TX>::put(rstd * (g - c1 - xhat * c2));
    }
  }
}
template <class TX, class TY>
__global__ void __launch_bounds__(256) k_norm_bwd_cols(const NormArgs a, int parts) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= a.d) return;
  const int per = (a.rows + parts - 1) / parts;
  const int r0 = blockIdx.y * per, r1 = min(a.rows, r0 + per);
  float dw = 0.f, db = 0.f;
  for (int row = r0; row < r1; ++row) {
    const float dy = Conv<TY>::get(static_cast<const TY*>(a.dy)[(size_t)row * a.lddy + c]);
    const float xc = Conv<TX>::get(static_cast<const TX*>(a.x)[(size_t)row * a.ldx + c]) - a.mean[row];
    dw = fmaf(dy, (xc - a.shift[row]) * a.rstd[row], dw);
    db += dy;
  }
  a.part[((size_t)blockIdx.y * 2 + 0) * a.d + c] = dw;
  a.part[((size_t)blockIdx.y * 2 + 1) * a.d + c] = db;
}

// dw[c], db[c] = sum over the CTAs' partial sums: a CTA takes 32 columns of the 2 d, eight warps an eighth of the
// partial rows each, and the eight sums are added in order
__global__ void __launch_bounds__(256) k_norm_bwd_join(const NormArgs a, int parts) {
  __shared__ float s[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t col = (int64_t)blockIdx.x * 32 + lane, n = 2 * (int64_t)a.d;
  float v = 0.f;
  if (col < n) {
    const float* p = a.part + col;
#pragma unroll 4
    for (int g = warp; g < parts; g += 8) v += p[(size_t)g * n];
  }
  s[warp][lane] = v;
  __syncthreads();
  if (warp == 0 && col < n) {
    float r = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) r += s[i][lane];
    if (col < a.d) { if (a.dw) store_any(a.dw, a.tw, col, r); }
    else if (a.db) store_any(a.db, a.tw, col - a.d, r);
  }
}

constexpr int kSms = 148;
constexpr int kLongParts = 32;

inline bool aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) % bytes) == 0; }

// CTAs of a launch: as many as are resident at once, or as the rows need
inline int grid_for(int rows, int rpc, int per_sm) { return std::max(1, std::min((rows + rpc - 1) / rpc, kSms * per_sm)); }

inline int bwd_threads(int d) { return d <= 2048 ? 256 : d <= 4096 ? 512 : 1024; }
inline int bwd_rpc(int d) { return d <= 64 ? 32 : d <= 256 ? 8 : d <= 1024 ? 2 : 1; }

template <class TX, class TY>
bool vec_ok(const NormArgs& a, bool bwd) {
  constexpr int V = sizeof(TX) == 4 ? 4 : 8;
  if (a.d % V || a.ldx % V || !aligned(a.x, V * sizeof(TX))) return false;
  if (!bwd) return a.ldy % V == 0 && aligned(a.y, V * sizeof(TY));
  return a.lddy % V == 0 && aligned(a.dy, V * sizeof(TY)) && (!a.dx || (a.lddx % V == 0 && aligned(a.dx, V * sizeof(TX))));
}

template <class TX, class TY, int TPR, int E, bool RES>
cudaError_t fwd_t(const NormArgs& a, cudaStream_t st) {
  constexpr int cta = norm_cta<TPR>, rpc = cta / TPR;
  const int grid = grid_for(a.rows, rpc, std::max(1, 2048 / cta / (E > 8 ? 2 : 1)));
  if (RES || vec_ok<TX, TY>(a, false)) k_norm<TX, TY, TPR, E, true, RES><<<grid, cta, 0, st>>>(a);
  else k_norm<TX, TY, TPR, E, false, false><<<grid, cta, 0, st>>>(a);
  return cudaGetLastError();
}

template <class TX, class TY, bool RES>
cudaError_t fwd(const NormArgs& a, cudaStream_t st) {
  if (a.d <= 64) return fwd_t<TX, TY, 8, 8, RES>(a, st);
  if (a.d <= 256) return fwd_t<TX, TY, 32, 8, RES>(a, st);
  if (a.d <= 1024) return fwd_t<TX, TY, 128, 8, RES>(a, st);
  if (a.d <= 2048) return fwd_t<TX, TY, 256, 8, RES>(a, st);
  if (a.d <= 4096) return fwd_t<TX, TY, 512, 8, RES>(a, st);
  if (a.d <= 8192) return fwd_t<TX, TY, 1024, 8, RES>(a, st);
  if (a.d <= 16384) return fwd_t<TX, TY, 1024, 16, RES>(a, st);
  if (RES) return cudaErrorInvalidValue;
  k_norm_long<TX, TY><<<std::min(a.rows, 2 * kSms), 1024, 0, st>>>(a);
  return cudaGetLastError();
}

template <class TX, class TY, int TPR, int E, bool VEC, bool SMEM>
cudaError_t bwd_k(const NormArgs& a, int grid, cudaStream_t st) {
  constexpr int cta = norm_cta<TPR>, rpc = cta / TPR;
  constexpr int smem = SMEM ? 2 * TPR * E * 4 : (rpc > 1 ? rpc * 2 * TPR * E * 4 : 0);
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(k_norm_bwd<TX, TY, TPR, E, VEC, SMEM>,
                                               cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
  }
  k_norm_bwd<TX, TY, TPR, E, VEC, SMEM><<<grid, cta, smem, st>>>(a);
  return cudaGetLastError();
}

template <class TX, class TY, int TPR, int E, bool SMEM>
cudaError_t bwd_t(const NormArgs& a, int grid, cudaStream_t st) {
  return vec_ok<TX, TY>(a, true) ? bwd_k<TX, TY, TPR, E, true, SMEM>(a, grid, st)
                                 : bwd_k<TX, TY, TPR, E, false, SMEM>(a, grid, st);
}

template <class TX, class TY>
cudaError_t bwd(const NormArgs& a, cudaStream_t st) {
  int parts = norm_parts(a.rows, a.d);
  cudaError_t e = cudaSuccess;
  if (a.rows > 0) {
    if (a.d <= 64) e = bwd_t<TX, TY, 8, 8, false>(a, parts, st);
    else if (a.d <= 256) e = bwd_t<TX, TY, 32, 8, false>(a, parts, st);
    else if (a.d <= 1024) e = bwd_t<TX, TY, 128, 8, false>(a, parts, st);
    else if (a.d <= 2048) e = bwd_t<TX, TY, 256, 8, false>(a, parts, st);
    else if (a.d <= 4096) e = bwd_t<TX, TY, 512, 8, false>(a, parts, st);
    else if (a.d <= 8192) e = bwd_t<TX, TY, 1024, 8, false>(a, parts, st);
    else if (a.d <= 16384) e = bwd_t<TX, TY, 1024, 16, true>(a, parts, st);
    else {
      k_norm_bwd_long<TX, TY><<<std::min(a.rows, 2 * kSms), 1024, 0, st>>>(a);
      e = cudaGetLastError();
      if (e == cudaSuccess && (a.dw || a.db)) {
        k_norm_bwd_cols<TX, TY><<<dim3((a.d + 255) / 256, parts), 256, 0, st>>>(a, parts);
        e = cudaGetLastError();
      }
    }
    if (e != cudaSuccess) return e;
  } else {
    parts = 0;                                     // no rows: the gradients are zeros
  }
  if (!a.dw && !a.db) return cudaSuccess;
  k_norm_bwd_join<<<(int)((2 * (int64_t)a.d + 31) / 32), 256, 0, st>>>(a, parts);
  return cudaGetLastError();
}

}  // namespace

bool norm_is_long(int d) { return d > 16384; }

int norm_parts(int rows, int d) {
  if (norm_is_long(d)) return std::max(1, std::min(rows, kLongParts));
  return grid_for(rows, bwd_rpc(d), std::max(1, 768 / bwd_threads(d)));
}

cudaError_t launch_norm(const NormArgs& a, cudaStream_t st) {
  if (a.rows <= 0) return cudaSuccess;
  if (a.res) return a.tx == SDS_F32 && a.ty == SDS_BF16 ? fwd<float, Bf16, true>(a, st) : cudaErrorInvalidValue;
  if (a.tx == SDS_F32 && a.ty == SDS_F32) return fwd<float, float, false>(a, st);
  if (a.tx == SDS_F32 && a.ty == SDS_BF16) return fwd<float, Bf16, false>(a, st);
  if (a.tx == SDS_F32 && a.ty == SDS_F16) return fwd<float, F16, false>(a, st);
  if (a.tx == SDS_BF16 && a.ty == SDS_BF16) return fwd<Bf16, Bf16, false>(a, st);
  if (a.tx == SDS_F16 && a.ty == SDS_F16) return fwd<F16, F16, false>(a, st);
  return cudaErrorInvalidValue;
}

cudaError_t launch_norm_backward(const NormArgs& a, cudaStream_t st) {
  if (a.tx == SDS_F32 && a.ty == SDS_F32) return bwd<float, float>(a, st);
  if (a.tx == SDS_F32 && a.ty == SDS_BF16) return bwd<float, Bf16>(a, st);
  if (a.tx == SDS_F32 && a.ty == SDS_F16) return bwd<float, F16>(a, st);
  if (a.tx == SDS_BF16 && a.ty == SDS_BF16) return bwd<Bf16, Bf16>(a, st);
  if (a.tx == SDS_F16 && a.ty == SDS_F16) return bwd<F16, F16>(a, st);
  return cudaErrorInvalidValue;
}

}  // namespace sds
