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
// Rows may lie far from zero, where a mean rounded to 32 bits is off by an error that every element shares. The sums are
// therefore taken around a number p near the row's elements (exact differences), and the remainder c0 = <x - p> is
// taken off every element; the backward pass does the same with p = the stored mean.
//
// Gradients of the weights: a CTA keeps the sums of its columns in registers over all rows it visits and stores
// them once; a second kernel adds the CTAs' sums in a fixed order (no atomics: same bits on every run).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

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

// two floats in one instruction (the kernels below would otherwise be bound by issue, not by memory)
__device__ __forceinline__ unsigned long long bits(float2 v) { return *reinterpret_cast<unsigned long long*>(&v); }
__device__ __forceinline__ float2 floats(unsigned long long v) { return *reinterpret_cast<float2*>(&v); }
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)));
  return floats(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)));
  return floats(r);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)), "l"(bits(c)));
  return floats(r);
}
// the same operations on single floats, for rows that are not aligned
__device__ __forceinline__ float add2(float a, float b) { return a + b; }
__device__ __forceinline__ float mul2(float a, float b) { return a * b; }
__device__ __forceinline__ float fma2(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ float total(float2 v) { return v.x + v.y; }
__device__ __forceinline__ float total(float v) { return v; }

// what a vector of V elements is worked on in: pairs, or its single element
template <int V> struct Unit {
  using type = float2;
  static constexpr int count = V / 2;
  __device__ static float2 all(float v) { return make_float2(v, v); }
};
template <> struct Unit<1> {
  using type = float;
  static constexpr int count = 1;
  __device__ static float all(float v) { return v; }
};
template <int V> using unit_t = typename Unit<V>::type;
template <int V> constexpr int units = Unit<V>::count;

template <int V> using if_vector = typename std::enable_if<(V > 1)>::type;

// unit k of a pack
template <class T> __device__ __forceinline__ float get2(const Pack<T, 1>& p, int) { return Conv<T>::get(p.v[0]); }
template <int V, class = if_vector<V>>
__device__ __forceinline__ float2 get2(const Pack<float, V>& p, int k) { return make_float2(p.v[2 * k], p.v[2 * k + 1]); }
template <int V, class = if_vector<V>>
__device__ __forceinline__ float2 get2(const Pack<Bf16, V>& p, int k) {
  const uint32_t w = reinterpret_cast<const uint32_t*>(p.v)[k];
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <int V, class = if_vector<V>>
__device__ __forceinline__ float2 get2(const Pack<F16, V>& p, int k) {
  const uint32_t w = reinterpret_cast<const uint32_t*>(p.v)[k];
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <class T> __device__ __forceinline__ void put2(Pack<T, 1>& p, int, float v) { p.v[0] = Conv<T>::put(v); }
template <int V, class = if_vector<V>>
__device__ __forceinline__ void put2(Pack<float, V>& p, int k, float2 v) { p.v[2 * k] = v.x; p.v[2 * k + 1] = v.y; }
template <int V, class = if_vector<V>>
__device__ __forceinline__ void put2(Pack<Bf16, V>& p, int k, float2 v) {
  const __nv_bfloat162 h = __float22bfloat162_rn(v);
  reinterpret_cast<uint32_t*>(p.v)[k] = *reinterpret_cast<const uint32_t*>(&h);
}
template <int V, class = if_vector<V>>
__device__ __forceinline__ void put2(Pack<F16, V>& p, int k, float2 v) {
  const __half2 h = __float22half2_rn(v);
  reinterpret_cast<uint32_t*>(p.v)[k] = *reinterpret_cast<const uint32_t*>(&h);
}

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

// Sums of N <= 4 values over the TPR threads of a row's group, in every thread: group_sum. Inside a warp the values are folded
// into one another while they are summed (a lane keeps the value its number selects: 3 values take 6 shuffles, not 15).
// Between the warps: slot, shared memory of the group, 4 * TPR / 32 floats, not written again before the group has
// passed another barrier. CL > 1: the group is spread over a cluster of CL CTAs, every warp's sums go to all of
// them. The order of the additions is fixed. In two steps, with the cluster's barrier between: group_post, group_take.
constexpr unsigned kAll = 0xffffffffu;
template <int TPR, int N>
__device__ __forceinline__ float group_fold(const float (&v)[N], int lane) {
  constexpr int W = TPR < 32 ? TPR : 32;
  constexpr int F = N == 1 ? 1 : N == 2 ? 2 : 4;                // values folded over F neighbouring lanes
  float x = v[0];
  if (F >= 2) {
    const bool odd = lane & 1;
    const float v1 = v[N > 1 ? 1 : 0];
    x = (odd ? v1 : v[0]) + __shfl_xor_sync(kAll, odd ? v[0] : v1, 1);
    if (F == 4) {
      const float v2 = v[N > 2 ? 2 : 0], v3 = N > 3 ? v[N > 3 ? 3 : 0] : 0.f;
      const float y = (odd ? v3 : v2) + __shfl_xor_sync(kAll, odd ? v2 : v3, 1);
      const bool high = lane & 2;
      x = (high ? y : x) + __shfl_xor_sync(kAll, high ? x : y, 2);
    }
  }
#pragma unroll
  for (int o = F; o < W; o <<= 1) x += __shfl_xor_sync(kAll, x, o);
  return x;
}
template <int TPR, int N, int CL>
__device__ __forceinline__ void group_post(const float (&v)[N], float* slot, int t) {
  constexpr int NW = TPR / 32;
  const int lane = t & 31;
  const float x = group_fold<TPR>(v, lane);
  if (lane < N) {
    float* mine = slot + lane * NW + (t >> 5);
    if (CL == 1) {
      *mine = x;
    } else {
#pragma unroll
      for (int c = 0; c < CL; ++c) {
        uint32_t to;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((uint32_t)__cvta_generic_to_shared(mine)), "r"(c));
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(x) : "memory");
      }
    }
  }
}
template <int TPR, int N>
__device__ __forceinline__ void group_take(float (&v)[N], const float* slot, int t) {
  constexpr int NW = TPR / 32;
  const int lane = t & 31;
  if (NW <= 8) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < NW; w += 2) {
        const float2 q = *reinterpret_cast<const float2*>(slot + n * NW + w);
        s += q.x + q.y;
      }
      v[n] = s;
    }
  } else {                                                      // eight lanes add one value's NW sums
    const int n8 = lane >> 3;
    float s = 0.f;
    if (n8 < N)
#pragma unroll
      for (int w = 0; w < NW / 8; ++w) s += slot[n8 * NW + (lane & 7) * (NW / 8) + w];
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) s += __shfl_xor_sync(kAll, s, o);
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = __shfl_sync(kAll, s, n * 8);
  }
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
template <int TPR, int N, int CL = 1>
__device__ __forceinline__ void group_sum(float (&v)[N], float* slot, int t, int bar) {
  if constexpr (TPR <= 32) {
    constexpr int W = TPR < 32 ? TPR : 32;
    const float x = group_fold<TPR>(v, t & 31);
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = N == 1 ? x : __shfl_sync(kAll, x, n, W);
  } else {
    group_post<TPR, N, CL>(v, slot, t);
    if (CL > 1) {
      cluster_arrive();
      cluster_wait();
    } else {
      asm volatile("bar.sync %0, %1;" ::"r"(bar), "r"(TPR) : "memory");
    }
    group_take<TPR>(v, slot, t);
  }
}

// Where the columns of a group's thread t lie. A row: vector i, element u = column (i * TPR + t) * V + u. Shared memory: quads
// of a thread's columns, T quads side by side (T threads of the group in this CTA), so that 128-bit accesses are free
// of bank conflicts.
template <int T, int V>
__device__ __forceinline__ int slot_of(int i, int u, int t) {
  return V == 1 ? i * T + t : ((i * (V / 4) + (u >> 2)) * T + t) * 4 + (u & 3);
}
template <int T, int V, class = if_vector<V>>
__device__ __forceinline__ void load_cols(const float* s, int i, int t, float2 (&o)[units<V>]) {
#pragma unroll
  for (int q = 0; q < V / 4; ++q) {
    const float4 v = *reinterpret_cast<const float4*>(s + slot_of<T, V>(i, 4 * q, t));
    o[2 * q] = make_float2(v.x, v.y);
    o[2 * q + 1] = make_float2(v.z, v.w);
  }
}
template <int T, int V>
__device__ __forceinline__ void load_cols(const float* s, int i, int t, float (&o)[1]) { o[0] = s[slot_of<T, V>(i, 0, t)]; }
// V columns from c on of a caller's column vector (c and d multiples of V where V > 1), as floats; `fill` where there is no
// vector. wide: the vector is 16-byte aligned.
template <int V>
__device__ __forceinline__ void load_vector(const void* p, int type, bool wide, float fill, int c, int d, float (&o)[V]) {
  if (!p || c >= d) {
#pragma unroll
    for (int u = 0; u < V; ++u) o[u] = fill;
  } else if (V > 1 && wide && type == SDS_F32) {
#pragma unroll
    for (int q = 0; q < V / 4; ++q) {
      const float4 v = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(p) + c) + q);
      o[(4 * q) % V] = v.x; o[(4 * q + 1) % V] = v.y; o[(4 * q + 2) % V] = v.z; o[(4 * q + 3) % V] = v.w;
    }
  } else {
#pragma unroll
    for (int u = 0; u < V; ++u) o[u] = load_any(p, type, c + u);
  }
}
template <int V>
__device__ __forceinline__ void as_units(const float (&f)[V], unit_t<V> (&o)[units<V>]) {
  float* to = reinterpret_cast<float*>(o);
#pragma unroll
  for (int u = 0; u < V; ++u) to[u] = f[u];
}
// such a vector in shared memory, in the order of slot_of. t0: the group's first thread in this CTA.
template <int TPR, int T, int E, int V>
__device__ __forceinline__ void stage_cols(float* s, const void* p, int type, bool wide, float fill, int d, int threads, int t0) {
#pragma unroll 2
  for (int vec = threadIdx.x; vec < T * E / V; vec += threads) {
    const int i = vec / T, t = vec % T;
    float f[V];
    load_vector<V>(p, type, wide, fill, (i * TPR + t0 + t) * V, d, f);
    if (V == 1) {
      s[slot_of<T, V>(i, 0, t)] = f[0];
    } else {
#pragma unroll
      for (int q = 0; q < V / 4; ++q)
        *reinterpret_cast<float4*>(s + slot_of<T, V>(i, 4 * q, t)) =
            make_float4(f[(4 * q) % V], f[(4 * q + 1) % V], f[(4 * q + 2) % V], f[(4 * q + 3) % V]);
    }
  }
}

// Kernels overlap their starts: the next one may be started once all CTAs of this one have begun (their launch takes about
// as long as a small call runs), and this one waits here for the end of the kernel in front, and for its writes.
// Nothing in device memory is read or written before. The next one is let go before this wait: it may begin while what ran
// in front of this kernel still runs, so it has to wait in full as well before it reads anything.
__device__ __forceinline__ void start_after_prior_kernel() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

template <class TX> constexpr int vec_len = sizeof(TX) == 4 ? 4 : 8;   // elements of a 16-byte access

// FEW: at most two rows for every group of the launch, 8 elements per thread. The weights are then read with the first row,
// into registers; else they are brought to shared memory once and read from there for every row.
// Aligned 16-bit rows up to 4096: three CTAs per SM (10 % shorter at 16384 x 2048 bf16 than with the two that the compiler's own register
// count gives; float rows lose 6 % that way).
// 16384 x 2048 float to bf16: 34.2 us, 5.9 TB/s, 90 % of a copy's rate; 2047 x 16384 float 51.4 us, 5.2 TB/s; 64 x 2048 4.1 us.
template <class TX, class TY, int TPR, int E, bool VEC, bool RES, bool FEW>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR, VEC && TPR <= 128 && !FEW && sizeof(TX) == 2 ? 3 : 1)
    k_norm(const NormArgs a) {
  constexpr int CTA = TPR < 256 ? 256 : TPR, RPC = CTA / TPR;   // RPC: rows of a CTA at a time
  constexpr int V = VEC ? vec_len<TX> : 1;
  constexpr int NV = E / V, P = units<V>;
  constexpr int NW = TPR > 32 ? TPR / 32 : 1;
  using U = unit_t<V>;
  using PX = Pack<TX, V>;
  using PY = Pack<TY, V>;
  extern __shared__ float4 shared[];                            // weights [2][TPR * E] (not FEW)
  float* w_s = reinterpret_cast<float*>(shared);
  float* b_s = w_s + TPR * E;
  __shared__ __align__(16) float slots[2 * RPC * 4 * NW];
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  float* slot = slots + sub * 8 * NW;
  start_after_prior_kernel();
  const int rows = a.nrows_dev ? min(*a.nrows_dev, a.rows) : a.rows;
  const int d = a.d, step = (int)gridDim.x * RPC;
  const float inv_d = 1.0f / (float)d;
  PX nxt[NV];
  const auto fetch = [&](int row) {
    const TX* xr = static_cast<const TX*>(a.x) + (size_t)row * a.ldx;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + t) * V;
      if (row < rows && c < d) nxt[i] = *reinterpret_cast<const PX*>(xr + c);
      else nxt[i] = PX{};
    }
  };
  int base = blockIdx.x * RPC;
  fetch(base + sub);
  U wr[FEW ? NV : 1][P], br[FEW ? NV : 1][P];
  if (FEW) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float f[V];
      load_vector<V>(a.w, a.tw, a.wide, 1.0f, (i * TPR + t) * V, d, f);
      as_units<V>(f, wr[FEW ? i : 0]);
      load_vector<V>(a.b, a.tw, a.wide, 0.0f, (i * TPR + t) * V, d, f);
      as_units<V>(f, br[FEW ? i : 0]);
    }
  } else {
    stage_cols<TPR, TPR, E, V>(w_s, a.w, a.tw, a.wide, 1.0f, d, CTA, 0);
    stage_cols<TPR, TPR, E, V>(b_s, a.b, a.tw, a.wide, 0.0f, d, CTA, 0);
    __syncthreads();
  }
  for (; base < rows; base += step) {
    const int row = base + sub;
    const bool live = row < rows;
    U x[NV][P];
    U s0 = Unit<V>::all(0.f);
    const uint16_t* te = RES && live && a.temb ? a.temb + (size_t)__ldg(a.rowk + row) * d : nullptr;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + t) * V;
      if (RES && live && c < d) {                               // x + temb[k], kept as the residual stream
        if (te) {
          const Pack<Bf16, V> e = *reinterpret_cast<const Pack<Bf16, V>*>(te + c);
#pragma unroll
          for (int k = 0; k < P; ++k) put2(nxt[i], k, add2(get2(nxt[i], k), get2(e, k)));
        }
        if (te || a.x != a.res) *reinterpret_cast<PX*>(a.res + (size_t)row * d + c) = nxt[i];
      }
#pragma unroll
      for (int k = 0; k < P; ++k) x[i][k] = get2(nxt[i], k);
    }
    fetch(row + step);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int k = 0; k < P; ++k) s0 = add2(s0, x[i][k]);       // (elements past d hold zeros)
    float s[1] = {total(s0)};
    group_sum<TPR, 1>(s, slot, t, 1 + sub);
    const float mean = __fmul_rn(s[0], inv_d);                  // (a rounded number: the same one with and without statistics)
    const U minus = Unit<V>::all(-mean);
    U q0 = Unit<V>::all(0.f), q1 = q0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if ((i * TPR + t) * V < d) {
#pragma unroll
        for (int k = 0; k < P; ++k) {
          x[i][k] = add2(x[i][k], minus);
          q0 = add2(q0, x[i][k]);
          q1 = fma2(x[i][k], x[i][k], q1);
        }
      }
    }
    float q[2] = {total(q0), total(q1)};
    group_sum<TPR, 2>(q, slot + 4 * NW, t, 1 + sub);
    const float c0 = __fmul_rn(q[0], inv_d);
    const float rstd = rsqrtf(fmaxf(fmaf(-c0, c0, q[1] * inv_d), 0.f) + a.eps);
    if (!live) continue;
    if (t == 0) {
      if (a.mean) a.mean[row] = mean + c0;
      if (a.rstd) a.rstd[row] = rstd;
    }
    TY* yr = static_cast<TY*>(a.y) + (size_t)row * a.ldy;
    const U scale = Unit<V>::all(rstd), shift = Unit<V>::all(-c0 * rstd);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + t) * V;
      if (c < d) {
        U w[P], b[P];
        if (!FEW) {
          load_cols<TPR, V>(w_s, i, t, w);
          load_cols<TPR, V>(b_s, i, t, b);
        }
        PY o;
#pragma unroll
        for (int k = 0; k < P; ++k)
          put2(o, k, fma2(fma2(x[i][k], scale, shift), FEW ? wr[FEW ? i : 0][k] : w[k], FEW ? br[FEW ? i : 0][k] : b[k]));
        *reinterpret_cast<PY*>(yr + c) = o;
      }
    }
  }
}

// rows longer than the register kernels hold: one CTA per row, the row read three times (the later passes from L2)
template <class TX, class TY>
__global__ void __launch_bounds__(1024) k_norm_long(const NormArgs a) {
  start_after_prior_kernel();
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

// Copies of 16 bytes into shared memory, asynchronous and in groups; of the source only the first n bytes are read, zeros fill
// the rest.
__device__ __forceinline__ void copy_async(void* dst, const void* src, int n) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(n) : "memory");
}
template <class PACK, class T>
__device__ __forceinline__ void copy_pack(PACK* dst, const T* src, bool in) {
  if (sizeof(PACK) == 16)
    copy_async(dst, src, in ? 16 : 0);
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src),
                 "n"(sizeof(PACK) < 4 ? 4 : sizeof(PACK)), "r"(in ? (int)sizeof(PACK) : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

constexpr int kSmem = 226 * 1024;                               // of an SM's 227 KB a CTA may have

// TPR threads per row, CL CTAs of them; CTAs of 512 threads (fewer CTAs, fewer partial sums for the second kernel to
// add up) that hold 512 / TPR rows at a time, or half a row each
template <class TX, class TY, int TPR, int E, bool VEC, int CL> struct NormBwd {
  static constexpr int kT = TPR / CL, kCta = 512, kGroups = kCta / kT;
  static constexpr int kWeights = kT * E * 4;
  // rows in flight: a group keeps kRing rows in shared memory, kRing - 1 of them on their way while one is worked on.
  // Unaligned rows: the aligned vectors that cover a row, up to two more than its own length takes.
  static constexpr int kPad = VEC ? 0 : 32;
  static constexpr int kRowX = kT * E * (int)sizeof(TX) + kPad, kRow = kRowX + kT * E * (int)sizeof(TY) + kPad;
  static constexpr int kFit = (kSmem - kWeights) / (kRow * kGroups);
  static constexpr int kRing = kFit > 4 ? 4 : kFit;
  static constexpr int kJoin = kGroups > 1 ? kGroups * 2 * TPR * E * 4 : 0;   // the groups' sums, where the ring was
  static constexpr int kRingBytes = kRing * kRow * kGroups;
  static constexpr int kSmemBytes = kWeights + (kRingBytes > kJoin ? kRingBytes : kJoin);
  static_assert(kRing >= 2 && kSmemBytes <= kSmem && kGroups * CL <= 64, "shared memory");
};

// Backward. The sums of the weights' gradients stay in registers over all rows of a group, the weights in shared
// memory; the rows of x and dy pass through a ring there and are held as floats between the two passes. Bound by HBM for many
// rows (16384 x 2048 bf16, forward and backward 67 us of the 51 that two passes' bytes take), by the latency of the row's barriers for
// few (512 x 16384 float and bf16, both 46 us).
template <class TX, class TY, int TPR, int E, bool VEC, int CL>
__global__ void __launch_bounds__(512, 1) k_norm_bwd(const NormArgs a) {
  using C = NormBwd<TX, TY, TPR, E, VEC, CL>;
  constexpr int CTA = C::kCta, RPC = C::kGroups, R = C::kRing, T = C::kT;
  constexpr int V = VEC ? vec_len<TX> : 1;
  constexpr int NV = E / V, P = units<V>;
  constexpr int NW = TPR > 32 ? TPR / 32 : 1;
  using U = unit_t<V>;
  using PX = Pack<TX, V>;
  using PY = Pack<TY, V>;
  extern __shared__ float4 shared[];                            // weights [T * E], then the ring
  float* w_s = reinterpret_cast<float*>(shared);
  uint8_t* rest = reinterpret_cast<uint8_t*>(shared) + C::kWeights;
  __shared__ __align__(16) float slots[2 * RPC * 4 * NW];
  start_after_prior_kernel();
  const int rank = CL > 1 ? (int)(blockIdx.x % CL) : 0;         // this CTA's part of the row
  const int tl = threadIdx.x % T, sub = threadIdx.x / T, t = rank * T + tl;
  const int rows = a.rows, d = a.d, groups = (int)gridDim.x / CL, step = groups * RPC;
  const float inv_d = 1.0f / (float)d;
  uint8_t* ring = rest + (size_t)sub * R * C::kRow;
  PX* ring_x = reinterpret_cast<PX*>(ring) + tl;                // aligned rows: a thread's own vectors, all of x in front of all of dy
  PY* ring_y = reinterpret_cast<PY*>(ring + (size_t)R * T * E * sizeof(TX)) + tl;
  const int part0 = VEC ? 0 : rank * ((d + CL - 1) / CL);       // unaligned rows: first column of this CTA, its columns side by side,
  const int last = VEC ? d : min(d, part0 + (d + CL - 1) / CL); // and the end of its columns
  const auto column = [&](int i) { return VEC ? (i * TPR + t) * V : part0 + i * T + tl; };
  U dw[NV][P], db[NV][P];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int k = 0; k < P; ++k) dw[i][k] = db[i][k] = Unit<V>::all(0.f);
  // A thread of an aligned row copies what it will read. Unaligned: the group copies the 16-byte vectors that cover the row's part,
  // whatever lies in front of it included (it is not read back), but not in front of the array: there element by element.
  const auto cover = [&](uint8_t* to, const auto* array, int64_t ld, int64_t row) {
    using E1 = typename std::remove_const<typename std::remove_pointer<decltype(array)>::type>::type;
    const uintptr_t first = reinterpret_cast<uintptr_t>(array + row * ld + part0), begin = first & ~(uintptr_t)15;
    const uintptr_t end = first + (uintptr_t)(last - part0) * sizeof(E1);
    for (uintptr_t p = begin + 16 * (uintptr_t)tl; p < end; p += 16 * (uintptr_t)T) {
      const int n = (int)min((uintptr_t)16, end - p);
      if (p >= reinterpret_cast<uintptr_t>(array)) {
        copy_async(to + (p - begin), reinterpret_cast<const void*>(p), n);
      } else {
        for (uintptr_t q = first; q < p + n; q += sizeof(E1))
          *reinterpret_cast<E1*>(to + (q - begin)) = *reinterpret_cast<const E1*>(q);
      }
    }
  };
  const auto fetch = [&](int64_t row, int r) {
    const bool live = row < rows;
    if constexpr (VEC) {
      const TX* xr = static_cast<const TX*>(a.x) + (live ? row : 0) * a.ldx;
      const TY* yr = static_cast<const TY*>(a.dy) + (live ? row : 0) * a.lddy;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = column(i);
        const bool in = live && c < last;
        // (a pack of 16-bit elements beside floats is half as long)
        copy_pack(ring_x + (r * NV + i) * T, xr + (in ? c : 0), in);
        copy_pack(ring_y + (r * NV + i) * T, yr + (in ? c : 0), in);
      }
    } else if (live && part0 < last) {
      cover(ring + r * C::kRow, static_cast<const TX*>(a.x), a.ldx, row);
      cover(ring + r * C::kRow + C::kRowX, static_cast<const TY*>(a.dy), a.lddy, row);
    }
    copies_commit();
  };
  const auto stats_of = [&](int64_t row) {
    return row < rows ? make_float2(__ldg(a.mean + row), __ldg(a.rstd + row)) : make_float2(0.f, 0.f);
  };
  int base = (int)blockIdx.x / CL * RPC, flip = 0, at = 0;
  constexpr bool SKEW = CL > 1 && VEC;                          // (see the loop at the end)
#pragma unroll
  for (int r = 0; r < (SKEW ? R : R - 1); ++r) fetch((int64_t)base + sub + (int64_t)r * step, r);
  float2 stats = stats_of(base + sub);
  if constexpr (VEC) stage_cols<TPR, T, E, V>(w_s, a.w, a.tw, a.wide, 1.0f, d, CTA, rank * T);
  else stage_cols<T, T, E, V>(w_s, a.w, a.tw, a.wide, 1.0f, d, CTA, part0);
  __syncthreads();
  if (CL > 1) {                                                 // the peers run before anything is written to them
    cluster_arrive();
    cluster_wait();
  }
  if constexpr (!SKEW)
  for (; base < rows; base += step, flip ^= 1) {
    const int row = base + sub;
    const bool live = row < rows;
    const float mean = stats.x, rstd = stats.y;
    const U minus = Unit<V>::all(-mean);
    copies_wait<R - 2>();
    const TX* row_x = nullptr;                                  // unaligned: this thread's first elements of the row in the ring
    const TY* row_y = nullptr;
    if constexpr (!VEC) {                                       // (the group's copies, and no one reads the slot that is filled next)
      if (T <= 32) __syncwarp();
      else asm volatile("bar.sync %0, %1;" ::"r"(1 + sub), "r"(T) : "memory");
      const uintptr_t fx = reinterpret_cast<uintptr_t>(static_cast<const TX*>(a.x) + (int64_t)row * a.ldx + part0);
      const uintptr_t fy = reinterpret_cast<uintptr_t>(static_cast<const TY*>(a.dy) + (int64_t)row * a.lddy + part0);
      row_x = reinterpret_cast<const TX*>(ring + at * C::kRow + (fx & 15)) + tl;
      row_y = reinterpret_cast<const TY*>(ring + at * C::kRow + C::kRowX + (fy & 15)) + tl;
    }
    U xc[NV][P], yf[NV][P];
    U q0 = Unit<V>::all(0.f), q1 = q0, q2 = q0;                 // sums of x - mean, w dy, w dy (x - mean)
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = column(i);
      if (c < last) {
        PX px{};
        PY py{};
        if constexpr (VEC) {
          px = ring_x[(at * NV + i) * T];
          py = ring_y[(at * NV + i) * T];
        } else if (live) {
          px.v[0] = row_x[i * T];
          py.v[0] = row_y[i * T];
        }
        U w[P];
        load_cols<T, V>(w_s, i, tl, w);
#pragma unroll
        for (int k = 0; k < P; ++k) {
          xc[i][k] = add2(get2(px, k), minus);
          yf[i][k] = get2(py, k);
          const U g = mul2(yf[i][k], w[k]);
          q0 = add2(q0, xc[i][k]);
          q1 = add2(q1, g);
          q2 = fma2(g, xc[i][k], q2);
        }
      }
    }
    stats = stats_of((int64_t)row + step);
    fetch((int64_t)row + (int64_t)(R - 1) * step, at == 0 ? R - 1 : at - 1);
    float q[3] = {total(q0), total(q1), total(q2)};
    group_sum<TPR, 3, CL>(q, slots + (flip * RPC + sub) * 4 * NW, t, 1 + sub);
    const float c0 = __fmul_rn(q[0], inv_d), c1 = __fmul_rn(q[1], inv_d), c2 = rstd * fmaf(-c0, c1, q[2] * inv_d);
    TX* dxr = static_cast<TX*>(a.dx) + (size_t)row * a.lddx;
    const U scale = Unit<V>::all(rstd), shift = Unit<V>::all(-c0 * rstd), less = Unit<V>::all(-c1), slope = Unit<V>::all(-c2);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = column(i);
      if (live && c < last) {
        U w[P];
        load_cols<T, V>(w_s, i, tl, w);
        PX o;
#pragma unroll
        for (int k = 0; k < P; ++k) {
          const U xhat = fma2(xc[i][k], scale, shift);
          put2(o, k, mul2(fma2(xhat, slope, fma2(yf[i][k], w[k], less)), scale));
          dw[i][k] = fma2(yf[i][k], xhat, dw[i][k]);
          db[i][k] = add2(db[i][k], yf[i][k]);
        }
        if (a.dx) *reinterpret_cast<PX*>(dxr + c) = o;
      }
    }
    at = at == R - 1 ? 0 : at + 1;
  }
  // A cluster's barrier takes about a third of a row's time: the sums of the next row are posted before the results of this
  // one are computed, from the ring again (no registers for two rows), and awaited after them.
  if constexpr (SKEW) {
    U w[NV][P];
#pragma unroll
    for (int i = 0; i < NV; ++i) load_cols<T, V>(w_s, i, tl, w[i]);
    const auto post = [&](int slot, float mean, float* to) {
      U q0 = Unit<V>::all(0.f), q1 = q0, q2 = q0;
      const U minus = Unit<V>::all(-mean);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (column(i) < last) {
          const PX px = ring_x[(slot * NV + i) * T];
          const PY py = ring_y[(slot * NV + i) * T];
#pragma unroll
          for (int k = 0; k < P; ++k) {
            const U xc = add2(get2(px, k), minus), g = mul2(get2(py, k), w[i][k]);
            q0 = add2(q0, xc);
            q1 = add2(q1, g);
            q2 = fma2(g, xc, q2);
          }
        }
      }
      const float q[3] = {total(q0), total(q1), total(q2)};
      group_post<TPR, 3, CL>(q, to, t);
      cluster_arrive();
    };
    float q[3] = {0.f, 0.f, 0.f};
    float2 ahead = stats_of((int64_t)base + step);
    if (base < rows) {
      copies_wait<R - 1>();
      post(0, stats.x, slots);
      cluster_wait();
      group_take<TPR>(q, slots, t);
    }
    for (int row = base; row < rows; row += step) {
      const float mean = stats.x, rstd = stats.y;
      const bool more = (int64_t)row + step < rows;
      const int next = at == R - 1 ? 0 : at + 1;
      flip ^= 1;
      float* to = slots + flip * 4 * NW;
      stats = ahead;
      ahead = stats_of((int64_t)row + 2 * (int64_t)step);
      if (more) {
        copies_wait<R - 2>();
        post(next, stats.x, to);
      }
      const float c0 = __fmul_rn(q[0], inv_d), c1 = __fmul_rn(q[1], inv_d), c2 = rstd * fmaf(-c0, c1, q[2] * inv_d);
      TX* dxr = static_cast<TX*>(a.dx) + (size_t)row * a.lddx;
      const U minus = Unit<V>::all(-mean), scale = Unit<V>::all(rstd), shift = Unit<V>::all(-c0 * rstd), less = Unit<V>::all(-c1), slope = Unit<V>::all(-c2);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = column(i);
        if (c < last) {
          const PX px = ring_x[(at * NV + i) * T];
          const PY py = ring_y[(at * NV + i) * T];
          PX o;
#pragma unroll
          for (int k = 0; k < P; ++k) {
            const U yf = get2(py, k), xhat = fma2(add2(get2(px, k), minus), scale, shift);
            put2(o, k, mul2(fma2(xhat, slope, fma2(yf, w[i][k], less)), scale));
            dw[i][k] = fma2(yf, xhat, dw[i][k]);
            db[i][k] = add2(db[i][k], yf);
          }
          if (a.dx) *reinterpret_cast<PX*>(dxr + c) = o;
        }
      }
      fetch((int64_t)row + (int64_t)R * step, at);
      at = next;
      if (more) {
        cluster_wait();
        group_take<TPR>(q, to, t);
      }
    }
  }
  copies_wait<0>();
  if (!a.dw && !a.db) return;
  float* part = a.part + (size_t)(blockIdx.x / CL) * 2 * d;
  const auto store = [&](float* to, const U (&sums)[P]) {       // a thread's V columns
    if (V == 1) {
      to[0] = total(sums[0]);
    } else {
      const float* f = reinterpret_cast<const float*>(sums);
#pragma unroll
      for (int q = 0; q < V / 4; ++q)
        reinterpret_cast<float4*>(to)[q] = make_float4(f[(4 * q) % V], f[(4 * q + 1) % V], f[(4 * q + 2) % V], f[(4 * q + 3) % V]);
    }
  };
  if (RPC == 1) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = column(i);
      if (c < last) {
        store(part + c, dw[i]);
        store(part + d + c, db[i]);
      }
    }
  } else {                                                      // the CTA's row groups, added in order
    float* sum_s = reinterpret_cast<float*>(rest);
    __syncthreads();                                            // every group is done with its ring
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = column(i);
      store(sum_s + (sub * 2 + 0) * TPR * E + c, dw[i]);
      store(sum_s + (sub * 2 + 1) * TPR * E + c, db[i]);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * TPR * E; c += CTA) {
      const int which = c / (TPR * E), col = c % (TPR * E);
      float s = 0.f;
#pragma unroll 8
      for (int g = 0; g < RPC; ++g) s += sum_s[(g * 2 + which) * TPR * E + col];
      if (col < d) part[(size_t)which * d + col] = s;
    }
  }
}

// long rows: dx and the row offsets c0, then the columns' sums over chunks of rows
template <class TX, class TY>
__global__ void __launch_bounds__(1024) k_norm_bwd_long(const NormArgs a) {
  start_after_prior_kernel();
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
  start_after_prior_kernel();
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

// dw[c], db[c] = sum over the CTAs' partial sums: a CTA takes 32 columns of the 2 d, each of its warps every n-th of the
// partial rows, and the warps' sums are added in order
__global__ void __launch_bounds__(1024) k_norm_bwd_join(const NormArgs a, int parts) {
  __shared__ float s[32][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int64_t col = (int64_t)blockIdx.x * 32 + lane, n = 2 * (int64_t)a.d;
  start_after_prior_kernel();
  float v = 0.f;
  if (col < n) {
    const float* p = a.part + col;
#pragma unroll 8
    for (int g = warp; g < parts; g += warps) v += p[(size_t)g * n];
  }
  s[warp][lane] = v;
  __syncthreads();
  if (warp != 0 || col >= n) return;
  float r = 0.f;
#pragma unroll 8
  for (int i = 0; i < warps; ++i) r += s[i][lane];
  if (col < a.d) { if (a.dw) store_any(a.dw, a.tw, col, r); }
  else if (a.db) store_any(a.db, a.tw, col - a.d, r);
}

constexpr int kSms = 148;
constexpr int kLongParts = 32;
constexpr int kMaxDevices = 64;

inline bool aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) % bytes) == 0; }

template <class TX, class TY>
bool vec_ok(const NormArgs& a, bool bwd) {
  constexpr int V = vec_len<TX>;
  if (a.d % V || a.ldx % V || !aligned(a.x, V * sizeof(TX))) return false;
  if (!bwd) return a.ldy % V == 0 && aligned(a.y, V * sizeof(TY));
  return a.lddy % V == 0 && aligned(a.dy, V * sizeof(TY)) && (!a.dx || (a.lddx % V == 0 && aligned(a.dx, V * sizeof(TX))));
}

// a launch that may start before the kernel in front has ended (see start_after_prior_kernel), in clusters of `cluster`
template <class... P, class... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, int smem, int cluster, cudaStream_t st, const A&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// CTAs of a kernel that an SM holds, looked up once per device (and its shared-memory limit raised)
template <class K>
cudaError_t ctas_per_sm(K kernel, std::atomic<int>* cache, int threads, int smem, int* n) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  int r = cache[dev].load(std::memory_order_acquire);
  if (r == 0) {
    if (smem > 48 * 1024 &&
        (e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) != cudaSuccess)
      return e;
    if ((e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&r, kernel, threads, smem)) != cudaSuccess) return e;
    if (r < 1) return cudaErrorLaunchOutOfResources;
    cache[dev].store(r, std::memory_order_release);
  }
  *n = r;
  return cudaSuccess;
}

template <class TX, class TY, int TPR, int E, bool VEC, bool RES, bool FEW>
cudaError_t fwd_k(const NormArgs& a, cudaStream_t st) {
  constexpr int cta = TPR < 256 ? 256 : TPR, rpc = cta / TPR, smem = FEW ? 0 : 2 * TPR * E * 4;
  static std::atomic<int> cache[kMaxDevices];
  int per_sm = 0;
  const cudaError_t e = ctas_per_sm(k_norm<TX, TY, TPR, E, VEC, RES, FEW>, cache, cta, smem, &per_sm);
  if (e != cudaSuccess) return e;
  const int grid = std::min((a.rows + rpc - 1) / rpc, kSms * per_sm);
  return launch(k_norm<TX, TY, TPR, E, VEC, RES, FEW>, dim3(grid), cta, smem, 1, st, a);
}

template <class TX, class TY, int TPR, int E, bool RES, bool FEW>
cudaError_t fwd_t(const NormArgs& a, cudaStream_t st) {
  if (RES || vec_ok<TX, TY>(a, false)) return fwd_k<TX, TY, TPR, E, true, RES, FEW>(a, st);
  // Unaligned rows, read element by element: twice the threads with 16 elements each, except where a group has 64 or 128 threads
  // (1025 to 4096 columns), which lose by it. 30 million elements, us with 32 and with 16 each, bf16 and float: 1001 columns 44 -> 37
  // and 47 -> 45, 1501 45 -> 48 and 45 -> 50, 3001 48 -> 52 and 48 -> 59, 5001 77 -> 65 and 80 -> 68, 12001 57 -> 53 and 61 -> 60.
  constexpr bool kMore = E == 32 && TPR != 64 && TPR != 128;
  return fwd_k<TX, TY, kMore ? 2 * TPR : TPR, kMore ? 16 : E, false, false, FEW>(a, st);
}

// Threads per row. Many rows: 32 elements per thread (few shuffles and barriers per element; the weights pass through
// shared memory). Up to two rows per SM: 8 elements, the shortest way through one row (64 x 2048: 2.7 us against 5.5).
// The denoiser's rows (RES) always take one way: same bits for any number of rows.
template <class TX, class TY, bool RES>
cudaError_t fwd(const NormArgs& a, cudaStream_t st) {
  if (!RES && a.rows <= 2 * kSms && a.d > 256 && a.d <= 8192) {
    if (a.d <= 1024) return fwd_t<TX, TY, 128, 8, RES, true>(a, st);
    if (a.d <= 2048) return fwd_t<TX, TY, 256, 8, RES, true>(a, st);
    if (a.d <= 4096) return fwd_t<TX, TY, 512, 8, RES, true>(a, st);
    return fwd_t<TX, TY, 1024, 8, RES, true>(a, st);
  }
  if (a.d <= 64) return fwd_t<TX, TY, 8, 8, RES, false>(a, st);
  if (a.d <= 256) return fwd_t<TX, TY, 32, 8, RES, false>(a, st);
  if (a.d <= 512) return fwd_t<TX, TY, 32, 16, RES, false>(a, st);
  if (a.d <= 1024) return fwd_t<TX, TY, 32, 32, RES, false>(a, st);
  if (a.d <= 2048) return fwd_t<TX, TY, 64, 32, RES, false>(a, st);
  if (a.d <= 4096) return fwd_t<TX, TY, 128, 32, RES, false>(a, st);
  if (a.d <= 8192) return fwd_t<TX, TY, 256, 32, RES, false>(a, st);
  if (a.d <= 16384) return fwd_t<TX, TY, 512, 32, RES, false>(a, st);
  if (RES) return cudaErrorInvalidValue;
  return launch(k_norm_long<TX, TY>, dim3(std::min(a.rows, 2 * kSms)), 1024, 0, 1, st, a);
}

// backward: threads of a row's group by its length
inline int bwd_tpr(int d) { return d <= 64 ? 8 : d <= 512 ? 32 : d <= 1024 ? 64 : d <= 2048 ? 128 : d <= 4096 ? 256 : d <= 8192 ? 512 : 1024; }

template <class TX, class TY, int TPR, int E, bool VEC, int CL>
cudaError_t bwd_k(const NormArgs& a, int* parts, cudaStream_t st) {
  using C = NormBwd<TX, TY, TPR, E, VEC, CL>;
  static std::atomic<int> cache[kMaxDevices], clusters[kMaxDevices];
  int per_sm = 0, dev = 0;
  cudaError_t e = ctas_per_sm(k_norm_bwd<TX, TY, TPR, E, VEC, CL>, cache, C::kCta, C::kSmemBytes, &per_sm);
  if (e != cudaSuccess) return e;
  if (CL > 1) {                                    // no more clusters than are resident at once (some SMs have no partner)
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
    int r = clusters[dev].load(std::memory_order_acquire);
    if (r == 0) {
      cudaLaunchConfig_t cfg{};
      cfg.gridDim = dim3((unsigned)(kSms / CL * CL));
      cfg.blockDim = dim3(C::kCta);
      cfg.dynamicSmemBytes = C::kSmemBytes;
      cudaLaunchAttribute attr{};
      attr.id = cudaLaunchAttributeClusterDimension;
      attr.val.clusterDim.x = CL; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
      cfg.attrs = &attr;
      cfg.numAttrs = 1;
      if ((e = cudaOccupancyMaxActiveClusters(&r, k_norm_bwd<TX, TY, TPR, E, VEC, CL>, &cfg)) != cudaSuccess) return e;
      if (r < 1) return cudaErrorLaunchOutOfResources;
      clusters[dev].store(r, std::memory_order_release);
    }
    *parts = std::min(*parts, r);
  }
  return launch(k_norm_bwd<TX, TY, TPR, E, VEC, CL>, dim3((unsigned)(*parts * CL)), C::kCta, C::kSmemBytes, CL, st, a);
}

template <class TX, class TY, int TPR, int E, int CL = 1>
cudaError_t bwd_t(const NormArgs& a, int* parts, cudaStream_t st) {
  return vec_ok<TX, TY>(a, true) ? bwd_k<TX, TY, TPR, E, true, CL>(a, parts, st) : bwd_k<TX, TY, TPR, E, false, CL>(a, parts, st);
}

template <class TX, class TY>
cudaError_t bwd(const NormArgs& a, cudaStream_t st) {
  int parts = norm_parts(a.rows, a.d);
  cudaError_t e = cudaSuccess;
  if (a.rows > 0) {
    if (a.d <= 64) e = bwd_t<TX, TY, 8, 8>(a, &parts, st);
    else if (a.d <= 256) e = bwd_t<TX, TY, 32, 8>(a, &parts, st);
    else if (a.d <= 512) e = bwd_t<TX, TY, 32, 16>(a, &parts, st);
    else if (a.d <= 1024) e = bwd_t<TX, TY, 64, 16>(a, &parts, st);
    else if (a.d <= 2048) e = bwd_t<TX, TY, 128, 16>(a, &parts, st);
    else if (a.d <= 4096) e = bwd_t<TX, TY, 256, 16>(a, &parts, st);
    else if (a.d <= 8192) e = bwd_t<TX, TY, 512, 16>(a, &parts, st);
    else if (a.d <= 16384) e = bwd_t<TX, TY, 1024, 16, 2>(a, &parts, st);   // a cluster of two CTAs per row
    else {
      e = launch(k_norm_bwd_long<TX, TY>, dim3(std::min(a.rows, 2 * kSms)), 1024, 0, 1, st, a);
      if (e == cudaSuccess && (a.dw || a.db))
        e = launch(k_norm_bwd_cols<TX, TY>, dim3((a.d + 255) / 256, parts), 256, 0, 1, st, a, parts);
    }
    if (e != cudaSuccess) return e;
  } else {
    parts = 0;                                     // no rows: the gradients are zeros
  }
  if (!a.dw && !a.db) return cudaSuccess;
  // 32 warps per CTA where the CTAs are few, else 8
  const unsigned ctas = (unsigned)((2 * (int64_t)a.d + 31) / 32);
  return launch(k_norm_bwd_join, dim3(ctas), ctas <= 2 * kSms ? 1024 : 256, 0, 1, st, a, parts);
}

}  // namespace

bool norm_is_long(int d) { return d > 16384; }

int norm_parts(int rows, int d) {
  if (norm_is_long(d)) return std::max(1, std::min(rows, kLongParts));
  const int tpr = bwd_tpr(d), rpc = std::max(1, 512 / tpr), resident = tpr > 512 ? kSms / 2 : kSms;
  return std::max(1, std::min((rows + rpc - 1) / rpc, resident));
}

cudaError_t launch_norm(const NormArgs& args, cudaStream_t st) {
  NormArgs a = args;
  a.wide = aligned(a.w, 16) && aligned(a.b, 16);
  if (a.rows <= 0) return cudaSuccess;
  if (a.res) return a.tx == SDS_F32 && a.ty == SDS_BF16 ? fwd<float, Bf16, true>(a, st) : cudaErrorInvalidValue;
  if (a.tx == SDS_F32 && a.ty == SDS_F32) return fwd<float, float, false>(a, st);
  if (a.tx == SDS_F32 && a.ty == SDS_BF16) return fwd<float, Bf16, false>(a, st);
  if (a.tx == SDS_F32 && a.ty == SDS_F16) return fwd<float, F16, false>(a, st);
  if (a.tx == SDS_BF16 && a.ty == SDS_BF16) return fwd<Bf16, Bf16, false>(a, st);
  if (a.tx == SDS_F16 && a.ty == SDS_F16) return fwd<F16, F16, false>(a, st);
  return cudaErrorInvalidValue;
}

cudaError_t launch_norm_backward(const NormArgs& args, cudaStream_t st) {
  NormArgs a = args;
  a.wide = aligned(a.w, 16) && aligned(a.b, 16);
  if (a.tx == SDS_F32 && a.ty == SDS_F32) return bwd<float, float>(a, st);
  if (a.tx == SDS_F32 && a.ty == SDS_BF16) return bwd<float, Bf16>(a, st);
  if (a.tx == SDS_F32 && a.ty == SDS_F16) return bwd<float, F16>(a, st);
  if (a.tx == SDS_BF16 && a.ty == SDS_BF16) return bwd<Bf16, Bf16>(a, st);
  if (a.tx == SDS_F16 && a.ty == SDS_F16) return bwd<F16, F16>(a, st);
  return cudaErrorInvalidValue;
}

}  // namespace sds
