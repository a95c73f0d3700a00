// Device-side building blocks of the kernels that hold rows in registers: element types, packs, and sums over the threads of a
// row's group.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/sds.h"

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

// Kernels overlap their starts: the next one may be started once all CTAs of this one have begun (their launch takes about
// as long as a small call runs), and this one waits here for the end of the kernel in front, and for its writes.
// Nothing in device memory is read or written before. The next one is let go before this wait: it may begin while what ran
// in front of this kernel still runs, so it has to wait in full as well before it reads anything. (Loads behind it are plain ones: the
// compiler may move read-only loads ahead of the wait.)
__device__ __forceinline__ void start_after_prior_kernel() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

}  // namespace

}  // namespace sds
