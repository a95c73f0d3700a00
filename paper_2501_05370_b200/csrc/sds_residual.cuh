// From one block of a residual network to the next, forward and backward, in one pass over the rows:
//
//   q  = post(h) wp  (post: the norm below, without weight; or q = h)
//   r' = r + alpha gate D q                                         (D: dropout, 0 or 1 / (1 - p))
//   n  = u (1 + scale) + shift,   u = xhat w + b,   xhat = (r' - m) s
//   layer norm: m = <r'>, s = 1 / sqrt(<(r' - m)^2> + eps);   rms: m = 0      (<.> = mean over the row)
// gate, scale and shift are one row for every `per` consecutive rows.
//
//   dx  = dn (1 + scale) w
//   g   = dr + s (dx - <dx> - xhat <dx xhat>)                       (rms: without <dx>); the gradient of r
//   dq  = alpha gate D g,   dh = dq or, behind post, the same formula with dq wp and post's statistics
// Sums over the rows of a group: A = sum dn xhat, B = sum dn, C = sum alpha D g q / wp. They give every gradient of a vector:
//   dshift = B, dscale = w A + b B, dgate = wp C;  dw = sum_groups (1 + scale) A, db = sum_groups (1 + scale) B,
//   dwp = sum_groups gate C.
//
// Bound by memory: r, h in and r', n out; r, h, dn, dr in and the gradients of r and h out. The backward pass makes r' again from r and
// h, which it needs anyway, so r' need not be kept, and xhat is not that of a rounded r'. A group of threads holds a row in registers,
// eight columns a thread, in pairs (the row kernels would otherwise be bound by issue). Statistics are held in float; layer norm takes them around the rounded mean and takes the mean's
// remainder back out, so that rows far from zero keep 24 bits of their spread.
//
// Sums over rows: a worker (the group of threads) adds its rows in registers, workers' sums are added by a second kernel in a
// fixed order (no atomics: same bits on every run).
#pragma once

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "sds_device.cuh"
#include "sds_layers.h"
#include "sds_rows.cuh"

namespace sds {

namespace {

constexpr int kStreamDropout = 3;
constexpr int kBlock = 8;                         // columns of one access of 16-bit types, and of one block of the generator

// how the rows of a backward call are dealt out (ResidualNormArgs::mode)
enum ResidualMode : int {
  kSumAll = 0,      // one group: a worker's rows, their plain sums A, B, C
  kSumWeighted = 1, // sums weighted with each row's own scale and gate; rows that are groups of their own write their gradients at once
  kSumGroups = 2,   // plain sums per group, whole ones and parts of those that cross workers, and the worker's weighted sums over them
};

// eight neighbouring columns as they lie in memory
template <class T> struct Raw {
  static constexpr int kUnits = sizeof(T) / 2;
  uint4 q[kUnits];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < kUnits; ++i) q[i] = *(reinterpret_cast<const uint4*>(p) + i);
  }
};
// (eight floats are one 32-byte load: as two of 16 bytes a warp would ask for half a sector at a time)
template <> __device__ __forceinline__ void Raw<float>::load(const float* p) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(q[0].x), "=r"(q[0].y), "=r"(q[0].z), "=r"(q[0].w), "=r"(q[1].x), "=r"(q[1].y), "=r"(q[1].z), "=r"(q[1].w)
               : "l"(p)
               : "memory");
}
// as four pairs of floats
constexpr int P = kBlock / 2;
__device__ __forceinline__ void words_to(const uint4* q, float2 (&o)[P], float) {
  o[0] = make_float2(__uint_as_float(q[0].x), __uint_as_float(q[0].y));
  o[1] = make_float2(__uint_as_float(q[0].z), __uint_as_float(q[0].w));
  o[2] = make_float2(__uint_as_float(q[1].x), __uint_as_float(q[1].y));
  o[3] = make_float2(__uint_as_float(q[1].z), __uint_as_float(q[1].w));
}
__device__ __forceinline__ float2 pair_of(uint32_t w, Bf16) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ float2 pair_of(uint32_t w, F16) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
template <class T> __device__ __forceinline__ void words_to(const uint4* q, float2 (&o)[P], T t) {
  o[0] = pair_of(q[0].x, t); o[1] = pair_of(q[0].y, t); o[2] = pair_of(q[0].z, t); o[3] = pair_of(q[0].w, t);
}
// (eight floats are one 32-byte store: as two of 16 bytes a warp would write half a sector at a time)
__device__ __forceinline__ void store_words(float* p, const float2 (&v)[P]) {
  asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v[0].x), "f"(v[0].y), "f"(v[1].x), "f"(v[1].y),
               "f"(v[2].x), "f"(v[2].y), "f"(v[3].x), "f"(v[3].y)
               : "memory");
}
template <class T> __device__ __forceinline__ void store_words(T* p, const float2 (&v)[P]) {
  Pack<T, 8> o;
#pragma unroll
  for (int i = 0; i < P; ++i) put2(o, i, v[i]);
  *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(&o);
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ float& element(float2* v, int e) { return reinterpret_cast<float*>(v)[e]; }
__device__ __forceinline__ float element(const float2* v, int e) { return reinterpret_cast<const float*>(v)[e]; }
// (rows lie less than 2^31 elements apart: one multiplication)
template <class T> __device__ __forceinline__ T* row_of(void* p, int row, int64_t ld) {
  return static_cast<T*>(p) + (uint64_t)(uint32_t)row * (uint32_t)ld;
}
template <class T> __device__ __forceinline__ const T* row_of(const void* p, int row, int64_t ld) {
  return static_cast<const T*>(p) + (uint64_t)(uint32_t)row * (uint32_t)ld;
}

// A group of TPR threads holds a row, T of them in each of CL CTAs.
template <int TPR, int CL> struct ResidualShape {
  static constexpr int T = TPR / CL;
  static constexpr int kCta = T < 128 ? 128 : T;
  static constexpr int kRows = kCta / T;                        // rows of a CTA at a time
  static constexpr int kSlots = 2 * kRows * 4 * (TPR > 32 ? TPR / 32 : 1);
  static constexpr int kStatSlots = kCta / (T < 32 ? T : 32);   // a row's statistics, for each warp (or each group in a warp)
};

// The eight columns of a group's thread t. VEC: neighbours; a thread beyond d computes on whatever it holds and is left out of sums and
// stores. Else: T apart, so that a warp's accesses are neighbours; columns beyond d hold zeros.
template <int TPR, int CL, bool VEC> struct Columns {
  static constexpr int T = TPR / CL;
  int c0, tid, d;
  bool live;
  __device__ Columns(int t, int d_) : c0(VEC ? t * kBlock : t / T * T * kBlock + t % T), tid(t % T), d(d_) { live = c0 < d; }
  __device__ __forceinline__ int at(int e) const { return VEC ? c0 + e : c0 + e * T; }
  __device__ __forceinline__ bool has(int e) const { return VEC ? live : c0 + e * T < d; }
};

template <class T, class C>
__device__ __forceinline__ void load_scalar(const T* row, const C& col, float2 (&o)[P]) {
#pragma unroll
  for (int e = 0; e < kBlock; ++e) element(o, e) = col.has(e) ? Conv<T>::get(row[col.at(e)]) : 0.f;
}
template <class T, int TPR, int CL, bool VEC>
__device__ __forceinline__ void store_row(T* row, const Columns<TPR, CL, VEC>& col, bool on, const float2 (&v)[P]) {
  if (VEC) {
    if (on && col.live) store_words(row + col.c0, v);
  } else {
#pragma unroll
    for (int e = 0; e < kBlock; ++e)
      if (on && col.has(e)) row[col.at(e)] = Conv<T>::put(element(v, e));
  }
}

// (Loads are plain ones: the compiler may move read-only loads ahead of the wait for the kernel in front.)
// A thread's columns of a vector of any of the three types. 16-bit vectors of whole pieces (VEC) can be requested ahead, as they lie in memory; floats are read where they are used (twice the registers, and they mostly lie in L1).
template <int TPR, int CL, bool VEC>
__device__ __forceinline__ void request_vector(uint4& r, const void* p, int type, uint64_t off, const Columns<TPR, CL, VEC>& col) {
  if (VEC && p && type != SDS_F32 && col.live) r = *(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + off + col.c0));
}
// (p is not NULL)
template <int TPR, int CL, bool VEC>
__device__ __forceinline__ void take_vector(const uint4& r, const void* p, int type, uint64_t off, const Columns<TPR, CL, VEC>& col,
                                            float2 (&o)[P]) {
  if (VEC) {
    if (type == SDS_F32) {
      Raw<float> f;
      f.load(static_cast<const float*>(p) + off + (col.live ? col.c0 : 0));
      words_to(f.q, o, 0.f);
    } else if (type == SDS_BF16) {
      words_to(&r, o, Bf16{});
    } else {
      words_to(&r, o, F16{});
    }
  } else if (type == SDS_F32) {
    load_scalar(static_cast<const float*>(p) + off, col, o);
  } else if (type == SDS_BF16) {
    load_scalar(static_cast<const Bf16*>(p) + off, col, o);
  } else {
    load_scalar(static_cast<const F16*>(p) + off, col, o);
  }
}
template <int TPR, int CL, bool VEC>
__device__ __forceinline__ void load_vector(const void* p, int type, uint64_t off, const Columns<TPR, CL, VEC>& col, float2 (&o)[P]) {
  uint4 r = make_uint4(0u, 0u, 0u, 0u);
  request_vector(r, p, type, off, col);
  take_vector(r, p, type, off, col, o);
}
template <class T, int TPR, int CL, bool VEC>
__device__ __forceinline__ void store_typed_vector(T* p, const Columns<TPR, CL, VEC>& col, bool on, const float2 (&v)[P]) {
  if (VEC) {
    if (on && col.live) store_words(p + col.c0, v);
  } else {
#pragma unroll
    for (int e = 0; e < kBlock; ++e)
      if (on && col.has(e)) p[col.at(e)] = Conv<T>::put(element(v, e));
  }
}
template <int TPR, int CL, bool VEC>
__device__ __forceinline__ void store_vector(void* p, int type, uint64_t off, const Columns<TPR, CL, VEC>& col, bool on, const float2 (&v)[P]) {
  if (type == SDS_F32) store_typed_vector(static_cast<float*>(p) + off, col, on, v);
  else if (type == SDS_BF16) store_typed_vector(static_cast<Bf16*>(p) + off, col, on, v);
  else store_typed_vector(static_cast<F16*>(p) + off, col, on, v);
}
// where a group's row of gate, scale or shift begins
__device__ __forceinline__ uint64_t cond_at(int group, int64_t ld) { return (uint64_t)(uint32_t)group * (uint32_t)ld; }

// Which of a thread's eight columns are kept: 16 of the block's 128 bits decide a column, low half of a word first.
struct Kept {
  uint32_t w[4], limit;                                         // limit: the threshold in the upper half
  __device__ __forceinline__ bool operator()(int e) const { return ((e & 1) ? w[e / 2] : w[e / 2] << 16) >= limit; }
};
__device__ __forceinline__ Kept kept_block(const DropoutArgs& a, uint32_t step, uint64_t row, uint32_t block) {
  const uint4 x = philox_block(a.seed, kStreamDropout, row, step, block);
  Kept k{{x.x, x.y, x.z, x.w}, a.threshold << 16};
  if (a.threshold >= 65536u) {                                  // nothing is kept
    k.w[0] = k.w[1] = k.w[2] = k.w[3] = 0u;
    k.limit = ~0u;
  }
  return k;
}
// The same for a thread's columns. Where these are not a block, the blocks of a warp's (or of a smaller group's) columns are drawn one by
// a lane, and a bit for each column changes hands. (All 32 lanes call it.)
template <int TPR, int CL, bool VEC>
__device__ __forceinline__ Kept kept_columns(const DropoutArgs& a, uint32_t step, int row, const Columns<TPR, CL, VEC>& col, int lane) {
  constexpr int T = TPR / CL, W = T < 32 ? T : 32, kPer = W / 8;     // W neighbours are kPer blocks
  const uint64_t r = a.row0 + (uint32_t)row;
  if (VEC) return kept_block(a, step, r, (uint32_t)col.c0 >> 3);
  const int in = lane % W;
  const Kept mine = kept_block(a, step, r, (uint32_t)(col.c0 - in + in / kPer * T + in % kPer * 8) >> 3);
  uint32_t bits = 0;
#pragma unroll
  for (int e = 0; e < kBlock; ++e) bits |= (mine(e) ? 1u : 0u) << e;
  Kept kept{{0u, 0u, 0u, 0u}, 0x80000000u};                     // (a kept column has the top bit of its half)
#pragma unroll
  for (int e = 0; e < kBlock; ++e) {
    const uint32_t bit = (__shfl_sync(kAll, bits, lane - in + e * kPer + (in >> 3)) >> (in & 7)) & 1u;
    kept.w[e / 2] |= bit << ((e & 1) ? 31 : 15);
  }
  return kept;
}
__device__ __forceinline__ uint32_t dropout_step(const DropoutArgs& a) { return a.step + (a.step_dev ? (uint32_t)*a.step_dev : 0u); }

// r + k q where a column is kept, else r
__device__ __forceinline__ void add_branch(float2& r, float2 k, float2 q, bool drops, const Kept& kept, int i) {
  if (!drops) {
    r = fma2(k, q, r);
  } else {
    if (kept(2 * i)) r.x = fmaf(k.x, q.x, r.x);
    if (kept(2 * i + 1)) r.y = fmaf(k.y, q.y, r.y);
  }
}
// v where a column is kept, else 0
__device__ __forceinline__ float2 select_kept(float2 v, const Kept& kept, int i) {
  return make_float2(kept(2 * i) ? v.x : 0.f, kept(2 * i + 1) ? v.y : 0.f);
}

// Sums over a group, each call in the other half of its slots: a half is written again only after the barrier of the call between.
template <int TPR, int CL> struct GroupSums {
  static constexpr int NW = TPR > 32 ? TPR / 32 : 1;
  float* slot;
  int t, bar, flip = 0;
  bool live;                                                    // threads beyond d are left out
  __device__ GroupSums(float* slots, int sub, int t_, bool live_) : slot(slots + sub * 8 * NW), t(t_), bar(1 + sub), live(live_) {}
  template <int N> __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = live ? v[n] : 0.f;
    float* at = slot + flip * 4 * NW;
    flip ^= 1;
    if constexpr (NW < 4 || NW > 16 || CL > 1) {
      group_sum<TPR, N, CL>(v, at, t, bar);
    } else {                                                    // four warps' sums at a time
      group_post<TPR, N, 1>(v, at, t);
      asm volatile("bar.sync %0, %1;" ::"r"(bar), "r"(TPR) : "memory");
#pragma unroll
      for (int n = 0; n < N; ++n) {
        float2 s = make_float2(0.f, 0.f);
#pragma unroll
        for (int w = 0; w < NW; w += 4) {
          const float4 q = *reinterpret_cast<const float4*>(at + n * NW + w);
          const float2 two = add2(make_float2(q.x, q.y), make_float2(q.z, q.w));
          s = w == 0 ? two : add2(s, two);
        }
        v[n] = total(s);
      }
    }
  }
};

// v - m, and (v - rest) s, where there are columns
template <class C>
__device__ __forceinline__ void shift_row(float2 (&v)[P], float m, const C& col, bool vec) {
  if (vec) {
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = add2(v[i], both(-m));
  } else {
#pragma unroll
    for (int e = 0; e < kBlock; ++e) element(v, e) = col.has(e) ? element(v, e) - m : 0.f;
  }
}
template <class C>
__device__ __forceinline__ void scale_row(float2 (&v)[P], float rest, float s, const C& col, bool vec) {
  if (vec) {
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = fma2(v[i], both(s), both(-rest * s));
  } else {
#pragma unroll
    for (int e = 0; e < kBlock; ++e) element(v, e) = col.has(e) ? (element(v, e) - rest) * s : 0.f;
  }
}
// sums of a and of a b over the thread's columns
__device__ __forceinline__ void pair_sums(const float2 (&a)[P], const float2 (&b)[P], float (&s)[2]) {
  float2 x = a[0], y = mul2(a[0], b[0]);
#pragma unroll
  for (int i = 1; i < P; ++i) {
    x = add2(x, a[i]);
    y = fma2(a[i], b[i], y);
  }
  s[0] = total(x);
  s[1] = total(y);
}

// Turns the row v into xhat; mean, remainder, 1 / size.
template <int TPR, int CL, bool VEC>
__device__ __forceinline__ float4 normalise(float2 (&v)[P], GroupSums<TPR, CL>& sums, const Columns<TPR, CL, VEC>& col, float inv_d, bool rms, float eps) {
  float4 st = make_float4(0.f, 0.f, 0.f, 0.f);
  if (rms) {
    float2 x = mul2(v[0], v[0]);
#pragma unroll
    for (int i = 1; i < P; ++i) x = fma2(v[i], v[i], x);
    float s[1] = {total(x)};
    sums(s);
    st.z = rsqrtf(fmaf(s[0], inv_d, eps));
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = mul2(v[i], both(st.z));
    return st;
  }
  float2 x = v[0];
#pragma unroll
  for (int i = 1; i < P; ++i) x = add2(x, v[i]);
  float s[1] = {total(x)};
  sums(s);
  st.x = s[0] * inv_d;
  shift_row(v, st.x, col, VEC);
  float q[2];
  pair_sums(v, v, q);
  sums(q);
  st.y = q[0] * inv_d;
  st.z = rsqrtf(fmaxf(fmaf(-st.y, st.y, q[1] * inv_d), 0.f) + eps);   // (of a constant row, the two may differ by their roundings either way)
  scale_row(v, st.y, st.z, col, VEC);
  return st;
}

// ---------------------------------------------------------------------------------------------
// rows to come: a ring in shared memory
// ---------------------------------------------------------------------------------------------

// VEC: a warp copies and reads its own columns, so there is no barrier, and the copies take no registers. Else the group copies the
// 16-byte pieces that cover its CTA's part of the row (they may begin up to 15 bytes before it and end as many behind: within
// pieces of memory that hold some of the row), and reads elements, behind a barrier.
template <class T, int TPR, int CL, bool VEC> struct RingRow {
  using S = ResidualShape<TPR, CL>;
  static constexpr int kUnits = sizeof(T) / 2;                  // 16-byte pieces of eight columns
  static constexpr int kGroup = S::T * kUnits + 2;              // not VEC: pieces of a group
  static constexpr int kPieces = VEC ? kUnits * S::kCta : kGroup * S::kRows;
};
constexpr int kRingStages = 3;
// where piece u of a row of floats lies: a lane reads two neighbouring pieces, eight lanes from all banks
__device__ __forceinline__ int ring_piece(int u) { return u ^ ((u >> 3) & 1); }

__device__ __forceinline__ void copy16(void* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kRingStages - 2) : "memory"); }

template <class T, int TPR, int CL, bool VEC>
__device__ __forceinline__ void ring_copy(uint4* to, const T* row, const Columns<TPR, CL, VEC>& col, int sub) {
  using R = RingRow<T, TPR, CL, VEC>;
  using S = ResidualShape<TPR, CL>;
  if (VEC) {
    if (R::kUnits == 1) {
      if (col.live) copy16(to + threadIdx.x, row + col.c0);
    } else {                                                    // lanes copy neighbouring pieces: whole sectors
      constexpr int W = S::T < 32 ? S::T : 32;
      const int in = (int)threadIdx.x % W, u0 = ((int)threadIdx.x - in) * 2 + in, first = col.c0 - in * kBlock;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (first + (in + i * W) * 4 < col.d) copy16(to + ring_piece(u0 + i * W), row + first + (in + i * W) * 4);
    }
  } else {
    const int part = col.c0 - col.tid, n = min(col.d - part, S::T * kBlock);      // the CTA's columns
    if (n <= 0) return;
    const uintptr_t first = reinterpret_cast<uintptr_t>(row + part);
    const char* from = reinterpret_cast<const char*>(first & ~(uintptr_t)15);
    const int pieces = ((int)(first & 15) + n * (int)sizeof(T) + 15) >> 4;
#pragma unroll
    for (int k = 0; k <= R::kUnits; ++k) {                      // (R::kGroup pieces at most: one beyond T kUnits at most where T > 1)
      const int i = col.tid + k * S::T;
      if (i < pieces) copy16(to + sub * R::kGroup + i, from + 16 * i);
    }
  }
}
template <class T, int TPR, int CL, bool VEC>
__device__ __forceinline__ void ring_take(const uint4* from, const T* row, const Columns<TPR, CL, VEC>& col, int sub, float2 (&o)[P]) {
  using R = RingRow<T, TPR, CL, VEC>;
  using S = ResidualShape<TPR, CL>;
  if (VEC) {
    uint4 w[R::kUnits];
#pragma unroll
    for (int i = 0; i < R::kUnits; ++i) w[i] = from[R::kUnits == 1 ? (int)threadIdx.x : ring_piece(2 * (int)threadIdx.x + i)];
    words_to(w, o, T{});
  } else {
    const char* mine = reinterpret_cast<const char*>(from + sub * R::kGroup) + (reinterpret_cast<uintptr_t>(row + (col.c0 - col.tid)) & 15);
#pragma unroll
    for (int e = 0; e < kBlock; ++e)
      element(o, e) = col.has(e) ? Conv<T>::get(reinterpret_cast<const T*>(mine)[e * S::T + col.tid]) : 0.f;
  }
}
// the group's copies are there for all of its threads
template <int TPR, int CL, bool VEC>
__device__ __forceinline__ void ring_ready(int sub) {
  copies_wait();
  constexpr int T = TPR / CL;
  if (!VEC && T > 32) asm volatile("bar.sync %0, %1;" ::"r"(1 + sub), "r"(T) : "memory");
  else __syncwarp();
}

// A worker's rows are neighbours: `row` up to `end`, `group` the row's group and `left` its rows from here on.
struct RowWalk {
  int row, end, group, left;
  __device__ RowWalk(const ResidualNormArgs& a, int worker) {
    const int64_t first = (int64_t)worker * a.share;
    row = (int)min((int64_t)a.rows, first);
    end = min(a.rows - row, a.share) + row;
    group = row / a.per;
    left = a.per - (row - group * a.per);
  }
  __device__ __forceinline__ bool on() const { return row < end; }
  __device__ __forceinline__ void next() { ++row; }
  __device__ __forceinline__ void next_group(int per) {         // behind next()
    if (--left == 0) { ++group; left = per; }
  }
};
// whether the worker, or another one of its warp (small groups: the warp's lanes stay together), has a row left
template <int T> __device__ __forceinline__ bool rows_left(bool on) { return T < 32 ? __any_sync(kAll, on) : on; }

// FULL: with post or dropout. Two kernels, as the time of either goes with the length of its code: with vectors of unaligned pieces in the
// aligned kernels too, these were twice as long and 16384 x 2048 backward took 142 us conditioned (119 without), 177 with all parts (156).
// A group takes neighbouring rows, which mostly share their row of gate, scale and shift. Rows come through the ring, vectors are requested
// before the sums that they wait for.
// HELD: the products of a group's vectors (alpha gate wp, w (1 + scale), b (1 + scale) + shift) stay in registers while the group lasts, at
// fewer CTAs of an SM. 16384 x 2048 float stream with post, gate, weights and dropout 81.7 -> 71.6 us, with scale, shift and bias too 88.5 ->
// 73, 65536 x 512 88.7 -> 74; without vectors 70.4 -> 78.6 (layer norm), every row its own 96 -> 113, bf16 stream 89.7 -> 99.6, clusters 127 -> 164.
// From eight rows a group on (16384 x 2048 with gate and weight, not held and held: 2 rows 86 and 92, 4 82 and 85, 6 82 and 82, 8 82 and 80, 16 82
// and 79; with gate, scale, shift and weight 94 and 99, 88 and 88, 88 and 84, 86 and 82, 85 and 80; 65536 x 512 107 and 107, 98 and 92, 94 and 88,
// 92 and 84, 92 and 82).
// 16384 x 2048, float stream and bf16 branch: conditioned 75 us (403 MB, 5.4 TB/s, 82 % of a copy's rate).
template <class TR, class TH, int TPR, int CL, bool VEC, bool FULL, bool HELD>
__global__ void __launch_bounds__(ResidualShape<TPR, CL>::kCta) k_residual_norm(const ResidualNormArgs a) {
  using S = ResidualShape<TPR, CL>;
  constexpr int kR = RingRow<TR, TPR, CL, VEC>::kPieces, kStage = kR + RingRow<TH, TPR, CL, VEC>::kPieces;
  extern __shared__ uint4 ring[];
  __shared__ __align__(16) float slots[S::kSlots];
  const int sub = threadIdx.x / S::T, lane = threadIdx.x & 31;
  const int t = (CL > 1 ? (int)(blockIdx.x % CL) * S::T : 0) + (int)threadIdx.x % S::T;
  const Columns<TPR, CL, VEC> col(t, a.d);
  GroupSums<TPR, CL> sums(slots, sub, t, !VEC || col.live);
  if (CL > 1) {                                                 // the peers' slots are there to be written
    cluster_arrive();
    cluster_wait();
  }
  start_after_prior_kernel();
  const float inv_d = 1.0f / (float)a.d;
  const bool drops = FULL && a.drop.threshold != 0;
  const uint32_t dstep = drops ? dropout_step(a.drop) : 0u;
  const float2 alpha = both(drops ? a.alpha * a.drop.scale : a.alpha);
  RowWalk at(a, (int)blockIdx.x / CL * S::kRows + sub);
  const auto request = [&](int row, int stage) {
    if (row < at.end) {
      uint4* to = ring + stage * kStage;
      ring_copy(to, row_of<TR>(a.r, row, a.ldr), col, sub);
      if (a.h) ring_copy(to + kR, row_of<TH>(a.h, row, a.ldh), col, sub);
    }
    copies_end();
  };
  for (int s = 0; s < kRingStages - 1; ++s) request(at.row + s, s);
  int stage = 0, held = -1;
  uint4 gate, scale, shift;
  float2 branch[P], norm[P], off[P];                            // HELD
  while (rows_left<S::T>(at.on())) {
    const bool on = at.on();
    const int row = on ? at.row : 0, group = on ? at.group : 0;
    float2 v[P], q[P], x[P];
    const bool other = group != held;
    if (other) {                                                // (kept while the group lasts)
      held = group;
      if (a.h) request_vector(gate, a.gate, a.tc, cond_at(group, a.ldgate), col);
      request_vector(scale, a.scale, a.tc, cond_at(group, a.ldscale), col);
      request_vector(shift, a.shift, a.tc, cond_at(group, a.ldshift), col);
    }
    ring_ready<TPR, CL, VEC>(sub);
    if (HELD && other) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        branch[i] = alpha;
        norm[i] = both(1.f);
        off[i] = both(0.f);
      }
      if (a.h && a.gate) {
        take_vector(gate, a.gate, a.tc, cond_at(group, a.ldgate), col, x);
#pragma unroll
        for (int i = 0; i < P; ++i) branch[i] = mul2(branch[i], x[i]);
      }
      if (a.wp) {
        load_vector(a.wp, a.tw, 0, col, x);
#pragma unroll
        for (int i = 0; i < P; ++i) branch[i] = mul2(branch[i], x[i]);
      }
      if (a.scale) {
        take_vector(scale, a.scale, a.tc, cond_at(group, a.ldscale), col, x);
#pragma unroll
        for (int i = 0; i < P; ++i) norm[i] = add2(norm[i], x[i]);
      }
      if (a.b) {
        load_vector(a.b, a.tw, 0, col, x);
#pragma unroll
        for (int i = 0; i < P; ++i) off[i] = mul2(norm[i], x[i]);
      }
      if (a.shift) {
        take_vector(shift, a.shift, a.tc, cond_at(group, a.ldshift), col, x);
#pragma unroll
        for (int i = 0; i < P; ++i) off[i] = add2(off[i], x[i]);
      }
      if (a.w) {
        load_vector(a.w, a.tw, 0, col, x);
#pragma unroll
        for (int i = 0; i < P; ++i) norm[i] = mul2(norm[i], x[i]);
      }
    }
    const uint4* mine = ring + stage * kStage;
    ring_take(mine, row_of<TR>(a.r, row, a.ldr), col, sub, v);
    if (a.h) {
      ring_take(mine + kR, row_of<TH>(a.h, row, a.ldh), col, sub, q);
      if (FULL && a.post) {
        const float4 st = normalise(q, sums, col, inv_d, a.rms, a.eps);
        if (!HELD && a.wp) {
          load_vector(a.wp, a.tw, 0, col, x);
#pragma unroll
          for (int i = 0; i < P; ++i) q[i] = mul2(q[i], x[i]);
        }
        if (a.stats && t == 0 && on) a.stats[2 * (size_t)row + 1] = st;
      }
      Kept kept;
      if (drops) kept = kept_columns(a.drop, dstep, row, col, lane);
      if (HELD) {
#pragma unroll
        for (int i = 0; i < P; ++i) add_branch(v[i], branch[i], q[i], drops, kept, i);
      } else if (a.gate) {
        take_vector(gate, a.gate, a.tc, cond_at(group, a.ldgate), col, x);
#pragma unroll
        for (int i = 0; i < P; ++i) add_branch(v[i], mul2(alpha, x[i]), q[i], drops, kept, i);
      } else {
#pragma unroll
        for (int i = 0; i < P; ++i) add_branch(v[i], alpha, q[i], drops, kept, i);
      }
      store_row(row_of<TR>(a.out, row, a.ldo), col, on, v);
    }
    const float4 st = normalise(v, sums, col, inv_d, a.rms, a.eps);
    // (behind a sum: all threads of the group are done with the row before, whose place this takes)
    request(at.row + kRingStages - 1, stage == 0 ? kRingStages - 1 : stage - 1);
    if (a.stats && t == 0 && on) a.stats[2 * (size_t)row] = st;
    if (HELD) {
#pragma unroll
      for (int i = 0; i < P; ++i) v[i] = fma2(v[i], norm[i], off[i]);
    } else {
      if (a.w) {
        load_vector(a.w, a.tw, 0, col, x);
#pragma unroll
        for (int i = 0; i < P; ++i) v[i] = mul2(v[i], x[i]);
      }
      if (a.b) {
        load_vector(a.b, a.tw, 0, col, x);
#pragma unroll
        for (int i = 0; i < P; ++i) v[i] = add2(v[i], x[i]);
      }
      if (a.scale) {
        take_vector(scale, a.scale, a.tc, cond_at(group, a.ldscale), col, x);
#pragma unroll
        for (int i = 0; i < P; ++i) v[i] = fma2(v[i], x[i], v[i]);
      }
      if (a.shift) {
        take_vector(shift, a.shift, a.tc, cond_at(group, a.ldshift), col, x);
#pragma unroll
        for (int i = 0; i < P; ++i) v[i] = add2(v[i], x[i]);
      }
    }
    store_row(row_of<TH>(a.n, row, a.ldn), col, on, v);
    at.next();
    at.next_group(a.per);
    stage = stage + 1 == kRingStages ? 0 : stage + 1;
  }
}

// ---------------------------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------------------------

// (the compiler spends more on pairing registers in the backward kernel than pairs save: 16384 x 2048 conditioned 142 us with them, 137 without)
__device__ __forceinline__ float2 each_fma2(float2 a, float2 b, float2 c) { return make_float2(fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y)); }
__device__ __forceinline__ float2 each_mul2(float2 a, float2 b) { return make_float2(a.x * b.x, a.y * b.y); }
__device__ __forceinline__ float2 each_add2(float2 a, float2 b) { return make_float2(a.x + b.x, a.y + b.y); }

template <class TR, class TH, int TPR, int CL, bool VEC> struct ResidualBwd {
  using S = ResidualShape<TPR, CL>;
  static constexpr int kR = RingRow<TR, TPR, CL, VEC>::kPieces, kH = RingRow<TH, TPR, CL, VEC>::kPieces;
  static constexpr int kStats = 2 * kR + 2 * kH;                // dr, r, dn, h, then the statistics
  static constexpr int kStage = kStats + 2 * S::kStatSlots;
  static constexpr int kSmemBytes = kRingStages * kStage * 16;
  static constexpr int kMinCtas = 512 / S::kCta;                // 512 threads of 128 registers
};

// total = or += k v
template <int TPR, int CL, bool VEC>
__device__ __forceinline__ void add_total(float* total, const float2 (&v)[P], const float2 (&k)[P], const Columns<TPR, CL, VEC>& col, bool first) {
  float2 o[P];
#pragma unroll
  for (int i = 0; i < P; ++i) o[i] = both(0.f);
  if (!first) load_scalar(total, col, o);
#pragma unroll
  for (int i = 0; i < P; ++i) o[i] = each_fma2(k[i], v[i], o[i]);
  store_typed_vector(total, col, true, o);
}

// 512 threads of 128 registers an SM: a row's values, the sums over rows and the products of a group's vectors are in registers, and issue is
// what bounds the parts beside the plain norm: with gate, post weight and weight read and multiplied row by row, 16384 x 2048 with all parts
// took 145 us (764 instructions of a warp for a row, 64 % of the issue slots), now 125 (604 MB, 4.8 TB/s; a bf16 stream 144 -> 117);
// conditioned, float stream and bf16 branch, 114 (5.3 TB/s). Held products cost where there is but one vector: a float stream with a weight
// alone 102 -> 106.
template <class TR, class TH, int TPR, int CL, bool VEC, bool FULL>
__global__ void __launch_bounds__(ResidualShape<TPR, CL>::kCta, ResidualBwd<TR, TH, TPR, CL, VEC>::kMinCtas) k_residual_norm_bwd(const ResidualNormArgs a) {
  using S = ResidualShape<TPR, CL>;
  using G = ResidualBwd<TR, TH, TPR, CL, VEC>;
  constexpr int kWarp = S::T < 32 ? S::T : 32;
  extern __shared__ uint4 ring[];
  __shared__ __align__(16) float slots[S::kSlots];
  const int sub = threadIdx.x / S::T, lane = threadIdx.x & 31;
  const int t = (CL > 1 ? (int)(blockIdx.x % CL) * S::T : 0) + (int)threadIdx.x % S::T;
  const Columns<TPR, CL, VEC> col(t, a.d);
  GroupSums<TPR, CL> sums(slots, sub, t, !VEC || col.live);
  if (CL > 1) {
    cluster_arrive();
    cluster_wait();
  }
  start_after_prior_kernel();
  const int worker = (int)blockIdx.x / CL * S::kRows + sub;
  const int d = a.d;
  const float inv_d = 1.0f / (float)d;
  const bool drops = FULL && a.drop.threshold != 0;
  const uint32_t dstep = drops ? dropout_step(a.drop) : 0u;
  const float2 alpha = both(drops ? a.alpha * a.drop.scale : a.alpha);     // of a kept column
  float2 sa[P], sb[P], sq[P];                                   // A, B, C, or their weighted forms
#pragma unroll
  for (int i = 0; i < P; ++i) sa[i] = sb[i] = sq[i] = both(0.f);
  bool first_flush = true;

  RowWalk at(a, worker);
  const int begin = at.row;
  const auto request = [&](int row, int stage) {
    if (row < at.end) {
      uint4* to = ring + stage * G::kStage;
      if (a.dr) ring_copy(to, row_of<TR>(a.dr, row, a.lddr), col, sub);
      ring_copy(to + G::kR, row_of<TR>(a.r, row, a.ldr), col, sub);
      ring_copy(to + 2 * G::kR, row_of<TH>(a.dn, row, a.lddn), col, sub);
      if (a.h) ring_copy(to + 2 * G::kR + G::kH, row_of<TH>(a.h, row, a.ldh), col, sub);
      if (threadIdx.x % kWarp == 0) {
        uint4* st = to + G::kStats + threadIdx.x / kWarp * 2;
        copy16(st, a.stats + 2 * (size_t)row);
        if (FULL && a.post) copy16(st + 1, a.stats + 2 * (size_t)row + 1);
      }
    }
    copies_end();
  };
  for (int s = 0; s < kRingStages - 1; ++s) request(at.row + s, s);
  int stage = 0, held = -1;
  // while their group lasts: alpha gate wp, and (1 + scale) w where the sums over rows do not need 1 + scale by itself
  float2 branch[P], norm[P];
  const bool weighted = a.mode == kSumWeighted, own_rows = weighted && a.per == 1;
  while (rows_left<S::T>(at.on())) {
    const bool on = at.on();
    const int row = on ? at.row : 0, group = on ? at.group : 0;
    uint4 gate_raw, scale_raw;
    const bool other = group != held;
    if (other || weighted) {
      held = group;
      if (a.h) request_vector(gate_raw, a.gate, a.tc, cond_at(group, a.ldgate), col);
      request_vector(scale_raw, a.scale, a.tc, cond_at(group, a.ldscale), col);
    }
    ring_ready<TPR, CL, VEC>(sub);
    if (other) {
      float2 x[P];
#pragma unroll
      for (int i = 0; i < P; ++i) {
        branch[i] = alpha;
        norm[i] = both(1.f);
      }
      if (a.h && a.gate) {
        take_vector(gate_raw, a.gate, a.tc, cond_at(group, a.ldgate), col, x);
#pragma unroll
        for (int i = 0; i < P; ++i) branch[i] = each_mul2(branch[i], x[i]);
      }
      if (FULL && a.wp) {
        load_vector(a.wp, a.tw, 0, col, x);
#pragma unroll
        for (int i = 0; i < P; ++i) branch[i] = each_mul2(branch[i], x[i]);
      }
      if (!weighted && a.scale) {
        take_vector(scale_raw, a.scale, a.tc, cond_at(group, a.ldscale), col, x);
#pragma unroll
        for (int i = 0; i < P; ++i) norm[i] = each_add2(norm[i], x[i]);
      }
      if (a.w) {
        load_vector(a.w, a.tw, 0, col, x);
#pragma unroll
        for (int i = 0; i < P; ++i) norm[i] = each_mul2(norm[i], x[i]);
      }
    }
    const uint4* mine = ring + stage * G::kStage;
    const float4* stats = reinterpret_cast<const float4*>(mine + G::kStats + threadIdx.x / kWarp * 2);
    float2 v[P], q[P], dx[P], x[P];
    ring_take(mine + G::kR, row_of<TR>(a.r, row, a.ldr), col, sub, v);
    // r' again, and xhat
    Kept kept;
    float post_scale = 1.f;
    if (a.h) {
      ring_take(mine + 2 * G::kR + G::kH, row_of<TH>(a.h, row, a.ldh), col, sub, q);
      if (drops) kept = kept_columns(a.drop, dstep, row, col, lane);
      if (FULL && a.post) {
        const float4 st = stats[1];
        post_scale = st.z;
        shift_row(q, st.x, col, VEC);
        scale_row(q, st.y, st.z, col, VEC);
      }
#pragma unroll
      for (int i = 0; i < P; ++i) add_branch(v[i], branch[i], q[i], drops, kept, i);
      if (drops && !a.post) {                                   // (0 times what was dropped is not always 0; behind post, all of its row is NaN then)
#pragma unroll
        for (int i = 0; i < P; ++i) q[i] = select_kept(q[i], kept, i);
      }
    }
    const float4 st = stats[0];
    shift_row(v, st.x, col, VEC);
    scale_row(v, st.y, st.z, col, VEC);
    ring_take(mine + 2 * G::kR, row_of<TH>(a.dn, row, a.lddn), col, sub, dx);
    if (S::T < 32 && !on) {                                     // (nothing of a row that is not there may reach the sums)
#pragma unroll
      for (int i = 0; i < P; ++i) v[i] = q[i] = dx[i] = both(0.f);
    }
    // A and B, and dn (1 + scale) w
    if (own_rows && a.dshift) store_vector(a.dshift, a.tc, cond_at(row, a.lddshift), col, on, dx);
    if (own_rows && a.dscale) {
      float2 o[P];
#pragma unroll
      for (int i = 0; i < P; ++i) o[i] = each_mul2(dx[i], v[i]);
      if (a.w) {
        load_vector(a.w, a.tw, 0, col, x);
#pragma unroll
        for (int i = 0; i < P; ++i) o[i] = each_mul2(o[i], x[i]);
      }
      if (a.b) {
        load_vector(a.b, a.tw, 0, col, x);
#pragma unroll
        for (int i = 0; i < P; ++i) o[i] = each_fma2(dx[i], x[i], o[i]);
      }
      store_vector(a.dscale, a.tc, cond_at(row, a.lddscale), col, on, o);
    }
    const auto add_ab = [&]() {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        sa[i] = each_fma2(dx[i], v[i], sa[i]);
        sb[i] = each_add2(sb[i], dx[i]);
      }
    };
    if (!weighted) add_ab();
    if (weighted && a.scale) {
      take_vector(scale_raw, a.scale, a.tc, cond_at(group, a.ldscale), col, x);
#pragma unroll
      for (int i = 0; i < P; ++i) dx[i] = each_fma2(dx[i], x[i], dx[i]);
    }
    if (weighted) add_ab();
    if (a.w || (!weighted && a.scale)) {
#pragma unroll
      for (int i = 0; i < P; ++i) dx[i] = each_mul2(dx[i], norm[i]);
    }
    float c[2];
    pair_sums(dx, v, c);
    sums(c);
    // (behind a sum: all threads of the group are done with the row before, whose place this takes)
    request(at.row + kRingStages - 1, stage == 0 ? kRingStages - 1 : stage - 1);
    const float2 c1 = both(a.rms ? 0.f : -c[0] * inv_d), c2 = both(-c[1] * inv_d);
    float2 g[P];
    if (a.dr) {
      ring_take(mine, row_of<TR>(a.dr, row, a.lddr), col, sub, g);
    } else {
#pragma unroll
      for (int i = 0; i < P; ++i) g[i] = both(0.f);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) g[i] = each_fma2(both(st.z), each_fma2(c2, v[i], each_add2(dx[i], c1)), g[i]);
    if (a.dr_in) store_row(row_of<TR>(a.dr_in, row, a.lddr_in), col, on, g);
    if (a.h) {
      // D g; alpha times its product with post(h) (or h) is the row's C
      if (drops) {
#pragma unroll
        for (int i = 0; i < P; ++i) g[i] = select_kept(g[i], kept, i);
      }
      if (own_rows && a.dgate) {
        float2 o[P];
#pragma unroll
        for (int i = 0; i < P; ++i) o[i] = each_mul2(alpha, each_mul2(g[i], q[i]));
        if (FULL && a.wp) {
          load_vector(a.wp, a.tw, 0, col, x);
#pragma unroll
          for (int i = 0; i < P; ++i) o[i] = each_mul2(o[i], x[i]);
        }
        store_vector(a.dgate, a.tc, cond_at(row, a.lddgate), col, on, o);
      }
      if (weighted && a.gate) {
        take_vector(gate_raw, a.gate, a.tc, cond_at(group, a.ldgate), col, x);
#pragma unroll
        for (int i = 0; i < P; ++i) sq[i] = S::T < 32 && !on ? sq[i] : each_fma2(each_mul2(g[i], x[i]), q[i], sq[i]);
      } else {
#pragma unroll
        for (int i = 0; i < P; ++i) sq[i] = S::T < 32 && !on ? sq[i] : each_fma2(g[i], q[i], sq[i]);
      }
      if (a.dh) {
#pragma unroll
        for (int i = 0; i < P; ++i) g[i] = each_mul2(branch[i], g[i]);
        if (FULL && a.post) {
          if (!VEC) {                                           // (beyond d, g holds the mean that it took off)
#pragma unroll
            for (int e = 0; e < kBlock; ++e)
              if (!col.has(e)) element(g, e) = 0.f;
          }
          float e2[2];
          pair_sums(g, q, e2);
          sums(e2);
          const float2 p1 = both(a.rms ? 0.f : -e2[0] * inv_d), p2 = both(-e2[1] * inv_d), ps = both(post_scale);
#pragma unroll
          for (int i = 0; i < P; ++i) g[i] = each_mul2(ps, each_fma2(p2, q[i], each_add2(g[i], p1)));
        }
        store_row(row_of<TH>(a.dh, row, a.lddh), col, on, g);
      }
    }
    at.next();
    stage = stage + 1 == kRingStages ? 0 : stage + 1;
    // a group's rows, or this worker's of them, are done: its sums are the group's, or a part of them
    if (a.mode == kSumGroups && on && (at.left == 1 || !at.on())) {
      const bool from_here = row - (a.per - at.left) >= begin, whole = from_here && at.left == 1;
#pragma unroll
      for (int i = 0; i < P; ++i) sq[i] = each_mul2(alpha, sq[i]);
      float* total = a.part + (size_t)worker * 3 * d;
      float2 f[P], k[P];
#pragma unroll
      for (int i = 0; i < P; ++i) f[i] = k[i] = both(0.f);
      if (a.scale) load_vector(a.scale, a.tc, cond_at(group, a.ldscale), col, f);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        f[i].x += 1.0f; f[i].y += 1.0f;
        k[i] = both(1.0f);
      }
      if (a.h && a.gate) load_vector(a.gate, a.tc, cond_at(group, a.ldgate), col, k);
      add_total(total, sa, f, col, first_flush);
      add_total(total + d, sb, f, col, first_flush);
      add_total(total + 2 * d, sq, k, col, first_flush);
      if (whole) {
        if (a.dshift) store_vector(a.dshift, a.tc, cond_at(group, a.lddshift), col, true, sb);
        if (a.dscale) {
          if (a.w) {
            load_vector(a.w, a.tw, 0, col, x);
#pragma unroll
            for (int i = 0; i < P; ++i) sa[i] = each_mul2(sa[i], x[i]);
          }
          if (a.b) {
            load_vector(a.b, a.tw, 0, col, x);
#pragma unroll
            for (int i = 0; i < P; ++i) sa[i] = each_fma2(sb[i], x[i], sa[i]);
          }
          store_vector(a.dscale, a.tc, cond_at(group, a.lddscale), col, true, sa);
        }
        if (a.dgate) {
          if (FULL && a.wp) {
            load_vector(a.wp, a.tw, 0, col, x);
#pragma unroll
            for (int i = 0; i < P; ++i) sq[i] = each_mul2(sq[i], x[i]);
          }
          store_vector(a.dgate, a.tc, cond_at(group, a.lddgate), col, true, sq);
        }
      } else {
        float* part = a.group_part + ((size_t)worker * 2 + (from_here ? 1 : 0)) * 3 * d;
        store_typed_vector(part, col, true, sa);
        store_typed_vector(part + d, col, true, sb);
        store_typed_vector(part + 2 * d, col, true, sq);
      }
#pragma unroll
      for (int i = 0; i < P; ++i) sa[i] = sb[i] = sq[i] = both(0.f);
      first_flush = false;
    }
    at.next_group(a.per);
  }
  if (a.mode != kSumGroups && worker < a.workers) {
    float* total = a.part + (size_t)worker * 3 * d;
    store_typed_vector(total, col, true, sa);
    store_typed_vector(total + d, col, true, sb);
#pragma unroll
    for (int i = 0; i < P; ++i) sq[i] = each_mul2(alpha, sq[i]);
    store_typed_vector(total + 2 * d, col, true, sq);
  }
}

// ---------------------------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------------------------

constexpr int kRowDevices = 64;
constexpr int kRowSms = 148;

// CTAs (clusters) of a kernel that the device holds at once, looked up once per device, and its shared-memory limit raised
template <class K>
cudaError_t row_resident(K kernel, std::atomic<int>* cache, int threads, int smem, int cluster, int* n) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= kRowDevices) return cudaErrorInvalidDevice;
  int r = cache[dev].load(std::memory_order_acquire);
  if (r == 0) {
    if (smem > 40 * 1024 && (e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) != cudaSuccess) return e;
    int sms = 0;
    if ((e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
    if (cluster > 1) {
      cudaLaunchConfig_t cfg{};
      cfg.gridDim = dim3((unsigned)(sms / cluster * cluster));
      cfg.blockDim = dim3(threads);
      cfg.dynamicSmemBytes = smem;
      cudaLaunchAttribute attr{};
      attr.id = cudaLaunchAttributeClusterDimension;
      attr.val.clusterDim.x = (unsigned)cluster; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
      cfg.attrs = &attr;
      cfg.numAttrs = 1;
      if ((e = cudaOccupancyMaxActiveClusters(&r, kernel, &cfg)) != cudaSuccess) return e;
    } else {
      if ((e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&r, kernel, threads, smem)) != cudaSuccess) return e;
      r *= sms;
    }
    if (r < 1) return cudaErrorLaunchOutOfResources;
    cache[dev].store(r, std::memory_order_release);
  }
  *n = r;
  return cudaSuccess;
}

template <class K, class... Args>
cudaError_t row_launch(K kernel, dim3 grid, int threads, int smem, int cluster, cudaStream_t st, const Args&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
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

template <class TR, class TH, int TPR, int CL, bool VEC, bool FULL, bool HELD>
cudaError_t residual_fwd_k(const ResidualNormArgs& a, cudaStream_t st) {
  using S = ResidualShape<TPR, CL>;
  constexpr int smem = kRingStages * (RingRow<TR, TPR, CL, VEC>::kPieces + RingRow<TH, TPR, CL, VEC>::kPieces) * 16;
  static std::atomic<int> cache[kRowDevices];
  int resident = 0;
  const cudaError_t e = row_resident(k_residual_norm<TR, TH, TPR, CL, VEC, FULL, HELD>, cache, S::kCta, smem, CL, &resident);
  if (e != cudaSuccess) return e;
  ResidualNormArgs g = a;
  const int64_t most = (int64_t)resident * S::kRows;
  g.share = (int)((a.rows + most - 1) / most);
  g.workers = (a.rows + g.share - 1) / g.share;
  const int grid = (g.workers + S::kRows - 1) / S::kRows;
  return row_launch(k_residual_norm<TR, TH, TPR, CL, VEC, FULL, HELD>, dim3((unsigned)(grid * CL)), S::kCta, smem, CL, st, g);
}

template <class TR, class TH, int TPR, int CL, bool VEC, bool FULL>
cudaError_t residual_bwd_k(ResidualNormArgs& g, cudaStream_t st) {
  using S = ResidualShape<TPR, CL>;
  constexpr int smem = ResidualBwd<TR, TH, TPR, CL, VEC>::kSmemBytes;
  static std::atomic<int> cache[kRowDevices];
  int resident = 0;
  const cudaError_t e = row_resident(k_residual_norm_bwd<TR, TH, TPR, CL, VEC, FULL>, cache, S::kCta, smem, CL, &resident);
  if (e != cudaSuccess) return e;
  // no more workers than run at once, nor than the workspace was made for
  const int64_t most = std::min<int64_t>(g.workers, (int64_t)resident * S::kRows);
  g.share = (int)((g.rows + most - 1) / most);
  g.workers = (g.rows + g.share - 1) / g.share;
  const int grid = (g.workers + S::kRows - 1) / S::kRows;
  return row_launch(k_residual_norm_bwd<TR, TH, TPR, CL, VEC, FULL>, dim3((unsigned)(grid * CL)), S::kCta, smem, CL, st, g);
}

// rows of whole pieces of eight columns
inline bool pieces8(const void* p, int64_t ld, int type) {
  const int bytes = type == SDS_F32 ? 32 : 16;
  return reinterpret_cast<uintptr_t>(p) % bytes == 0 && ld * (bytes / 8) % bytes == 0;
}

template <class TR, class TH, int TPR, int CL, bool VEC>
cudaError_t residual_t(ResidualNormArgs& a, bool backward, cudaStream_t st) {
  const bool full = a.post || a.drop.threshold != 0;
  if (backward) return full ? residual_bwd_k<TR, TH, TPR, CL, VEC, true>(a, st) : residual_bwd_k<TR, TH, TPR, CL, VEC, false>(a, st);
  // (see HELD)
  if constexpr (VEC && CL == 1 && std::is_same<TR, float>::value) {
    const int vectors = (a.gate != nullptr) + (a.wp != nullptr) + (a.w != nullptr) + (a.b != nullptr) + (a.scale != nullptr) + (a.shift != nullptr);
    if (full && a.h && vectors >= 2 && a.per >= 8) return residual_fwd_k<TR, TH, TPR, CL, VEC, true, true>(a, st);
  }
  return full ? residual_fwd_k<TR, TH, TPR, CL, VEC, true, false>(a, st) : residual_fwd_k<TR, TH, TPR, CL, VEC, false, false>(a, st);
}
template <class TR, class TH, int TPR, int CL>
cudaError_t residual_t(ResidualNormArgs& a, bool vec, bool backward, cudaStream_t st) {
  return vec ? residual_t<TR, TH, TPR, CL, true>(a, backward, st) : residual_t<TR, TH, TPR, CL, false>(a, backward, st);
}

// threads of a row's group: part of a warp, one CTA, a cluster of two or four beyond 4096 columns
inline int residual_threads(int d) { return d <= 64 ? 8 : d <= 256 ? 32 : d <= 512 ? 64 : d <= 1024 ? 128 : d <= 2048 ? 256 : d <= 4096 ? 512 : d <= 8192 ? 1024 : 2048; }
template <class TR, class TH>
cudaError_t residual_launch(ResidualNormArgs& a, bool vec, bool backward, cudaStream_t st) {
  switch (residual_threads(a.d)) {
    case 8: return residual_t<TR, TH, 8, 1>(a, vec, backward, st);
    case 32: return residual_t<TR, TH, 32, 1>(a, vec, backward, st);
    case 64: return residual_t<TR, TH, 64, 1>(a, vec, backward, st);
    case 128: return residual_t<TR, TH, 128, 1>(a, vec, backward, st);
    case 256: return residual_t<TR, TH, 256, 1>(a, vec, backward, st);
    case 512: return residual_t<TR, TH, 512, 1>(a, vec, backward, st);
    case 1024: return residual_t<TR, TH, 1024, 2>(a, vec, backward, st);
    default: return residual_t<TR, TH, 2048, 4>(a, vec, backward, st);
  }
}

}  // namespace

// one source for each pair of types; backward: a.workers becomes the number of workers launched
cudaError_t residual_f32(ResidualNormArgs& a, bool vec, bool backward, cudaStream_t st);
cudaError_t residual_f32_bf16(ResidualNormArgs& a, bool vec, bool backward, cudaStream_t st);
cudaError_t residual_f32_f16(ResidualNormArgs& a, bool vec, bool backward, cudaStream_t st);
cudaError_t residual_bf16(ResidualNormArgs& a, bool vec, bool backward, cudaStream_t st);
cudaError_t residual_f16(ResidualNormArgs& a, bool vec, bool backward, cudaStream_t st);

}  // namespace sds
