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
// Sums over the rows of a group: A = sum dn xhat, B = sum dn, C = sum g D q/wp. They give every gradient of a vector:
//   dshift = B, dscale = w A + b B, dgate = alpha wp C;  dw = sum_groups (1 + scale) A, db = sum_groups (1 + scale) B,
//   dwp = sum_groups alpha gate C.
//
// Bound by memory: r, h in and r', n out; r, h, dn, dr in and the gradients of r and h out. The backward pass makes r' again from r and
// h, which it needs anyway, so r' need not be kept, and xhat is not that of a rounded r'. A group of threads holds a row in registers,
// eight columns a thread. Statistics are held in float; layer norm takes them around the rounded mean and takes the mean's
// remainder back out, so that rows far from zero keep 24 bits of their spread.
//
// Sums over rows: a worker (the group of threads) adds its rows in registers, workers' sums are added by a second kernel in a
// fixed order (no atomics: same bits on every run).
#pragma once

#include <algorithm>
#include <atomic>

#include "sds_device.cuh"
#include "sds_layers.h"
#include "sds_rows.cuh"

namespace sds {

namespace {

constexpr int kStreamDropout = 3;
constexpr int kE = 8;                             // columns of a thread: one 16-byte access of 16-bit types, one block of the generator

// how the rows of a backward call are dealt out (ResidualNormArgs::mode)
enum ResidualMode : int {
  kSumAll = 0,      // one group: a worker's rows, their plain sums A, B, C
  kSumWeighted = 1, // sums weighted with each row's own scale and gate; rows that are groups of their own write their gradients at once
  kSumGroups = 2,   // pieces of groups: plain sums per piece, and the worker's weighted sums over its pieces
};

// eight columns of a thread as they lie in memory
template <class T, bool VEC> struct Raw;
template <class T> struct Raw<T, true> {
  static constexpr int kUnits = sizeof(T) / 2;
  uint4 q[kUnits];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < kUnits; ++i) q[i] = *(reinterpret_cast<const uint4*>(p) + i);
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kUnits; ++i) q[i] = make_uint4(0u, 0u, 0u, 0u);
  }
};

__device__ __forceinline__ void words_to(const uint4 (&q)[2], float (&o)[kE], float) {
  const uint32_t w[8] = {q[0].x, q[0].y, q[0].z, q[0].w, q[1].x, q[1].y, q[1].z, q[1].w};
#pragma unroll
  for (int e = 0; e < kE; ++e) o[e] = __uint_as_float(w[e]);
}
__device__ __forceinline__ void words_to(const uint4 (&q)[1], float (&o)[kE], Bf16) {
  const uint32_t w[4] = {q[0].x, q[0].y, q[0].z, q[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o[2 * i] = __uint_as_float(w[i] << 16);
    o[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void words_to(const uint4 (&q)[1], float (&o)[kE], F16) {
  const uint32_t w[4] = {q[0].x, q[0].y, q[0].z, q[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    o[2 * i] = v.x;
    o[2 * i + 1] = v.y;
  }
}
__device__ __forceinline__ void store_words(float* p, const float (&v)[kE]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
template <class T> __device__ __forceinline__ void store_words(T* p, const float (&v)[kE]) {
  Pack<T, 8> o;
#pragma unroll
  for (int i = 0; i < 4; ++i) put2(o, i, make_float2(v[2 * i], v[2 * i + 1]));
  *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(&o);
}

// The columns of a group's thread t. VEC: eight neighbours. Else: 32 neighbours for a warp, eight times, each as many columns further as the
// group has threads in a CTA.
template <int TPR, int CL, bool VEC> struct Columns {
  static constexpr int T = TPR / CL;
  int c0;
  __device__ explicit Columns(int t) : c0(VEC ? t * kE : t / T * T * kE + t % T) {}
  __device__ __forceinline__ int at(int e) const { return VEC ? c0 + e : c0 + e * T; }
};

template <class T, class C>
__device__ __forceinline__ void load_scalar(const T* row, const C& col, int d, float (&o)[kE]) {
#pragma unroll
  for (int e = 0; e < kE; ++e) o[e] = col.at(e) < d ? Conv<T>::get(row[col.at(e)]) : 0.f;
}
template <class T, bool VEC, class C>
__device__ __forceinline__ void store_row(T* row, const C& col, int d, const float (&v)[kE]) {
  if (VEC) {
    if (col.c0 < d) store_words(row + col.c0, v);
  } else {
#pragma unroll
    for (int e = 0; e < kE; ++e)
      if (col.at(e) < d) row[col.at(e)] = Conv<T>::put(v[e]);
  }
}

// a thread's columns of a vector of any of the three types, `fill` where there is none
template <bool VEC, class C>
__device__ __forceinline__ void load_vector8(const void* p, int type, bool wide, size_t off, const C& col, int d, float fill, float (&o)[kE]) {
  if (!p) {
#pragma unroll
    for (int e = 0; e < kE; ++e) o[e] = fill;
  } else if (VEC && wide) {
    if (col.c0 >= d) {
#pragma unroll
      for (int e = 0; e < kE; ++e) o[e] = 0.f;
    } else if (type == SDS_F32) {
      Raw<float, true> r;
      r.load(static_cast<const float*>(p) + off + col.c0);
      words_to(r.q, o, 0.f);
    } else if (type == SDS_BF16) {
      Raw<Bf16, true> r;
      r.load(static_cast<const Bf16*>(p) + off + col.c0);
      words_to(r.q, o, Bf16{});
    } else {
      Raw<F16, true> r;
      r.load(static_cast<const F16*>(p) + off + col.c0);
      words_to(r.q, o, F16{});
    }
  } else {
#pragma unroll
    for (int e = 0; e < kE; ++e) o[e] = col.at(e) < d ? load_any(p, type, off + col.at(e)) : 0.f;
  }
}
template <bool VEC, class C>
__device__ __forceinline__ void store_vector8(void* p, int type, bool wide, size_t off, const C& col, int d, const float (&v)[kE]) {
  if (VEC && wide) {
    if (col.c0 >= d) return;
    if (type == SDS_F32) store_words(static_cast<float*>(p) + off + col.c0, v);
    else if (type == SDS_BF16) store_words(static_cast<Bf16*>(p) + off + col.c0, v);
    else store_words(static_cast<F16*>(p) + off + col.c0, v);
  } else {
#pragma unroll
    for (int e = 0; e < kE; ++e)
      if (col.at(e) < d) store_any(p, type, off + col.at(e), v[e]);
  }
}

// One bit for each of the eight columns of a block: kept. 16 of the block's 128 bits decide a column, low half of a word first.
__device__ __forceinline__ uint32_t kept_block(const DropoutArgs& a, uint32_t step, uint64_t row, uint32_t block) {
  const uint4 x = philox_block(a.seed, kStreamDropout, row, step, block);
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t kept = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    kept |= ((w[i] & 0xffffu) >= a.threshold ? 1u : 0u) << (2 * i);
    kept |= ((w[i] >> 16) >= a.threshold ? 1u : 0u) << (2 * i + 1);
  }
  return kept;
}
// The same for a thread's columns. Where these are not one block, a warp's 256 columns are 32 blocks: a lane draws one, and the
// bits change hands. (All 32 lanes call it.)
template <int TPR, int CL, bool VEC>
__device__ __forceinline__ uint32_t kept_columns(const DropoutArgs& a, uint32_t step, int row, const Columns<TPR, CL, VEC>& col, int lane) {
  if (VEC) return kept_block(a, step, a.row0 + (uint32_t)row, (uint32_t)col.c0 >> 3);
  const uint32_t mine = kept_block(a, step, a.row0 + (uint32_t)row,
                                   (uint32_t)(col.c0 - lane + (lane >> 2) * Columns<TPR, CL, VEC>::T + (lane & 3) * 8) >> 3);
  uint32_t kept = 0;
#pragma unroll
  for (int e = 0; e < kE; ++e) kept |= ((__shfl_sync(kAll, mine, e * 4 + (lane >> 3)) >> (lane & 7)) & 1u) << e;
  return kept;
}
__device__ __forceinline__ uint32_t dropout_step(const DropoutArgs& a) { return a.step + (a.step_dev ? (uint32_t)*a.step_dev : 0u); }

// Sums over a group, each call in the other half of its slots: a half is written again only after the barrier of the call between.
template <int TPR, int CL> struct GroupSums {
  static constexpr int NW = TPR > 32 ? TPR / 32 : 1;
  float* slot;
  int t, bar, flip = 0;
  __device__ GroupSums(float* slots, int sub, int t_) : slot(slots + sub * 8 * NW), t(t_), bar(1 + sub) {}
  template <int N> __device__ __forceinline__ void operator()(float (&v)[N]) {
    group_sum<TPR, N, CL>(v, slot + flip * 4 * NW, t, bar);
    flip ^= 1;
  }
};

// r + alpha gate D q, in the forward pass and again in the backward one
__device__ __forceinline__ float add_branch(float r, float k, float q, uint32_t kept, int e, const DropoutArgs& drop) {
  return (kept >> e) & 1u ? fmaf(drop.threshold ? k * drop.scale : k, q, r) : r;
}

struct RowStats { float mean, rest, scale; };
// Turns the row v into xhat. Columns beyond d hold zeros, and do so afterwards.
template <int TPR, int CL, class C>
__device__ __forceinline__ RowStats normalise(float (&v)[kE], GroupSums<TPR, CL>& sums, const C& col, int d, float inv_d, bool rms, float eps) {
  RowStats st{0.f, 0.f, 0.f};
  if (rms) {
    float s[1] = {0.f};
#pragma unroll
    for (int e = 0; e < kE; ++e) s[0] = fmaf(v[e], v[e], s[0]);
    sums(s);
    st.scale = rsqrtf(fmaf(s[0], inv_d, eps));
  } else {
    float s[1] = {0.f};
#pragma unroll
    for (int e = 0; e < kE; ++e) s[0] += v[e];
    sums(s);
    st.mean = s[0] * inv_d;
    float q[2] = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      v[e] = col.at(e) < d ? v[e] - st.mean : 0.f;
      q[0] += v[e];
      q[1] = fmaf(v[e], v[e], q[1]);
    }
    sums(q);
    st.rest = q[0] * inv_d;
    st.scale = rsqrtf(fmaf(-st.rest, st.rest, q[1] * inv_d) + eps);
#pragma unroll
    for (int e = 0; e < kE; ++e) v[e] = col.at(e) < d ? v[e] - st.rest : 0.f;
  }
#pragma unroll
  for (int e = 0; e < kE; ++e) v[e] *= st.scale;
  return st;
}

template <int TPR, int CL> struct ResidualShape {
  static constexpr int T = TPR / CL;                            // threads of a row in one CTA
  static constexpr int kCta = T < 128 ? 128 : T;
  static constexpr int kRows = kCta / T;                        // rows of a CTA at a time
  static constexpr int kSlots = 2 * kRows * 4 * (TPR > 32 ? TPR / 32 : 1);
};

template <class TR, class TH, int TPR, int CL, bool VEC>
__global__ void __launch_bounds__(ResidualShape<TPR, CL>::kCta) k_residual_norm(const ResidualNormArgs a) {
  using S = ResidualShape<TPR, CL>;
  __shared__ __align__(16) float slots[S::kSlots];
  const int sub = threadIdx.x / S::T, lane = threadIdx.x & 31;
  const int t = (CL > 1 ? (int)(blockIdx.x % CL) * S::T : 0) + (int)threadIdx.x % S::T;
  const Columns<TPR, CL, VEC> col(t);
  GroupSums<TPR, CL> sums(slots, sub, t);
  if (CL > 1) {                                                 // the peers' slots are there to be written
    cluster_arrive();
    cluster_wait();
  }
  start_after_prior_kernel();
  const int d = a.d, step = (int)gridDim.x / CL * S::kRows;
  const float inv_d = 1.0f / (float)d;
  const uint32_t dstep = a.drop.threshold ? dropout_step(a.drop) : 0u;
  const bool live = col.c0 < d;
  Raw<TR, true> rn;
  Raw<TH, true> hn;
  const auto fetch = [&](int row) {
    if (!VEC) return;
    rn.zero();
    hn.zero();
    if (live && row < a.rows) {
      rn.load(static_cast<const TR*>(a.r) + (size_t)row * a.ldr + col.c0);
      if (a.h) hn.load(static_cast<const TH*>(a.h) + (size_t)row * a.ldh + col.c0);
    }
  };
  int row = (int)blockIdx.x / CL * S::kRows + sub;
  fetch(row);
  for (; row < a.rows; row += step) {
    float v[kE], q[kE];
    if (VEC) {
      words_to(rn.q, v, TR{});
      words_to(hn.q, q, TH{});
    } else {
      load_scalar(static_cast<const TR*>(a.r) + (size_t)row * a.ldr, col, d, v);
      if (a.h) load_scalar(static_cast<const TH*>(a.h) + (size_t)row * a.ldh, col, d, q);
    }
    if (row < a.rows - step) fetch(row + step);
    const int group = a.per == 1 ? row : row / a.per;
    if (a.h) {
      if (a.post) {
        const RowStats st = normalise(q, sums, col, d, inv_d, a.rms, a.eps);
        float wp[kE];
        load_vector8<VEC>(a.wp, a.tw, a.wide_w, 0, col, d, 1.f, wp);
#pragma unroll
        for (int e = 0; e < kE; ++e) q[e] *= wp[e];
        if (a.stats && t == 0) {
          a.stats[(size_t)3 * a.rows + row] = st.mean;
          a.stats[(size_t)4 * a.rows + row] = st.rest;
          a.stats[(size_t)5 * a.rows + row] = st.scale;
        }
      }
      const uint32_t kept = a.drop.threshold ? kept_columns(a.drop, dstep, row, col, lane) : 0xffu;
      float gate[kE];
      load_vector8<VEC>(a.gate, a.tc, a.wide_c, (size_t)group * a.ldgate, col, d, 1.f, gate);
#pragma unroll
      for (int e = 0; e < kE; ++e) v[e] = add_branch(v[e], a.alpha * gate[e], q[e], kept, e, a.drop);
      store_row<TR, VEC>(static_cast<TR*>(a.out) + (size_t)row * a.ldo, col, d, v);
    }
    const RowStats st = normalise(v, sums, col, d, inv_d, a.rms, a.eps);
    if (a.stats && t == 0) {
      a.stats[row] = st.mean;
      a.stats[(size_t)a.rows + row] = st.rest;
      a.stats[(size_t)2 * a.rows + row] = st.scale;
    }
    if (a.w || a.b) {
      float w[kE], b[kE];
      load_vector8<VEC>(a.w, a.tw, a.wide_w, 0, col, d, 1.f, w);
      load_vector8<VEC>(a.b, a.tw, a.wide_w, 0, col, d, 0.f, b);
#pragma unroll
      for (int e = 0; e < kE; ++e) v[e] = fmaf(v[e], w[e], b[e]);
    }
    if (a.scale || a.shift) {
      float sc[kE], sh[kE];
      load_vector8<VEC>(a.scale, a.tc, a.wide_c, (size_t)group * a.ldscale, col, d, 0.f, sc);
      load_vector8<VEC>(a.shift, a.tc, a.wide_c, (size_t)group * a.ldshift, col, d, 0.f, sh);
#pragma unroll
      for (int e = 0; e < kE; ++e) v[e] = fmaf(v[e], 1.0f + sc[e], sh[e]);
    }
    store_row<TH, VEC>(static_cast<TH*>(a.n) + (size_t)row * a.ldn, col, d, v);
  }
}

// ---------------------------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------------------------

// The rows to come pass through a ring in shared memory, each thread's own columns: it copies and reads them itself, so there is no
// barrier, and the copies take no registers.
template <class TR, class TH> struct ResidualRing {
  static constexpr int kStages = 3;
  static constexpr int kR = sizeof(TR) / 2, kH = sizeof(TH) / 2;          // 16-byte pieces of a thread's columns
  static constexpr int kPieces = 2 * kR + 2 * kH;                         // dr, r, dn, h
};

__device__ __forceinline__ void copy16(void* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}

// Where a worker stands: its row, the end of its piece, the piece.
struct RowWalk {
  int row, end, piece;
  __device__ __forceinline__ void enter(const ResidualNormArgs& a, int p) {
    piece = p;
    if (a.mode == kSumGroups) {
      const int g = p / a.pieces, j = p - g * a.pieces;
      row = g * a.per + j * a.piece;
      end = min(row + a.piece, (g + 1) * a.per);
    } else {
      row = p * a.piece;
      end = min(row + a.piece, a.rows);
    }
  }
  __device__ __forceinline__ bool done(const ResidualNormArgs& a) const { return piece >= a.total; }
  __device__ __forceinline__ void next(const ResidualNormArgs& a) {
    if (++row < end) return;
    const int p = piece + a.workers;
    if (p < a.total) enter(a, p);
    else piece = a.total;
  }
};

template <class TR, class TH, int TPR, int CL, bool VEC>
__global__ void __launch_bounds__(ResidualShape<TPR, CL>::kCta, ResidualShape<TPR, CL>::kCta <= 256 ? 512 / ResidualShape<TPR, CL>::kCta : 1)
    k_residual_norm_bwd(const ResidualNormArgs a) {
  using S = ResidualShape<TPR, CL>;
  using G = ResidualRing<TR, TH>;
  extern __shared__ uint4 ring[];                               // [stage][piece][thread] (VEC)
  __shared__ __align__(16) float slots[S::kSlots];
  const int sub = threadIdx.x / S::T, lane = threadIdx.x & 31;
  const int t = (CL > 1 ? (int)(blockIdx.x % CL) * S::T : 0) + (int)threadIdx.x % S::T;
  const Columns<TPR, CL, VEC> col(t);
  GroupSums<TPR, CL> sums(slots, sub, t);
  if (CL > 1) {
    cluster_arrive();
    cluster_wait();
  }
  start_after_prior_kernel();
  const int worker = (int)blockIdx.x / CL * S::kRows + sub;
  const int d = a.d;
  const float inv_d = 1.0f / (float)d;
  const uint32_t dstep = a.drop.threshold ? dropout_step(a.drop) : 0u;
  const bool live = col.c0 < d;
  if (worker >= a.workers) return;                              // (a whole group; with clusters there is none)
  float sa[kE] = {}, sb[kE] = {}, sc_[kE] = {};                 // A, B, C, or their weighted forms
  bool first_flush = true;

  RowWalk ahead, at;
  at.enter(a, worker);
  ahead = at;
  const auto request = [&](int stage) {
    if (VEC && live && !ahead.done(a)) {
      uint4* to = ring + (size_t)stage * G::kPieces * S::kCta + threadIdx.x;
      const TR* dr = static_cast<const TR*>(a.dr) + (size_t)ahead.row * a.lddr + col.c0;
      const TR* r = static_cast<const TR*>(a.r) + (size_t)ahead.row * a.ldr + col.c0;
      const TH* dn = static_cast<const TH*>(a.dn) + (size_t)ahead.row * a.lddn + col.c0;
      const TH* h = static_cast<const TH*>(a.h) + (size_t)ahead.row * a.ldh + col.c0;
#pragma unroll
      for (int i = 0; i < G::kR; ++i) {
        if (a.dr) copy16(to + i * S::kCta, dr + i * 4);
        copy16(to + (G::kR + i) * S::kCta, r + i * 4);
      }
#pragma unroll
      for (int i = 0; i < G::kH; ++i) {
        copy16(to + (2 * G::kR + i) * S::kCta, dn + i * 4);
        if (a.h) copy16(to + (2 * G::kR + G::kH + i) * S::kCta, h + i * 4);
      }
    }
    if (!ahead.done(a)) ahead.next(a);
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if (VEC)
    for (int s = 0; s < G::kStages - 1; ++s) request(s);
  int stage = 0;

  for (; !at.done(a);) {
    const int row = at.row, group = a.per == 1 ? row : row / a.per;
    float v[kE], q[kE], dx[kE], g[kE];
    if (VEC) {
      asm volatile("cp.async.wait_group %0;" ::"n"(G::kStages - 2) : "memory");
      const uint4* from = ring + (size_t)stage * G::kPieces * S::kCta + threadIdx.x;
      const auto take = [&](auto type, int piece, float (&o)[kE], bool there) {
        uint4 w[sizeof(type) / 2];
#pragma unroll
        for (int i = 0; i < (int)sizeof(type) / 2; ++i) w[i] = there && live ? from[(piece + i) * S::kCta] : make_uint4(0u, 0u, 0u, 0u);
        words_to(w, o, type);
      };
      take(TR{}, 0, g, a.dr != nullptr);
      take(TR{}, G::kR, v, true);
      take(TH{}, 2 * G::kR, dx, true);
      take(TH{}, 2 * G::kR + G::kH, q, a.h != nullptr);
    } else {
#pragma unroll
      for (int e = 0; e < kE; ++e) g[e] = q[e] = 0.f;
      if (a.dr) load_scalar(static_cast<const TR*>(a.dr) + (size_t)row * a.lddr, col, d, g);
      load_scalar(static_cast<const TR*>(a.r) + (size_t)row * a.ldr, col, d, v);
      load_scalar(static_cast<const TH*>(a.dn) + (size_t)row * a.lddn, col, d, dx);
      if (a.h) load_scalar(static_cast<const TH*>(a.h) + (size_t)row * a.ldh, col, d, q);
    }
    if (VEC) {
      const int free_stage = stage == 0 ? G::kStages - 1 : stage - 1;     // (its row is done)
      request(free_stage);
      stage = stage + 1 == G::kStages ? 0 : stage + 1;
    }
    // r' again, and xhat
    uint32_t kept = 0xffu;
    float gate[kE], wp[kE];
    float post_scale = 1.f;
    if (a.h) {
      if (a.post) {
        const float pm = a.stats[(size_t)3 * a.rows + row], pr = a.stats[(size_t)4 * a.rows + row];
        post_scale = a.stats[(size_t)5 * a.rows + row];
#pragma unroll
        for (int e = 0; e < kE; ++e) q[e] = col.at(e) < d ? ((q[e] - pm) - pr) * post_scale : 0.f;
      }
      load_vector8<VEC>(a.wp, a.tw, a.wide_w, 0, col, d, 1.f, wp);
      load_vector8<VEC>(a.gate, a.tc, a.wide_c, (size_t)group * a.ldgate, col, d, 1.f, gate);
      if (a.drop.threshold) kept = kept_columns(a.drop, dstep, row, col, lane);
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        v[e] = add_branch(v[e], a.alpha * gate[e], a.post ? q[e] * wp[e] : q[e], kept, e, a.drop);
      }
    }
    const float m = a.stats[row], rest = a.stats[(size_t)a.rows + row], s = a.stats[(size_t)2 * a.rows + row];
#pragma unroll
    for (int e = 0; e < kE; ++e) v[e] = col.at(e) < d ? ((v[e] - m) - rest) * s : 0.f;
    // A and B, and dn (1 + scale) w
    float own_a[kE];                                            // rows that are groups: A of this row
    {
      float sc[kE];
      load_vector8<VEC>(a.scale, a.tc, a.wide_c, (size_t)group * a.ldscale, col, d, 0.f, sc);
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        const float f = 1.0f + sc[e];
        const float k = a.mode == kSumWeighted ? f : 1.0f;
        own_a[e] = dx[e] * v[e];
        sa[e] = fmaf(k, own_a[e], sa[e]);
        sb[e] = fmaf(k, dx[e], sb[e]);
      }
      if (a.mode == kSumWeighted && a.per == 1) {
        if (a.dshift) store_vector8<VEC>(a.dshift, a.tc, a.wide_c, (size_t)row * a.lddshift, col, d, dx);
        if (a.dscale) {
          float w[kE], b[kE];
          load_vector8<VEC>(a.w, a.tw, a.wide_w, 0, col, d, 1.f, w);
          load_vector8<VEC>(a.b, a.tw, a.wide_w, 0, col, d, 0.f, b);
#pragma unroll
          for (int e = 0; e < kE; ++e) own_a[e] = fmaf(w[e], own_a[e], b[e] * dx[e]);
          store_vector8<VEC>(a.dscale, a.tc, a.wide_c, (size_t)row * a.lddscale, col, d, own_a);
        }
      }
#pragma unroll
      for (int e = 0; e < kE; ++e) dx[e] *= 1.0f + sc[e];
      if (a.w) {
        float w[kE];
        load_vector8<VEC>(a.w, a.tw, a.wide_w, 0, col, d, 1.f, w);
#pragma unroll
        for (int e = 0; e < kE; ++e) dx[e] *= w[e];
      }
    }
    float c[2] = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      c[0] += dx[e];
      c[1] = fmaf(dx[e], v[e], c[1]);
    }
    sums(c);
    const float c1 = a.rms ? 0.f : c[0] * inv_d, c2 = c[1] * inv_d;
#pragma unroll
    for (int e = 0; e < kE; ++e) g[e] = fmaf(s, dx[e] - c1 - v[e] * c2, g[e]);
    if (a.dr_in) store_row<TR, VEC>(static_cast<TR*>(a.dr_in) + (size_t)row * a.lddr_in, col, d, g);
    if (a.h) {
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        if (a.drop.threshold) g[e] = (kept >> e) & 1u ? g[e] * a.drop.scale : 0.f;
        const float k = a.alpha * gate[e];
        const float own = g[e] * q[e];                          // C of this row
        sc_[e] = fmaf(a.mode == kSumWeighted ? k : 1.0f, own, sc_[e]);
        v[e] = a.alpha * (a.post ? wp[e] : 1.f) * own;          // the row's dgate
        g[e] *= k;                                              // dq
      }
      if (a.mode == kSumWeighted && a.per == 1 && a.dgate)
        store_vector8<VEC>(a.dgate, a.tc, a.wide_c, (size_t)row * a.lddgate, col, d, v);
      if (a.dh) {
        if (a.post) {
          float e2[2] = {0.f, 0.f};
#pragma unroll
          for (int e = 0; e < kE; ++e) {
            g[e] = col.at(e) < d ? g[e] * wp[e] : 0.f;
            e2[0] += g[e];
            e2[1] = fmaf(g[e], q[e], e2[1]);
          }
          sums(e2);
          const float p1 = a.rms ? 0.f : e2[0] * inv_d, p2 = e2[1] * inv_d;
#pragma unroll
          for (int e = 0; e < kE; ++e) g[e] = post_scale * (g[e] - p1 - q[e] * p2);
        }
        store_row<TH, VEC>(static_cast<TH*>(a.dh) + (size_t)row * a.lddh, col, d, g);
      }
    }
    const bool piece_ends = row + 1 == at.end;
    const int piece = at.piece;
    at.next(a);
    if (a.mode == kSumGroups && piece_ends) {
      float sc[kE];
      load_vector8<VEC>(a.scale, a.tc, a.wide_c, (size_t)group * a.ldscale, col, d, 0.f, sc);
      if (!a.h || !a.gate)
#pragma unroll
        for (int e = 0; e < kE; ++e) gate[e] = 1.f;
      float* total = a.part + (size_t)worker * 3 * d;
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        const int cc = col.at(e);
        if (cc >= d) continue;
        const float wa = (1.0f + sc[e]) * sa[e], wb = (1.0f + sc[e]) * sb[e], wc = a.alpha * gate[e] * sc_[e];
        total[cc] = first_flush ? wa : total[cc] + wa;
        total[d + cc] = first_flush ? wb : total[d + cc] + wb;
        total[2 * d + cc] = first_flush ? wc : total[2 * d + cc] + wc;
        if (a.pieces == 1) {
          const float w = a.w ? load_any(a.w, a.tw, cc) : 1.f, b = a.b ? load_any(a.b, a.tw, cc) : 0.f;
          if (a.dshift) store_any(a.dshift, a.tc, (size_t)group * a.lddshift + cc, sb[e]);
          if (a.dscale) store_any(a.dscale, a.tc, (size_t)group * a.lddscale + cc, fmaf(w, sa[e], b * sb[e]));
          if (a.dgate) store_any(a.dgate, a.tc, (size_t)group * a.lddgate + cc, a.alpha * (a.post && a.wp ? load_any(a.wp, a.tw, cc) : 1.f) * sc_[e]);
        } else {
          float* mine = a.piece_part + (size_t)piece * 3 * d;
          mine[cc] = sa[e];
          mine[d + cc] = sb[e];
          mine[2 * d + cc] = sc_[e];
        }
        sa[e] = sb[e] = sc_[e] = 0.f;
      }
      first_flush = false;
    }
  }
  if (a.mode != kSumGroups) {
    float* total = a.part + (size_t)worker * 3 * d;
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const int cc = col.at(e);
      if (cc >= d) continue;
      total[cc] = sa[e];
      total[d + cc] = sb[e];
      total[2 * d + cc] = sc_[e];
    }
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

template <class TR, class TH, int TPR, int CL, bool VEC>
cudaError_t residual_fwd_k(const ResidualNormArgs& a, cudaStream_t st) {
  using S = ResidualShape<TPR, CL>;
  static std::atomic<int> cache[kRowDevices];
  int resident = 0;
  const cudaError_t e = row_resident(k_residual_norm<TR, TH, TPR, CL, VEC>, cache, S::kCta, 0, CL, &resident);
  if (e != cudaSuccess) return e;
  const int grid = std::min((a.rows + S::kRows - 1) / S::kRows, resident);
  return row_launch(k_residual_norm<TR, TH, TPR, CL, VEC>, dim3((unsigned)(grid * CL)), S::kCta, 0, CL, st, a);
}

template <class TR, class TH, int TPR, int CL, bool VEC>
cudaError_t residual_bwd_k(const ResidualNormArgs& a, cudaStream_t st) {
  using S = ResidualShape<TPR, CL>;
  constexpr int smem = VEC ? ResidualRing<TR, TH>::kStages * ResidualRing<TR, TH>::kPieces * S::kCta * 16 : 0;
  static std::atomic<int> cache[kRowDevices];
  int resident = 0;
  const cudaError_t e = row_resident(k_residual_norm_bwd<TR, TH, TPR, CL, VEC>, cache, S::kCta, smem, CL, &resident);
  if (e != cudaSuccess) return e;
  const int grid = (a.workers + S::kRows - 1) / S::kRows;       // (workers beyond the resident ones run after them)
  return row_launch(k_residual_norm_bwd<TR, TH, TPR, CL, VEC>, dim3((unsigned)(grid * CL)), S::kCta, smem, CL, st, a);
}

inline bool pieces16(const void* p, int64_t ld, int type) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * (type == SDS_F32 ? 4 : 2) % 16 == 0;
}

template <class TR, class TH, int TPR, int CL>
cudaError_t residual_t(const ResidualNormArgs& a, bool vec, bool backward, cudaStream_t st) {
  if (backward) return vec ? residual_bwd_k<TR, TH, TPR, CL, true>(a, st) : residual_bwd_k<TR, TH, TPR, CL, false>(a, st);
  return vec ? residual_fwd_k<TR, TH, TPR, CL, true>(a, st) : residual_fwd_k<TR, TH, TPR, CL, false>(a, st);
}

// eight columns per thread: a warp up to 256 columns, one CTA up to 4096, a cluster of two or four beyond
template <class TR, class TH>
cudaError_t residual_launch(const ResidualNormArgs& a, bool vec, bool backward, cudaStream_t st) {
  if (a.d <= 256) return residual_t<TR, TH, 32, 1>(a, vec, backward, st);
  if (a.d <= 512) return residual_t<TR, TH, 64, 1>(a, vec, backward, st);
  if (a.d <= 1024) return residual_t<TR, TH, 128, 1>(a, vec, backward, st);
  if (a.d <= 2048) return residual_t<TR, TH, 256, 1>(a, vec, backward, st);
  if (a.d <= 4096) return residual_t<TR, TH, 512, 1>(a, vec, backward, st);
  if (a.d <= 8192) return residual_t<TR, TH, 1024, 2>(a, vec, backward, st);
  return residual_t<TR, TH, 2048, 4>(a, vec, backward, st);
}

}  // namespace

// one source for each pair of types
cudaError_t residual_f32(const ResidualNormArgs& a, bool vec, bool backward, cudaStream_t st);
cudaError_t residual_f32_bf16(const ResidualNormArgs& a, bool vec, bool backward, cudaStream_t st);
cudaError_t residual_f32_f16(const ResidualNormArgs& a, bool vec, bool backward, cudaStream_t st);
cudaError_t residual_bf16(const ResidualNormArgs& a, bool vec, bool backward, cudaStream_t st);
cudaError_t residual_f16(const ResidualNormArgs& a, bool vec, bool backward, cudaStream_t st);

}  // namespace sds
