// Products on the tensor cores with fused epilogues, in two forms (kernels, and their launches):
//   - k_ffn_tile: persistent CTA pairs on 256 x 256 tiles (single CTAs on 128 x 128 tiles where there are few), for
//     batches. Operands arrive by TMA in either order (K contiguous, or M / N contiguous for the transposed
//     operands of the gradients: the matrix descriptors and the instruction descriptor say which, nothing is
//     transposed in memory). Two accumulators: the epilogue of a tile runs under the next tile's products.
//   - k_ffn_split: few rows. The time is that of reading the weights once, so the weights are the 128 rows of the
//     instruction and the tokens its 16 to 128 columns; K is split over a cluster of CTAs so that all SMs
//     read, and the partial sums are added through distributed shared memory in the order of K.
// Sums are held in 32 bits (tensor memory) throughout. Each source that includes this has kernels of its own, and its own word
// for waits that gave up.
#pragma once

#include <atomic>
#include <algorithm>

#include <cuda_fp16.h>

#include "../../include/sds.h"
#include "sds_device.cuh"
#include "sds_layers.h"
#include "sds_tc.h"
#include "sds_umma.cuh"

namespace sds {

namespace {

enum FfnEpi : int {
  kFfnGlu = 0,     // accumulator holds G | U: h and the kept factors
  kFfnOut = 1,     // out (16 bit) = acc
  kFfnAdd = 2,     // out (float) += acc
  kFfnDGlu = 3,    // accumulator holds dH: dG, dU
  kLinear = 4,     // out (16 bit or float) = act(acc + bias + table[step]) + residual, and the kept factor act'
  kLinearNarrow = 5,  // the same where output, residual or table do not lie in whole 16-byte pieces
};
__host__ __device__ constexpr bool is_linear(int epi) { return epi == kLinear || epi == kLinearNarrow; }

constexpr int kBM = 128;                          // rows of one CTA's accumulator
constexpr int kBK = 64;                           // elements of K per stage: one 128-byte swizzle row
constexpr int kChunkBytes = 64 * kBK * 2;         // 64 x 64 elements
// Epilogue warps: one per quarter of the lanes. The main loop takes up shared memory (operand tiles written and read:
// 128 bytes per cycle), and every warp that stages and polls beside it costs; four finish a tile well within the next
// one's products. Measured at 16384 rows, d = 2048, f = 8192 in a long run: forward projections 806 us with 4 warps, 896
// with 8; dH 550 and 566; second product 430 and 447. Since the feeding lanes are elected (elect_one), 16384 rows forward 1197 and 1209 us,
// 8192 rows forward and backward 2152 and 2172; short sums gain by 8 (16384 x 512 x 2048 forward 101 and 96).
constexpr int kEpiWarps = 4;
constexpr int tile_threads(int epilogue_warps) { return 64 + 32 * epilogue_warps; }   // warp 0: TMA, warp 1: MMA and tensor memory
constexpr int kWarpStage = 2048;                  // staging bytes of an epilogue warp: 32 rows of 64 bytes

// one product C[M, N] = sum over segments A_s B_s, with every operand K-major ([M or N, K]) or MN-major ([K, M or N])
struct FfnProduct {
  CUtensorMap a[2], b[2];                         // kFfnGlu: b[0] = Wg, b[1] = Wu, one segment
  int M, N, K;                                    // K of one segment
  int nseg, a_mn;
  int band;                                       // tile rows of a band (see tile_at)
  int parts;                                      // > 1: K is cut into so many, a tile is one part of one output tile, and
  float* part;                                    // its sums go here (part_index) for k_ffn_join
  void* out;
  int64_t ldo;
};

// kLinear: what its epilogue adds to a product, and where act' goes
struct LinearEpilogue {
  const void* bias;                               // [N] of tbias, NULL = none
  const uint16_t* table;                          // [steps, N] of the operands' type, NULL = none
  const int* step;                                // [M] row of the table; a row whose step is outside the table is NaN
  const void* residual;                           // [M, N] of the output's type, NULL = none
  float* factor;                                  // [M, ldf], ldf = N rounded up to 8, NULL = not kept
  int64_t ldr, ldf;
  int tbias, ty, steps;                           // ty: output and residual, SDS_F32 or (else) the operands' type
};

constexpr int kMaxProducts = 4;
struct FfnTileArgs {
  FfnProduct p[kMaxProducts];
  int np;
  int na, give;                                   // order of the tiles (see tile_index)
  int f16, act;
  const int* nrows_dev;                           // row count of p[0] on the device (NULL: p[0].M)
  float* keep;
  void* out2;                                     // kFfnDGlu: dU (out is dG)
  int* err;
  int clear_err;                                  // (see FfnSplitArgs)
  int beside;                                     // reads nothing of the kernel in front: runs beside it, and waits for
                                                  // it only in the end
  LinearEpilogue lin;                             // kLinear
};

// ---------------------------------------------------------------------------------------------
// the epilogues' arithmetic
// ---------------------------------------------------------------------------------------------

// a = act(g), da = act'(g). The fast exponential and division are accurate to a few units of the 24-bit significand per unit of the
// exponent: far inside the rounding of a 16-bit result; a float one is within 2^-18 of itself up to |g| = 30.
// GELU: with z = |g| / sqrt(2), Phi(-|g|) = erfcx(z) exp(-z^2) / 2, and the exponential is that of the density. The scaled
// function is smooth in t = 1 / (1 + 0.33 z): t times a polynomial of degree 7, fitted (least squares, reweighted towards the
// smallest largest relative error) to 8.2e-8 for z up to 9.6. In floats Phi(-|g|) is off by at most 6e-7 of
// itself up to |g| = 3 and 1.3e-6 up to 6. (With erfcf and a second exponential the epilogue took longer than the
// products up to d = 2048: 16384 x 512 x 2048 forward 182 us.)
template <int ACT>
__device__ __forceinline__ void activation(float g, float& a, float& da) {
  if (ACT == SDS_ACT_NONE) {
    a = g;
    da = 1.0f;
  } else if (ACT == SDS_ACT_SILU) {
    const float p = __fdividef(1.0f, 1.0f + __expf(-g));
    a = g * p;
    da = p * fmaf(g, 1.0f - p, 1.0f);
  } else if (ACT == SDS_ACT_GELU) {
    const float e = __expf(-0.5f * g * g), t = __fdividef(1.0f, fmaf(fabsf(g), 0.23334524f, 1.0f));
    float q = fmaf(t, -0.067964397f, 0.23134409f);
    q = fmaf(q, t, -0.17771943f);
    q = fmaf(q, t, 0.20627075f);
    q = fmaf(q, t, 0.022505348f);
    q = fmaf(q, t, 0.10096190f);
    q = fmaf(q, t, 0.091418624f);
    q = fmaf(q, t, 0.093183056f) * t * e;                     // Phi(-|g|)
    const float p = g < 0.f ? q : 1.0f - q;
    a = g * p;
    da = fmaf(g * 0.39894228040143268f, e, p);
  } else {
    const float k2 = 1.5957691216057308f, c = 0.044715f;      // 2 sqrt(2 / pi)
    const float g2 = g * g;
    const float p = __fdividef(1.0f, 1.0f + __expf(-k2 * g * fmaf(c, g2, 1.0f)));
    const float t = p * (1.0f - p);
    a = g * p;
    da = t > 0.f ? fmaf(g * t * k2, fmaf(3.0f * c, g2, 1.0f), p) : p;   // (t = 0 where g^2 might overflow)
  }
}

template <int N> struct Act { static constexpr int value = N; };
template <bool B> struct Bool { static constexpr bool value = B; };
// f(Act<act>): the choice is made once per tile or row and not per element
template <class F>
__device__ __forceinline__ void with_activation(int act, F f) {
  if (act == SDS_ACT_SILU) f(Act<SDS_ACT_SILU>());
  else if (act == SDS_ACT_GELU) f(Act<SDS_ACT_GELU>());
  else f(Act<SDS_ACT_GELU_TANH>());
}
template <class F>
__device__ __forceinline__ void with_activation_or_none(int act, F f) {
  if (act == SDS_ACT_NONE) f(Act<SDS_ACT_NONE>());
  else with_activation(act, f);
}

__device__ __forceinline__ uint32_t pack16(float lo, float hi, int f16) {
  if (f16) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  return pack_bf16x2(lo, hi);
}

// the kept factors of 32 x 32 blocks of (row, column of f): [row block][column block][factor][column quad][row] quads
__device__ __forceinline__ size_t keep_index(int row, int col, int ncc, int which) {
  return ((((size_t)(row >> 5) * ncc + (col >> 5)) * 2 + which) * 8 + ((col & 31) >> 2)) * 128 + (size_t)(row & 31) * 4;
}

// 32 rows of 64 bytes, one per lane as 16 words, to global memory: turned through shared memory so that four lanes
// write the 64 bytes of a row. Piece p of row r lies at p ^ (r / 2 % 4): 128-bit accesses free of bank conflicts both ways.
__device__ __forceinline__ void store_rows64(uint4* stg, const uint32_t* w, char* out, size_t ld_bytes, int nrows,
                                             int npieces, int lane) {
#pragma unroll
  for (int p = 0; p < 4; ++p)
    stg[lane * 4 + (p ^ ((lane >> 1) & 3))] = make_uint4(w[4 * p], w[4 * p + 1], w[4 * p + 2], w[4 * p + 3]);
  __syncwarp();
  const int pc = lane & 3;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 8 * i + (lane >> 2);
    const uint4 v = stg[r * 4 + (pc ^ ((r >> 1) & 3))];
    if (r < nrows && pc < npieces) *reinterpret_cast<uint4*>(out + (size_t)r * ld_bytes + pc * 16) = v;
  }
  __syncwarp();
}

// the same for an accumulation in place: out (float) += the 16 floats of every row
__device__ __forceinline__ void add_rows64(uint4* stg, const uint32_t* w, float* out, size_t ld, int nrows, int npieces,
                                           int lane) {
#pragma unroll
  for (int p = 0; p < 4; ++p)
    stg[lane * 4 + (p ^ ((lane >> 1) & 3))] = make_uint4(w[4 * p], w[4 * p + 1], w[4 * p + 2], w[4 * p + 3]);
  __syncwarp();
  const int pc = lane & 3;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 8 * i + (lane >> 2);
    const uint4 v = stg[r * 4 + (pc ^ ((r >> 1) & 3))];
    if (r < nrows && pc < npieces) {
      float4* o = reinterpret_cast<float4*>(out + (size_t)r * ld + pc * 4);
      float4 c = *o;
      c.x += __uint_as_float(v.x); c.y += __uint_as_float(v.y); c.z += __uint_as_float(v.z); c.w += __uint_as_float(v.w);
      *o = c;
    }
  }
  __syncwarp();
}

__device__ __forceinline__ float unpack16(uint32_t bits, int f16) {
  return f16 ? __half2float(__ushort_as_half((unsigned short)bits)) : __uint_as_float(bits << 16);
}
__device__ __forceinline__ float2 unpack16x2(uint32_t w, int f16) {
  return f16 ? __half22float2(*reinterpret_cast<const __half2*>(&w)) : make_float2(bf16_lo(w), bf16_hi(w));
}
__device__ __forceinline__ float load_typed(const void* p, int type, size_t i) {
  return type == SDS_F32 ? static_cast<const float*>(p)[i] : unpack16(static_cast<const uint16_t*>(p)[i], type == SDS_F16);
}
__device__ __forceinline__ uint16_t round16(float v, int f16) {
  return f16 ? __half_as_ushort(__float2half_rn(v)) : (uint16_t)(pack_bf16x2(v, 0.f) & 0xffffu);
}

// kLinear. A warp's 32 rows of 64 bytes change hands through its staging area: in memory's order (four lanes to a row, or, where
// rows are not whole 16-byte pieces, an element per lane), and one row to a lane, as 16 words.
struct Rows64 { uint4 v[4]; };
__device__ __forceinline__ uint4* staged(uint4* stg, int row, int piece) { return stg + row * 4 + (piece ^ ((row >> 1) & 3)); }
__device__ __forceinline__ uint16_t* staged16(uint4* stg, int row, int c) { return reinterpret_cast<uint16_t*>(staged(stg, row, c >> 3)) + (c & 7); }
__device__ __forceinline__ uint32_t* staged32(uint4* stg, int row, int c) { return reinterpret_cast<uint32_t*>(staged(stg, row, c >> 2)) + (c & 3); }
// whole pieces: requested ahead of their use; at(i) is this lane's piece of row 8 i + lane / 4, NULL where there is none
template <class F>
__device__ __forceinline__ void fetch_rows(Rows64& r, F at) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4* p = at(i);
    r.v[i] = p ? *p : make_uint4(0u, 0u, 0u, 0u);
  }
}
__device__ __forceinline__ void take_staged(uint4* stg, uint32_t (&w)[16], int lane) {
  __syncwarp();
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const uint4 v = *staged(stg, lane, p);
    w[4 * p] = v.x; w[4 * p + 1] = v.y; w[4 * p + 2] = v.z; w[4 * p + 3] = v.w;
  }
  __syncwarp();
}
__device__ __forceinline__ void rows_to_lanes(uint4* stg, const Rows64& r, uint32_t (&w)[16], int lane) {
#pragma unroll
  for (int i = 0; i < 4; ++i) *staged(stg, 8 * i + (lane >> 2), lane & 3) = r.v[i];
  take_staged(stg, w, lane);
}
// element by element: from(row) points to the first column of a row, NULL = zeros; ncols columns are there
template <class F>
__device__ __forceinline__ void narrow16_to_lanes(uint4* stg, F from, int ncols, uint32_t (&w)[16], int lane) {
  uint16_t v[32];
#pragma unroll
  for (int r = 0; r < 32; ++r) {
    const uint16_t* p = from(r);
    v[r] = p && lane < ncols ? p[lane] : (uint16_t)0;
  }
#pragma unroll
  for (int r = 0; r < 32; ++r) *staged16(stg, r, lane) = v[r];
  take_staged(stg, w, lane);
}
template <class F>
__device__ __forceinline__ void narrow32_to_lanes(uint4* stg, F from, int ncols, uint32_t (&w)[16], int lane) {
  uint32_t v[16];
  const int c = lane & 15;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t* p = from(2 * i + (lane >> 4));
    v[i] = p && c < ncols ? p[c] : 0u;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) *staged32(stg, 2 * i + (lane >> 4), c) = v[i];
  take_staged(stg, w, lane);
}
__device__ __forceinline__ void stage_lanes(uint4* stg, const uint32_t* w, int lane) {
#pragma unroll
  for (int p = 0; p < 4; ++p) *staged(stg, lane, p) = make_uint4(w[4 * p], w[4 * p + 1], w[4 * p + 2], w[4 * p + 3]);
  __syncwarp();
}
__device__ __forceinline__ void store_narrow16(uint4* stg, const uint32_t (&w)[16], uint16_t* out, int64_t ld, int nrows, int ncols, int lane) {
  stage_lanes(stg, w, lane);
#pragma unroll
  for (int r = 0; r < 32; ++r) {
    const uint16_t v = *staged16(stg, r, lane);
    if (r < nrows && lane < ncols) out[(size_t)r * ld + lane] = v;
  }
  __syncwarp();
}
__device__ __forceinline__ void store_narrow32(uint4* stg, const uint32_t* w, uint32_t* out, int64_t ld, int nrows, int ncols, int lane) {
  stage_lanes(stg, w, lane);
  const int c = lane & 15;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int r = 2 * i + (lane >> 4);
    const uint32_t v = *staged32(stg, r, c);
    if (r < nrows && c < ncols) out[(size_t)r * ld + c] = v;
  }
  __syncwarp();
}

// (Loads of what another kernel wrote are plain ones throughout: the compiler may move read-only loads ahead of the wait for it.)
// kLinear with a float result, 16 columns of the warp's rows at a time (a lane's each): what the sums of SUMS leave of the registers
template <int EPI>
__device__ __forceinline__ void linear_floats(const LinearEpilogue& e, int act, uint4* stg, float (&z)[16], int table_row, float* out, int64_t ldo,
                                              int row0, int nrows, int col, int N, int f16, int lane) {
  constexpr bool WHOLE = EPI == kLinear;
  const int ncols = min(16, N - col);
  if (e.bias) {
    reinterpret_cast<float*>(stg)[lane & 15] = (lane & 15) < ncols ? load_typed(e.bias, e.tbias, (size_t)(col + (lane & 15))) : 0.f;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 b = reinterpret_cast<const float4*>(stg)[i];
      z[4 * i] += b.x; z[4 * i + 1] += b.y; z[4 * i + 2] += b.z; z[4 * i + 3] += b.w;
    }
    __syncwarp();
  }
  if (e.table) {
    const uint16_t* from = e.table + (size_t)max(table_row, 0) * N + col;
    const float bad = table_row < 0 ? __int_as_float(0x7fffffff) : 0.f;
    if (WHOLE) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint4 t = 8 * k < ncols ? *reinterpret_cast<const uint4*>(from + 8 * k) : make_uint4(0u, 0u, 0u, 0u);
        const uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 v = unpack16x2(w[i], f16);
          z[8 * k + 2 * i] += v.x + bad;
          z[8 * k + 2 * i + 1] += v.y + bad;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) z[i] += (i < ncols ? unpack16(from[i], f16) : 0.f) + bad;
    }
  }
  uint32_t w[16];
  with_activation_or_none(act, [&](auto a) {
    constexpr int ACT = decltype(a)::value;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float d;
      activation<ACT>(z[i], z[i], d);
      w[i] = __float_as_uint(d);
    }
  });
  if (e.factor)
    store_rows64(stg, w, reinterpret_cast<char*>(e.factor + (size_t)row0 * e.ldf + col), (size_t)e.ldf * 4, nrows, min(4, ((int)e.ldf - col) >> 2), lane);
  if (e.residual) {
    const float* res = static_cast<const float*>(e.residual) + (size_t)row0 * e.ldr + col;
    if (WHOLE) {
      Rows64 r;
      fetch_rows(r, [&](int i) -> const uint4* {
        const int row = 8 * i + (lane >> 2), c = 4 * (lane & 3);
        return row < nrows && c < ncols ? reinterpret_cast<const uint4*>(res + (size_t)row * e.ldr + c) : nullptr;
      });
      rows_to_lanes(stg, r, w, lane);
    } else {
      narrow32_to_lanes(stg, [&](int row) -> const uint32_t* {
        return row < nrows ? reinterpret_cast<const uint32_t*>(res + (size_t)row * e.ldr) : nullptr;
      }, ncols, w, lane);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] += __uint_as_float(w[i]);
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(z[i]);
  float* to = out + (size_t)row0 * ldo + col;
  if (WHOLE) store_rows64(stg, w, reinterpret_cast<char*>(to), (size_t)ldo * 4, nrows, ncols >> 2, lane);
  else store_narrow32(stg, w, reinterpret_cast<uint32_t*>(to), ldo, nrows, ncols, lane);
}

// eight columns of the warp's 32 lanes back to tensor memory; they may be loaded again behind tmem_st_wait
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]),
               "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Kernels overlap their starts: one may be started when all CTAs of the one in front have said so (or ended), and waits
// for that kernel's end, and for its writes, here. Two kinds read device memory before that wait: k_ffn_split in a call's later
// products, the weights, which nothing in the call writes; and a tile launch `beside` (FfnTileArgs), all it needs, as it reads
// nothing of the kernel in front. Both are right only because the kernel directly in front is one of the same call that said so
// after its own wait: what ran before that one had then ended. So neither a norm kernel (it says so before its wait) nor
// a launch `beside` (it waits in the end) may stand there: behind these come only first kernels of calls and k_ffn_join, which
// wait before they read anything.
__device__ __forceinline__ void launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_prior_kernel() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// One lane of a converged warp. The compiler knows of elect.sync that a single lane goes on and keeps the descriptors, addresses and
// barriers of its copies and products in the warp's uniform registers; behind `lane == 0` it did not, and a step of K took 0.33 us
// whatever the tile, where it now takes 0.14 (128 x 128) or 0.27 (256 x 256, the tensor cores' own time): 8192 x 2048 x 2048
// 56.9 -> 49.6 us, 2048 x 1024 x 4096 27.9 -> 16.8.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}

// A wait for the products of `steps` steps of K: the limit of one wait, and of another for every 2^15 steps (about 10 ms).
__device__ __forceinline__ bool wait_for_sums(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int steps) {
  for (int i = 0; i <= steps >> 15; ++i) {
    if (mbar_wait_warp(bar, parity, abort_flag)) return true;
    if (__any_sync(0xffffffffu, *abort_flag != 0)) return false;
  }
  return false;
}

// A role that gave up says so in the call's status word, and in one per device that stays until it is asked for: the status word
// lies in the workspace, which a caller may have let go by then (sds_gated_ffn_gave_up).
__device__ int gave_up_word;
__device__ __forceinline__ void give_up(int* err, int role) {
  atomicExch(err, role);
  atomicExch(&gave_up_word, role);
}

// ---------------------------------------------------------------------------------------------
// batches: persistent tiles
// ---------------------------------------------------------------------------------------------

template <int BN, bool PAIR, int EW = kEpiWarps> struct FfnTile {
  static constexpr int kTM = PAIR ? 2 * kBM : kBM;                 // rows of a tile
  static constexpr int kBRows = PAIR ? BN / 2 : BN;                // rows of B that one CTA stages
  static constexpr int kABytes = kBM * kBK * 2;
  static constexpr int kBBytes = kBRows * kBK * 2;
  static constexpr int kStageBytes = kABytes + kBBytes;
  static constexpr int kFixedBytes = 1024 /*align*/ + 256 /*barriers*/ + EW * kWarpStage;
  static constexpr int kStages = (227 * 1024 - kFixedBytes) / kStageBytes;
  static constexpr int kSmemBytes = kStages * kStageBytes + kFixedBytes;
  static constexpr int kTmemCols = 2 * BN;
  static_assert(kStages >= 3 && kStages <= 12 && kTmemCols <= 512, "stages and tensor memory");
};

struct TileAt {
  int prod, m, n, part;                           // product, tile row, tile column, part of K
};

// first step of K of part `i`
__device__ __forceinline__ int first_step(int steps, int parts, int i) { return (int)((int64_t)steps * i / parts); }

// the sums of a cut product, in 32 x 32 blocks: [row block][column block][part][column quad][row] quads, the order in which an
// epilogue's threads hold them
__device__ __forceinline__ size_t part_index(int row, int col, int ncc, int parts, int part) {
  return ((((size_t)(row >> 5) * ncc + (col >> 5)) * parts + part) * 8 + ((col & 31) >> 2)) * 128 + (size_t)(row & 31) * 4;
}

// Tiles of all products in one sequence. Within a product, bands of `band` tile rows are walked column by column: the
// band's rows of A stay in L2 while B passes by.
template <int TM, int TN, bool CUT>
__device__ __forceinline__ bool tile_at(const FfnTileArgs& g, int m0_rows, int t, TileAt* at) {
  for (int p = 0; p < g.np; ++p) {
    const int M = p == 0 ? m0_rows : g.p[p].M;
    const int mt = (M + TM - 1) / TM, nt = (g.p[p].N + TN - 1) / TN;
    const int n = mt * nt * (CUT ? g.p[p].parts : 1);
    if (t < n) {
      if (CUT) {
        at->part = t / (mt * nt);
        t -= at->part * mt * nt;
      }
      const int height = g.p[p].band, band = t / (height * nt), in = t - band * height * nt;
      const int rows = min(height, mt - band * height);
      at->prod = p;
      at->m = band * height + in % rows;
      at->n = in / rows;
      return true;
    }
    t -= n;
  }
  return false;
}

// The i-th tile of a worker. One class of tiles: dealt round robin. Two (the first `na` tiles take about `give` times as
// long as the others): the long ones round robin, then `give` short ones to every worker that got one long tile
// less, then the rest round robin. Known in advance, so no role has to ask another.
__device__ __forceinline__ int tile_index(const FfnTileArgs& g, int worker, int nworkers, int i) {
  if (g.give == 0) return worker + i * nworkers;
  const int rest = g.na % nworkers, mine = g.na / nworkers + (worker < rest ? 1 : 0);
  if (i < mine) return worker + i * nworkers;
  i -= mine;
  int t = g.na;
  if (rest > 0) {
    if (worker >= rest) {
      if (i < g.give) return t + (worker - rest) * g.give + i;
      i -= g.give;
    }
    t += (nworkers - rest) * g.give;
  }
  return t + worker + i * nworkers;
}

// MN: B is MN-major and A either (the gradients); else both are K-major. The loops of the two single threads that feed the
// tensor cores are written out per order: with the order looked up in every step they took 735 cycles per step of K where
// the products take 512 (16384 x 2048 x 8192, forward projections: 676 -> 611 us at full clocks).
// Bound by the tensor cores: 16384 x 2048 x 8192 forward 1147 to 1254 us, 1310 to 1440 TFLOP/s (power sets the clock of a long run); 8192 rows
// forward and backward 2110 to 2190 us beside the kept factors. kLinear, pairs: 16384 x 2048 x 2048 95 us, 1447 TFLOP/s, with bias, table and
// SiLU 105, GELU 110, with a float residual 124.
// CUT: products whose K is cut (FfnProduct::parts); its own kernel, as the others lose up to 5 % to the arithmetic.
// EW: epilogue warps, four, eight (two for each quarter of the lanes, half of the columns each) or sixteen.
// SUMS: the tensor cores add to their accumulator without rounding to nearest, so a long sum comes out short. Measured, of itself: terms of
// either sign lose 0.25 to 0.3 times 2^-24 an addition of 16 products (60 additions 0.9e-6 to 1.0e-6, 384 6.7e-6), terms of one sign 0.5 at 60
// (2.0e-6) and 1.0 at 384 (2.4e-5); a float's own rounding is 6e-8 at most. Where the result is a float, every kSumSteps steps of K
// have an accumulator of their own, and the epilogue's warps add these in registers (sixteen warps hold a tile's), while the next is filled:
// a result is then short by one or two millionths, however long the sum. 16384 x 8192 x 2048 with a float residual, at length: 12 steps 593 us, 15 572, 24 546, 64 522
// (before the feeding lanes were elected; now 15 steps 431 in short runs, 502 at length, against 424 in one accumulator).
constexpr int kSumSteps = 15;
template <int BN, int EPI, bool PAIR, bool MN, bool CUT, int EW, bool SUMS>
__global__ void __launch_bounds__(64 + 32 * EW, 1) k_ffn_tile(const __grid_constant__ FfnTileArgs g) {
  using C = FfnTile<BN, PAIR, EW>;
  constexpr int TM = C::kTM, TN = EPI == kFfnGlu ? BN / 2 : BN;    // output columns of a tile
  extern __shared__ uint8_t smem_raw[];
  uint8_t* stages = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(stages + C::kStages * C::kStageBytes);
  uint64_t* empty_bar = full_bar + C::kStages;
  uint64_t* tfull_bar = empty_bar + C::kStages;
  uint64_t* tempty_bar = tfull_bar + 2;
  uint32_t* tmem_base_s = reinterpret_cast<uint32_t*>(tempty_bar + 2);
  volatile int* abort_s = reinterpret_cast<volatile int*>(tmem_base_s + 1);
  uint8_t* epi_stage = reinterpret_cast<uint8_t*>(full_bar) + 256;

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
  const int worker = PAIR ? (int)(blockIdx.x >> 1) : (int)blockIdx.x;
  const int nworkers = PAIR ? (int)(gridDim.x >> 1) : (int)gridDim.x;
  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) { mbar_init(full_bar + s, 1); mbar_init(empty_bar + s, 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(tfull_bar + s, 1); mbar_init(tempty_bar + s, PAIR ? 2 * EW : EW); }
    *abort_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_base_s)),
                   "r"((uint32_t)C::kTmemCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_base_s)),
                   "r"((uint32_t)C::kTmemCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_base_s;
  if (!g.beside) wait_for_prior_kernel();         // (nothing in device memory is read or written before)
  launch_dependents();
  if (g.clear_err && blockIdx.x == 0 && threadIdx.x == 0) *g.err = 0;
  const int M0 = g.nrows_dev ? min(*g.nrows_dev, g.p[0].M) : g.p[0].M;

  TileAt at;
  if (warp == 0) {
    // ---------------- TMA producer ----------------
    if (elect_one()) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      const uint32_t leader_full0 = PAIR ? map_to_cta(smem_u32(full_bar), 0u) : 0u;
      for (int it = 0; ok && tile_at<TM, TN, CUT>(g, M0, tile_index(g, worker, nworkers, it), &at); ++it) {
        const FfnProduct& p = g.p[at.prod];
        const int m0 = at.m * TM + (int)rank * kBM;
        const int n0 = at.n * TN + (EPI == kFfnGlu ? 0 : (int)rank * C::kBRows);
        const int K = p.K, nseg = p.nseg;
        int seg_steps = 0, kb0 = 0, kb1 = 0;      // CUT: of a segment; first and behind the last of this part
        if (CUT) {
          seg_steps = (K + kBK - 1) / kBK;
          kb0 = first_step(seg_steps * nseg, p.parts, at.part);
          kb1 = first_step(seg_steps * nseg, p.parts, at.part + 1);
        }
        const auto feed = [&](auto order) {
          constexpr bool a_mn = decltype(order)::value;
          for (int seg = 0; seg < nseg && ok; ++seg) {
            const CUtensorMap* ta = &p.a[seg];
            // the tile's columns of Wg, then those of Wu: one CTA of a pair each, or one after the other
            const CUtensorMap* tb = &p.b[EPI == kFfnGlu && PAIR ? (int)rank : seg];
            const int begin = CUT ? max(kb0 - seg * seg_steps, 0) * kBK : 0;
            const int end = CUT ? min(kb1 - seg * seg_steps, seg_steps) * kBK : K;
            for (int kk = begin; kk < end; kk += kBK) {
              if (!mbar_wait(empty_bar + stage, phase ^ 1u, abort_s)) { ok = false; break; }
              uint8_t* sa = stages + stage * C::kStageBytes;
              uint8_t* sb = sa + C::kABytes;
              const uint32_t fb = PAIR ? leader_full0 + (uint32_t)stage * 8u : 0u;
              if (PAIR) {
                if (rank == 0) mbar_expect_tx(full_bar + stage, 2u * (uint32_t)C::kStageBytes);
              } else {
                mbar_expect_tx(full_bar + stage, (uint32_t)C::kStageBytes);
              }
              const auto load = [&](uint8_t* dst, const CUtensorMap* tm, int c0, int c1) {
                if (PAIR) tma_load_2d_pair(dst, tm, c0, c1, fb);
                else tma_load_2d(dst, tm, c0, c1, full_bar + stage);
              };
              if (a_mn) {
#pragma unroll
                for (int j = 0; j < kBM / 64; ++j) load(sa + j * kChunkBytes, ta, m0 + 64 * j, kk);
              } else {
                load(sa, ta, kk, m0);
              }
              if (EPI == kFfnGlu && !PAIR) {
                load(sb, tb, kk, n0);
                load(sb + C::kBBytes / 2, tb + 1, kk, n0);
              } else if (MN) {
#pragma unroll
                for (int j = 0; j < C::kBRows / 64; ++j) load(sb + j * kChunkBytes, tb, n0 + 64 * j, kk);
              } else {
                load(sb, tb, kk, n0);
              }
              if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
            }
          }
        };
        if (MN && p.a_mn) feed(Bool<MN>()); else feed(Bool<false>());
      }
      if (!ok) {
        raise_abort(abort_s, PAIR);
        give_up(g.err, 1);
      }
    }
  } else if (warp == 1) {
    // ---------------- MMA issuer ----------------
    if (rank == 0 && elect_one()) {
      int stage = 0, it = 0, use = 0;             // use: accumulators filled so far
      uint32_t phase = 0;
      bool ok = true;
      bool more = tile_at<TM, TN, CUT>(g, M0, tile_index(g, worker, nworkers, 0), &at);
      for (; ok && more; ++it) {
        const FfnProduct& p = g.p[at.prod];
        const int all = (p.K + kBK - 1) / kBK * p.nseg;
        const int nkb = CUT ? first_step(all, p.parts, at.part + 1) - first_step(all, p.parts, at.part) : all;
        const int accumulators = SUMS ? (nkb + kSumSteps - 1) / kSumSteps : 1;
        for (int part = 0; ok && part < accumulators; ++part, ++use) {
          const int buf = use & 1, kb0 = SUMS ? part * kSumSteps : 0, kb1 = SUMS ? min(nkb, kb0 + kSumSteps) : nkb;
          if (!mbar_wait(tempty_bar + buf, ((uint32_t)(use >> 1) & 1u) ^ 1u, abort_s)) { ok = false; break; }
          tc_fence_after();
          const uint32_t d_tmem = tmem_base + (uint32_t)(buf * BN);
          const auto multiply = [&](auto order) {
            constexpr bool a_mn = decltype(order)::value;
            const uint32_t idesc = make_idesc(TM, BN, g.f16 != 0, a_mn, MN);
            const uint64_t adesc0 = make_sdesc(smem_u32(stages), a_mn ? (uint32_t)kChunkBytes : 0u);
            const uint64_t bdesc0 = make_sdesc(smem_u32(stages) + C::kABytes, MN ? (uint32_t)kChunkBytes : 0u);
            constexpr uint64_t a_step = a_mn ? 128u : 2u, b_step = MN ? 128u : 2u;    // 16 elements of K, in 16 bytes
            for (int kb = kb0; kb < kb1; ++kb) {
              if (!mbar_wait(full_bar + stage, phase, abort_s)) { ok = false; break; }
              tc_fence_after();
              const uint64_t adesc = adesc0 + (uint64_t)(stage * (C::kStageBytes >> 4));
              const uint64_t bdesc = bdesc0 + (uint64_t)(stage * (C::kStageBytes >> 4));
#pragma unroll
              for (int k = 0; k < kBK / 16; ++k) {
                if (PAIR) umma_f16_pair(d_tmem, adesc + a_step * k, bdesc + b_step * k, idesc, (kb > kb0 || k) ? 1u : 0u);
                else umma_f16(d_tmem, adesc + a_step * k, bdesc + b_step * k, idesc, (kb > kb0 || k) ? 1u : 0u);
              }
              if (PAIR) umma_commit_pair(empty_bar + stage); else umma_commit(empty_bar + stage);
              if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
              // where the next tile lies takes a few divisions: worked out while this tile's products run
              if (kb == 0) more = tile_at<TM, TN, CUT>(g, M0, tile_index(g, worker, nworkers, it + 1), &at);
            }
          };
          if (MN && p.a_mn) multiply(Bool<MN>()); else multiply(Bool<false>());
          if (ok) { if (PAIR) umma_commit_pair(tfull_bar + buf); else umma_commit(tfull_bar + buf); }
        }
      }
      if (!ok) {
        raise_abort(abort_s, PAIR);
        give_up(g.err, 2);
      }
    }
  } else {
    // ---------------- epilogue: a warp reaches the 32 tensor-memory lanes of quarter warp % 4 ----------------
    const int q = warp & 3;
    constexpr int kChunks = TN / 32 / (EW / 4);   // chunks of 32 output columns of a warp
    const int first_chunk = (warp - 2) / 4 * kChunks, last_chunk = first_chunk + kChunks - 1;
    uint4* stg = reinterpret_cast<uint4*>(epi_stage + (warp - 2) * kWarpStage);
    const uint32_t drained0 = (PAIR && rank != 0) ? map_to_cta(smem_u32(tempty_bar), 0u) : 0u;
    const int f16 = g.f16;
    int it = 0, use = 0;
    bool ok = true;
    for (; ok && tile_at<TM, TN, CUT>(g, M0, tile_index(g, worker, nworkers, it), &at); ++it) {
      const FfnProduct& p = g.p[at.prod];
      const int M = at.prod == 0 ? M0 : p.M, N = p.N;
      int buf = it & 1;                           // (SUMS: the last one of the tile)
      const int row0 = at.m * TM + (int)rank * kBM + q * 32, n0 = at.n * TN;
      const int nlive = min(32, M - row0);        // (may be negative)
      const int ncc = (N + 31) >> 5;
      // the kept factors do not depend on this product: requested before its accumulator is waited for
      float4 kp[8], kq[8];
      auto keep_fetch = [&](int col) {
        const bool in = nlive > 0 && col < N;
        const float4* kp0 = reinterpret_cast<const float4*>(g.keep + (in ? keep_index(row0 + lane, col, ncc, 0) : 0));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          kp[i] = in ? kp0[i * 32] : make_float4(0.f, 0.f, 0.f, 0.f);
          kq[i] = in ? kp0[(8 + i) * 32] : make_float4(0.f, 0.f, 0.f, 0.f);
        }
      };
      if (EPI == kFfnDGlu) keep_fetch(n0);
      // neither do the bias, the rows of the table and the residual (kLinear): requested a chunk ahead
      int table_row = -1, piece_row[4] = {-1, -1, -1, -1};   // of the lane's row; of the rows of which it fetches a piece
      Rows64 tab, res[2];
      float bias_next = 0.f;
      const auto added_fetch = [&](int col) {
        const LinearEpilogue& e = g.lin;
        const int pc = lane & 3;
        if (e.bias) bias_next = col + lane < N ? load_typed(e.bias, e.tbias, (size_t)(col + lane)) : 0.f;
        if (EPI == kLinear && e.table)
          fetch_rows(tab, [&](int i) -> const uint4* {
            const bool in = piece_row[i] >= 0 && col + 8 * pc < N;
            return in ? reinterpret_cast<const uint4*>(e.table + (size_t)piece_row[i] * N + col) + pc : nullptr;
          });
        if (EPI == kLinear && e.residual) {
          const int per = e.ty == SDS_F32 ? 4 : 8;              // columns of a piece; 16 or 32 of a row of 64 bytes
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
            if (hf == 0 || per == 4)
              fetch_rows(res[hf], [&](int i) -> const uint4* {
                const int r = 8 * i + (lane >> 2), c = col + 16 * hf + per * pc;
                const char* at = static_cast<const char*>(e.residual) + ((size_t)(row0 + r) * e.ldr + c) * (16 / per);
                return r < nlive && c < N ? reinterpret_cast<const uint4*>(at) : nullptr;
              });
        }
      };
      const auto find_table_row = [&]() {
        if (!g.lin.table || lane >= nlive) return;
        const int s = g.lin.step[row0 + lane];
        table_row = s >= 0 && s < g.lin.steps ? s : -1;
      };
      if (is_linear(EPI) && !SUMS) {              // (SUMS: the registers hold sums)
        find_table_row();
        if (g.lin.table)
#pragma unroll
          for (int i = 0; i < 4; ++i) piece_row[i] = __shfl_sync(0xffffffffu, table_row, 8 * i + (lane >> 2));
        added_fetch(n0 + first_chunk * 32);
      }
      const auto hand_back = [&](int b) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (PAIR && rank != 0) mbar_arrive_cluster(drained0 + (uint32_t)b * 8u);
          else mbar_arrive(tempty_bar + b);
        }
      };
      if (SUMS) {                                 // the sum of a tile's accumulators goes back to the last one's place
        float run[SUMS ? kChunks * 32 : 1];
        const int nkb = (p.K + kBK - 1) / kBK * p.nseg;
        for (int kb = 0; kb < nkb; kb += kSumSteps, ++use) {
          if (!wait_for_sums(tfull_bar + (use & 1), (uint32_t)(use >> 1) & 1u, abort_s, kSumSteps)) { ok = false; break; }
          tc_fence_after();
          const uint32_t from = tmem_base + (uint32_t)((use & 1) * BN + first_chunk * 32) + ((uint32_t)(q * 32) << 16);
          const bool last = kb + kSumSteps >= nkb;
#pragma unroll
          for (int k = 0; k < (SUMS ? kChunks * 32 : 1); k += 8) {
            uint32_t part[8];
            tmem_ld8(from + (uint32_t)k, part);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float v = __uint_as_float(part[i]);
              run[(k + i) % (SUMS ? kChunks * 32 : 1)] = kb == 0 ? v : run[(k + i) % (SUMS ? kChunks * 32 : 1)] + v;
              part[i] = __float_as_uint(run[(k + i) % (SUMS ? kChunks * 32 : 1)]);
            }
            if (last) tmem_st8(from + (uint32_t)k, part);
          }
          if (last) {
            tmem_st_wait();
            buf = use & 1;
          } else {
            hand_back(use & 1);
          }
        }
        if (!ok) break;
      } else {
        if (!wait_for_sums(tfull_bar + buf, (uint32_t)(it >> 1) & 1u, abort_s, (p.K + kBK - 1) / kBK * p.nseg)) { ok = false; break; }
        tc_fence_after();
      }
      const uint32_t tbase = tmem_base + (uint32_t)(buf * BN) + ((uint32_t)(q * 32) << 16);
      if (SUMS) {
        find_table_row();
#pragma unroll 1
        for (int c = first_chunk * 32; c < (last_chunk + 1) * 32; c += 16) {
          float z[16];
          uint32_t part[16];
          tmem_ld8(tbase + (uint32_t)c, part);
          tmem_ld8(tbase + (uint32_t)c + 8u, part + 8);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 16; ++i) z[i] = __uint_as_float(part[i]);
          if (c == last_chunk * 32 + 16) hand_back(buf);
          if (nlive > 0 && n0 + c < N)
            linear_floats<EPI>(g.lin, g.act, stg, z, table_row, static_cast<float*>(p.out), p.ldo, row0, nlive, n0 + c, N, f16, lane);
        }
      }
#pragma unroll 1
      for (int chunk = SUMS ? last_chunk + 1 : first_chunk; chunk <= last_chunk; ++chunk) {
        const int c = chunk * 32, col = n0 + c;
        uint32_t acc[32], up[EPI == kFfnGlu ? 32 : 1];
        tmem_ld32(tbase + (uint32_t)c, acc);
        if (EPI == kFfnGlu) tmem_ld32(tbase + (uint32_t)(BN / 2 + c), reinterpret_cast<uint32_t(&)[32]>(up));
        if (chunk == last_chunk) hand_back(buf);  // accumulator read
        if (nlive <= 0 || col >= N) continue;     // (uniform over the warp)
        const int npieces = min(4, (N - col) >> 3);               // pieces of eight 16-bit columns
        if (EPI == kFfnGlu) {
          uint32_t w[16];
          float4* keep = g.keep ? reinterpret_cast<float4*>(g.keep + keep_index(row0 + lane, col, ncc, 0)) : nullptr;
          with_activation(g.act, [&](auto act) {
            constexpr int ACT = decltype(act)::value;
            if (keep) {
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                float pg[4], pu[4], hh[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                  const float uu = __uint_as_float(up[(4 * i + u) % (EPI == kFfnGlu ? 32 : 1)]);
                  float da;
                  activation<ACT>(__uint_as_float(acc[4 * i + u]), pu[u], da);
                  hh[u] = pu[u] * uu;
                  pg[u] = da * uu;
                }
                w[2 * i] = pack16(hh[0], hh[1], f16);
                w[2 * i + 1] = pack16(hh[2], hh[3], f16);
                keep[i * 32] = make_float4(pg[0], pg[1], pg[2], pg[3]);
                keep[(8 + i) * 32] = make_float4(pu[0], pu[1], pu[2], pu[3]);
              }
            } else {
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                float a0, a1, da;
                activation<ACT>(__uint_as_float(acc[2 * i]), a0, da);
                activation<ACT>(__uint_as_float(acc[2 * i + 1]), a1, da);
                w[i] = pack16(a0 * __uint_as_float(up[(2 * i) % (EPI == kFfnGlu ? 32 : 1)]),
                              a1 * __uint_as_float(up[(2 * i + 1) % (EPI == kFfnGlu ? 32 : 1)]), f16);
              }
            }
          });
          store_rows64(stg, w, static_cast<char*>(p.out) + ((size_t)row0 * p.ldo + col) * 2, (size_t)p.ldo * 2, nlive,
                       npieces, lane);
        } else if (CUT && p.parts > 1) {
          float4* to = reinterpret_cast<float4*>(p.part + part_index(row0 + lane, col, ncc, p.parts, at.part));
#pragma unroll
          for (int i = 0; i < 8; ++i)
            to[i * 32] = make_float4(__uint_as_float(acc[4 * i]), __uint_as_float(acc[4 * i + 1]),
                                     __uint_as_float(acc[4 * i + 2]), __uint_as_float(acc[4 * i + 3]));
        } else if (EPI == kFfnOut) {
          uint32_t w[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) w[i] = pack16(__uint_as_float(acc[2 * i]), __uint_as_float(acc[2 * i + 1]), f16);
          store_rows64(stg, w, static_cast<char*>(p.out) + ((size_t)row0 * p.ldo + col) * 2, (size_t)p.ldo * 2, nlive,
                       npieces, lane);
        } else if (is_linear(EPI)) {
          const LinearEpilogue& e = g.lin;
          const int ncols = min(32, N - col);
          const bool float_out = e.ty == SDS_F32;
          uint32_t w[16];
          if (e.bias) {
            reinterpret_cast<float*>(stg)[lane] = bias_next;
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float4 b = reinterpret_cast<const float4*>(stg)[i];
              acc[4 * i] = __float_as_uint(__uint_as_float(acc[4 * i]) + b.x);
              acc[4 * i + 1] = __float_as_uint(__uint_as_float(acc[4 * i + 1]) + b.y);
              acc[4 * i + 2] = __float_as_uint(__uint_as_float(acc[4 * i + 2]) + b.z);
              acc[4 * i + 3] = __float_as_uint(__uint_as_float(acc[4 * i + 3]) + b.w);
            }
            __syncwarp();
          }
          const auto add16 = [&](float bad) {     // w as 32 16-bit values, plus `bad`
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float2 t = unpack16x2(w[i], f16);
              acc[2 * i] = __float_as_uint(__uint_as_float(acc[2 * i]) + (t.x + bad));
              acc[2 * i + 1] = __float_as_uint(__uint_as_float(acc[2 * i + 1]) + (t.y + bad));
            }
          };
          if (e.table) {
            if (EPI == kLinear) {
              rows_to_lanes(stg, tab, w, lane);
            } else {
              narrow16_to_lanes(stg, [&](int r) -> const uint16_t* {
                const int s = __shfl_sync(0xffffffffu, table_row, r);
                return s >= 0 ? e.table + (size_t)s * N + col : nullptr;
              }, ncols, w, lane);
            }
            add16(table_row < 0 ? __int_as_float(0x7fffffff) : 0.f);
          }
          Rows64 res_now[2] = {res[0], res[1]};
          if (chunk < last_chunk) added_fetch(col + 32);
          if (g.act != SDS_ACT_NONE)
            with_activation(g.act, [&](auto act) {
              constexpr int ACT = decltype(act)::value;
#pragma unroll
              for (int hf = 0; hf < 2; ++hf) {
                uint32_t da[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                  float a0, d0;
                  activation<ACT>(__uint_as_float(acc[16 * hf + i]), a0, d0);
                  acc[16 * hf + i] = __float_as_uint(a0);
                  da[i] = __float_as_uint(d0);
                }
                if (e.factor && col + 16 * hf < (int)e.ldf)
                  store_rows64(stg, da, reinterpret_cast<char*>(e.factor + (size_t)row0 * e.ldf + col + 16 * hf), (size_t)e.ldf * 4, nlive,
                               min(4, ((int)e.ldf - col - 16 * hf) >> 2), lane);
              }
            });
          if (e.residual && !float_out) {
            if (EPI == kLinear) rows_to_lanes(stg, res_now[0], w, lane);
            else narrow16_to_lanes(stg, [&](int r) -> const uint16_t* {
              return r < nlive ? static_cast<const uint16_t*>(e.residual) + (size_t)(row0 + r) * e.ldr + col : nullptr;
            }, ncols, w, lane);
            add16(0.f);
          } else if (e.residual) {
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              if (EPI == kLinear) rows_to_lanes(stg, res_now[hf], w, lane);
              else narrow32_to_lanes(stg, [&](int r) -> const uint32_t* {
                return r < nlive ? static_cast<const uint32_t*>(e.residual) + (size_t)(row0 + r) * e.ldr + col + 16 * hf : nullptr;
              }, ncols - 16 * hf, w, lane);
#pragma unroll
              for (int i = 0; i < 16; ++i)
                acc[16 * hf + i] = __float_as_uint(__uint_as_float(acc[16 * hf + i]) + __uint_as_float(w[i]));
            }
          }
          if (!float_out) {
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = pack16(__uint_as_float(acc[2 * i]), __uint_as_float(acc[2 * i + 1]), f16);
            uint16_t* out = static_cast<uint16_t*>(p.out) + (size_t)row0 * p.ldo + col;
            if (EPI == kLinear) store_rows64(stg, w, reinterpret_cast<char*>(out), (size_t)p.ldo * 2, nlive, npieces, lane);
            else store_narrow16(stg, w, out, p.ldo, nlive, ncols, lane);
          } else {
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              if (16 * hf >= ncols) continue;
              uint32_t* out = static_cast<uint32_t*>(p.out) + (size_t)row0 * p.ldo + col + 16 * hf;
              if (EPI == kLinear) store_rows64(stg, acc + 16 * hf, reinterpret_cast<char*>(out), (size_t)p.ldo * 4, nlive, min(4, (ncols - 16 * hf) >> 2), lane);
              else store_narrow32(stg, acc + 16 * hf, out, p.ldo, nlive, ncols - 16 * hf, lane);
            }
          }
        } else if (EPI == kFfnAdd) {
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
            if (col + 16 * hf < N)
              add_rows64(stg, acc + 16 * hf, static_cast<float*>(p.out) + (size_t)row0 * p.ldo + col + 16 * hf,
                         (size_t)p.ldo, nlive, min(4, (N - col - 16 * hf) >> 2), lane);
        } else {
          uint32_t wgr[16], wur[16];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float a0 = __uint_as_float(acc[4 * i]), a1 = __uint_as_float(acc[4 * i + 1]);
            const float a2 = __uint_as_float(acc[4 * i + 2]), a3 = __uint_as_float(acc[4 * i + 3]);
            wgr[2 * i] = pack16(a0 * kp[i].x, a1 * kp[i].y, f16);
            wgr[2 * i + 1] = pack16(a2 * kp[i].z, a3 * kp[i].w, f16);
            wur[2 * i] = pack16(a0 * kq[i].x, a1 * kq[i].y, f16);
            wur[2 * i + 1] = pack16(a2 * kq[i].z, a3 * kq[i].w, f16);
          }
          if (chunk < last_chunk) keep_fetch(col + 32);
          const size_t off = ((size_t)row0 * p.ldo + col) * 2;
          store_rows64(stg, wgr, static_cast<char*>(p.out) + off, (size_t)p.ldo * 2, nlive, npieces, lane);
          store_rows64(stg, wur, static_cast<char*>(g.out2) + off, (size_t)p.ldo * 2, nlive, npieces, lane);
        }
      }
    }
    if (!ok && lane == 0) {
      raise_abort(abort_s, PAIR);
      give_up(g.err, 3);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_s && threadIdx.x == 0) {
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);   // copies still in flight land before the memory is released
  }
  if (g.beside) wait_for_prior_kernel();
  __syncthreads();
  if (PAIR) cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    if (PAIR)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)C::kTmemCols) : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)C::kTmemCols) : "memory");
  }
}

struct FfnJoinArgs {
  struct { const float* part; uint16_t* out; int M, N; } p[3];
  int np, parts, f16;
};

// The parts of cut products, added in the order of K. A warp takes a quad of columns of a 32 x 32 block, a lane one row of
// it. Bound by the latency of reading the parts, which lie in L2 (products are cut only where they are small).
constexpr int kJoinThreads = 256;
__global__ void __launch_bounds__(kJoinThreads) k_ffn_join(const FfnJoinArgs g) {
  const int lane = threadIdx.x & 31;
  int64_t b = ((int64_t)blockIdx.x * kJoinThreads + threadIdx.x) >> 5;
  wait_for_prior_kernel();
  launch_dependents();
  for (int p = 0; p < g.np; ++p) {
    const int M = g.p[p].M, N = g.p[p].N, ncc = (N + 31) >> 5;
    const int64_t n = (int64_t)((M + 31) >> 5) * ncc * 8;
    if (b < n) {
      const int block = (int)(b >> 3), row = block / ncc * 32 + lane, col = block % ncc * 32 + (int)(b & 7) * 4;
      if (row >= M || col >= N) return;
      const float4* from = reinterpret_cast<const float4*>(g.p[p].part + part_index(row, col, ncc, g.parts, 0));
      float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
      for (int i = 0; i < g.parts; ++i) {
        const float4 v = from[(size_t)i * 256];
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
      }
      *reinterpret_cast<uint2*>(g.p[p].out + (size_t)row * N + col) = make_uint2(pack16(s.x, s.y, g.f16), pack16(s.z, s.w, g.f16));
      return;
    }
    b -= n;
  }
}

// ---------------------------------------------------------------------------------------------
// few rows: weights as the 128 rows of the instruction, K split over a cluster
// ---------------------------------------------------------------------------------------------

struct FfnSplitArgs {
  CUtensorMap w[2], t[2];                         // weights and tokens per segment (kFfnGlu: w = Wg, Wu, one t)
  int rows, N, K;                                 // tokens, output columns, K of one segment
  int nseg, w_mn;                                 // w_mn: weights lie [K, N]
  int f16, act;
  float* keep;
  void* out;
  void* out2;
  int64_t ldo;
  int* err;
  int clear_err;                                  // first kernel of a call: the status word starts at zero. A wait gives
                                                  // up only after millions of polls, long after the first CTA began.
  LinearEpilogue lin;                             // kLinear
};

constexpr int kSplitThreads = 256;

// kLinear with a float result: a CTA's steps of K are dealt to up to so many accumulators (see SUMS), added in order behind them: as many
// as fit half of the tensor memory (two CTAs share an SM). None takes more than kFewRowSteps: no form is chosen that would ask for more.
__host__ __device__ constexpr int split_accumulators(int bn, int epi) { return is_linear(epi) ? 256 / bn : 1; }
constexpr int kFewRowSteps = 16;
template <int BN, int EPI> struct FfnSplit {
  static constexpr int kABytes = kBM * kBK * 2, kBBytes = BN * kBK * 2, kStageBytes = kABytes + kBBytes;
  static constexpr int kFixedBytes = 1024 + 256;
  // half of an SM's shared memory, so that two CTAs share an SM: clusters of eight are then all resident at once, and
  // the CTAs of the next product request their weights while the last ones of this product finish
  static constexpr int kStages = (113 * 1024 - kFixedBytes) / kStageBytes;
  static constexpr int kSmemBytes = kStages * kStageBytes + kFixedBytes;
  static constexpr int kAccumulators = split_accumulators(BN, EPI);
  static constexpr int kTmemCols = BN * kAccumulators < 32 ? 32 : BN * kAccumulators;
  static_assert(kStages * kStageBytes >= BN * kBM * 4, "the partial sums fit where the stages were");
};

__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}

// 2048 x 8192 bf16, both products: 1 row 24.1 us (4.2 TB/s of weights), 64 rows 30; 8 rows of 4096 x 14336 60.6 us
// (5.8 TB/s, 89 % of a copy's rate). kLinear: 1 row of 2048 x 2048 5.0 us in a graph, of 8192 x 2048 7.9. What is left of a small call is the ramp of the requests and the exchange, once per product.
template <int BN, int EPI>
__global__ void __launch_bounds__(kSplitThreads, 2) k_ffn_split(const __grid_constant__ FfnSplitArgs g) {
  using C = FfnSplit<BN, EPI>;
  constexpr int TN = EPI == kFfnGlu ? 64 : 128;   // output columns of a CTA
  extern __shared__ uint8_t smem_raw[];
  uint8_t* stages = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(stages + C::kStages * C::kStageBytes);
  uint64_t* empty_bar = full_bar + C::kStages;
  uint64_t* tfull_bar = empty_bar + C::kStages;
  uint32_t* tmem_base_s = reinterpret_cast<uint32_t*>(tfull_bar + 1);
  volatile int* abort_s = reinterpret_cast<volatile int*>(tmem_base_s + 1);
  float* part = reinterpret_cast<float*>(stages); // [BN][128], once the products are done

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  uint32_t nsplit;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(nsplit));
  const uint32_t rank = cluster_ctarank();
  const int n0 = (int)(blockIdx.x / nsplit) * TN, tok0 = (int)blockIdx.y * BN;
  const int kb_seg = (g.K + kBK - 1) / kBK, nkb = kb_seg * g.nseg;
  const int kb0 = (int)((int64_t)nkb * rank / nsplit), kb1 = (int)((int64_t)nkb * (rank + 1) / nsplit);
  // steps of an accumulator (of a float result: kSumSteps where there are accumulators enough, never more than kFewRowSteps)
  const int per = C::kAccumulators == 1 || g.lin.ty != SDS_F32
                      ? kb1 - kb0 : max(kSumSteps, (kb1 - kb0 + C::kAccumulators - 1) / C::kAccumulators);

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) { mbar_init(full_bar + s, 1); mbar_init(empty_bar + s, 1); }
    mbar_init(tfull_bar, 1);
    *abort_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_base_s)),
                 "r"((uint32_t)C::kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_base_s;

  if (warp == 0 && elect_one()) {
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    auto weights = [&](int kb) {
      uint8_t* sa = stages + stage * C::kStageBytes;
      const int seg = kb >= kb_seg ? 1 : 0, kk = (kb - seg * kb_seg) * kBK;
      mbar_expect_tx(full_bar + stage, (uint32_t)C::kStageBytes);
      if (EPI == kFfnGlu) {                       // rows 0..63 of the instruction: Wg, rows 64..127: Wu
        tma_load_2d(sa, &g.w[0], kk, n0, full_bar + stage);
        tma_load_2d(sa + C::kABytes / 2, &g.w[1], kk, n0, full_bar + stage);
      } else if (g.w_mn) {
        tma_load_2d(sa, &g.w[seg], n0, kk, full_bar + stage);
        tma_load_2d(sa + kChunkBytes, &g.w[seg], n0 + 64, kk, full_bar + stage);
      } else {
        tma_load_2d(sa, &g.w[seg], kk, n0, full_bar + stage);
      }
    };
    auto tokens = [&](int kb) {
      const int seg = kb >= kb_seg ? 1 : 0, kk = (kb - seg * kb_seg) * kBK;
      tma_load_2d(stages + stage * C::kStageBytes + C::kABytes, &g.t[seg], kk, tok0, full_bar + stage);
    };
    // Behind a kernel of the same call, which waited before it let this one start and writes the tokens, not the weights: the
    // first stages' weights are requested before it has ended. A call's first kernel may have anything in front and waits.
    const int ahead = min(kb1 - kb0, C::kStages);
    if (g.clear_err) wait_for_prior_kernel();
    for (int i = 0; i < ahead; ++i) { weights(kb0 + i); ++stage; }
    wait_for_prior_kernel();
    for (stage = 0; stage < ahead; ++stage) tokens(kb0 + stage);
    stage = 0;
    phase = 1;
    for (int kb = kb0 + ahead; kb < kb1; ++kb) {
      if (!mbar_wait(empty_bar + stage, phase ^ 1u, abort_s)) { ok = false; break; }
      weights(kb);
      tokens(kb);
      if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
    }
    if (!ok) {
      *abort_s = 1;
      give_up(g.err, 1);
    }
  } else if (warp == 1 && elect_one()) {
    const uint32_t idesc = make_idesc(kBM, BN, g.f16 != 0, g.w_mn != 0, false);
    const uint32_t a_chunk = g.w_mn ? (uint32_t)kChunkBytes : 0u;
    const uint64_t a_step = g.w_mn ? 128u : 2u;
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    wait_for_prior_kernel();                      // (however long that one runs: the polls below count from here)
    for (int kb = kb0; kb < kb1; ++kb) {
      if (!mbar_wait(full_bar + stage, phase, abort_s)) { ok = false; break; }
      tc_fence_after();
      const uint32_t sa = smem_u32(stages + stage * C::kStageBytes);
      const uint64_t adesc = make_sdesc(sa, a_chunk), bdesc = make_sdesc(sa + C::kABytes);
      const int at = C::kAccumulators == 1 ? 0 : (kb - kb0) / per;
      const bool begun = C::kAccumulators == 1 ? kb > kb0 : kb - kb0 > at * per;
#pragma unroll
      for (int k = 0; k < kBK / 16; ++k)
        umma_f16(tmem_base + (uint32_t)(at * BN), adesc + a_step * k, bdesc + (uint64_t)(2 * k), idesc, (begun || k) ? 1u : 0u);
      umma_commit(empty_bar + stage);
      if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
    }
    if (ok) {
      umma_commit(tfull_bar);
    } else {
      *abort_s = 1;
      give_up(g.err, 2);
    }
  }
  __syncwarp();

  wait_for_prior_kernel();                        // (nothing else in device memory is read or written before)
  launch_dependents();
  if (g.clear_err && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *g.err = 0;
  // kLinear: what is added to this lane's four columns of a token, requested before the sums are waited for, then a token ahead; a
  // lane holds the table's row of its own one of the warp's tokens
  const int share = BN / (int)nsplit, first = tok0 + (int)rank * share + warp, lin_col = n0 + 4 * lane, live = min(4, g.N - lin_col);
  float lin_bias[4] = {0.f, 0.f, 0.f, 0.f};
  uint32_t lin_table[4] = {0u, 0u, 0u, 0u}, lin_residual[4] = {0u, 0u, 0u, 0u};
  int lin_rows = -1, lin_row = -1;
  const auto request_four = [&](uint32_t (&w)[4], const void* p, bool floats, size_t i) {
    if (EPI == kLinear) {
      if (floats) {
        const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const float*>(p) + i);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
      } else {
        const uint2 v = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + i);
        w[0] = v.x; w[1] = v.y;
      }
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (u < live) w[u] = floats ? static_cast<const uint32_t*>(p)[i + u] : static_cast<const uint16_t*>(p)[i + u];
    }
  };
  const auto four = [&](const uint32_t (&w)[4], bool floats, float (&v)[4]) {
    if (floats) {
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = __uint_as_float(w[u]);
    } else if (EPI == kLinear) {
      const float2 lo = unpack16x2(w[0], g.f16), hi = unpack16x2(w[1], g.f16);
      v[0] = lo.x; v[1] = lo.y; v[2] = hi.x; v[3] = hi.y;
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = unpack16(w[u], g.f16);
    }
  };
  const auto request_added = [&](int k) {         // for the warp's k-th token
    if (g.lin.table) {
      lin_row = __shfl_sync(0xffffffffu, lin_rows, k);
      if (lin_row >= 0 && live > 0) request_four(lin_table, g.lin.table, false, (size_t)lin_row * g.N + lin_col);
    }
    const int tok = first + k * (kSplitThreads / 32);
    if (g.lin.residual && tok < g.rows && live > 0)
      request_four(lin_residual, g.lin.residual, g.lin.ty == SDS_F32, (size_t)tok * g.lin.ldr + lin_col);
  };
  if (is_linear(EPI)) {
    if (g.lin.bias)
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (u < live) lin_bias[u] = load_typed(g.lin.bias, g.lin.tbias, (size_t)(lin_col + u));
    if (g.lin.table) {
      const int i = lane * (kSplitThreads / 32), tok = first + i;
      if (warp + i < share && tok < g.rows) {
        const int at = g.lin.step[tok];
        lin_rows = at >= 0 && at < g.lin.steps ? at : -1;
      }
    }
    request_added(0);
  }
  // the accumulator to shared memory, [token][row of the instruction]
  const bool ok = wait_for_sums(tfull_bar, 0u, abort_s, kb1 - kb0);
  if (ok) {
    tc_fence_after();
    const int q = warp & 3, half = warp >> 2;
    uint32_t acc[BN / 2];
#pragma unroll
    for (int c = 0; c < BN / 2; c += 8)
      tmem_ld8(tmem_base + (uint32_t)(half * (BN / 2) + c) + ((uint32_t)(q * 32) << 16), acc + c);
    tmem_ld_wait();
    if (C::kAccumulators > 1)
      for (int b = 1; b * per < kb1 - kb0; ++b) {
#pragma unroll
        for (int c = 0; c < BN / 2; c += 8) {
          uint32_t more[8];
          tmem_ld8(tmem_base + (uint32_t)(b * BN + half * (BN / 2) + c) + ((uint32_t)(q * 32) << 16), more);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[c + i] = __float_as_uint(__uint_as_float(acc[c + i]) + __uint_as_float(more[i]));
        }
      }
#pragma unroll
    for (int c = 0; c < BN / 2; ++c) part[(half * (BN / 2) + c) * kBM + q * 32 + lane] = __uint_as_float(acc[c]);
  } else if (lane == 0) {
    *abort_s = 1;
    give_up(g.err, 3);
  }
  tc_fence_before();
  if (nsplit > 1) cluster_sync_all(); else __syncthreads();

  // this CTA's share of the tokens: partial sums added in the order of K, then the epilogue; a lane holds four columns
  const uint32_t part_a = smem_u32(part);
  const int ncc = (g.N + 31) >> 5;
  float4 sums[8];                                 // of a token, one for each CTA; requested a token ahead
  const auto request_sums = [&](int i) {
    const uint32_t off = (uint32_t)(((int)rank * share + i) * kBM + lane * 4) * 4u;
#pragma unroll
    for (uint32_t r = 0; r < 8; ++r)
      if (r < nsplit) sums[r] = ld_cluster4(map_to_cta(part_a + off, r));
  };
  if (warp < share) request_sums(warp);
  for (int i = warp; i < share; i += kSplitThreads / 32) {
    const int tok = first + i - warp;
    if (tok >= g.rows) break;
    float4 s = sums[0];
    if (nsplit > 1) {
      s.x += 0.f; s.y += 0.f; s.z += 0.f; s.w += 0.f;
#pragma unroll
      for (uint32_t r = 1; r < 8; ++r)
        if (r < nsplit) { s.x += sums[r].x; s.y += sums[r].y; s.z += sums[r].z; s.w += sums[r].w; }
    }
    const bool more = i + kSplitThreads / 32 < share;
    if (more) request_sums(i + kSplitThreads / 32);
    if (EPI == kFfnGlu) {
      float4 u;
      u.x = __shfl_down_sync(0xffffffffu, s.x, 16); u.y = __shfl_down_sync(0xffffffffu, s.y, 16);
      u.z = __shfl_down_sync(0xffffffffu, s.z, 16); u.w = __shfl_down_sync(0xffffffffu, s.w, 16);
      const int col = n0 + 4 * lane;
      if (lane < 16 && col < g.N) {
        float4 a, da;
        with_activation(g.act, [&](auto act) {
          constexpr int ACT = decltype(act)::value;
          activation<ACT>(s.x, a.x, da.x); activation<ACT>(s.y, a.y, da.y);
          activation<ACT>(s.z, a.z, da.z); activation<ACT>(s.w, a.w, da.w);
        });
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(g.out) + (size_t)tok * g.ldo + col) =
            make_uint2(pack16(a.x * u.x, a.y * u.y, g.f16), pack16(a.z * u.z, a.w * u.w, g.f16));
        if (g.keep) {
          *reinterpret_cast<float4*>(g.keep + keep_index(tok, col, ncc, 0)) = make_float4(da.x * u.x, da.y * u.y, da.z * u.z, da.w * u.w);
          *reinterpret_cast<float4*>(g.keep + keep_index(tok, col, ncc, 1)) = a;
        }
      }
    } else if (is_linear(EPI)) {
      const LinearEpilogue& e = g.lin;
      const int col = lin_col;
      float t[4], added[4];
      four(lin_table, false, t);
      four(lin_residual, e.ty == SDS_F32, added);
      const bool known = lin_row >= 0;
      if (more) request_added((i - warp) / (kSplitThreads / 32) + 1);
      if (live > 0) {
        float z[4] = {s.x + lin_bias[0], s.y + lin_bias[1], s.z + lin_bias[2], s.w + lin_bias[3]}, da[4];
        if (e.table) {
#pragma unroll
          for (int u = 0; u < 4; ++u) z[u] += known ? t[u] : __int_as_float(0x7fffffff);
        }
        with_activation_or_none(g.act, [&](auto act) {
          constexpr int ACT = decltype(act)::value;
#pragma unroll
          for (int u = 0; u < 4; ++u) activation<ACT>(z[u], z[u], da[u]);
        });
        if (e.factor)                             // (its rows are padded to eight columns)
          *reinterpret_cast<float4*>(e.factor + (size_t)tok * e.ldf + col) = make_float4(da[0], da[1], da[2], da[3]);
        const size_t to = (size_t)tok * g.ldo + col;
        if (e.residual)
#pragma unroll
          for (int u = 0; u < 4; ++u) z[u] += added[u];
        if (EPI == kLinear && e.ty == SDS_F32) {
          *reinterpret_cast<float4*>(static_cast<float*>(g.out) + to) = make_float4(z[0], z[1], z[2], z[3]);
        } else if (EPI == kLinear) {
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(g.out) + to) = make_uint2(pack16(z[0], z[1], g.f16), pack16(z[2], z[3], g.f16));
        } else {
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            if (u >= live) break;
            if (e.ty == SDS_F32) static_cast<float*>(g.out)[to + u] = z[u];
            else static_cast<uint16_t*>(g.out)[to + u] = round16(z[u], g.f16);
          }
        }
      }
    } else {
      const int col = n0 + 4 * lane;
      if (col < g.N) {
        if (EPI == kFfnOut) {
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(g.out) + (size_t)tok * g.ldo + col) =
              make_uint2(pack16(s.x, s.y, g.f16), pack16(s.z, s.w, g.f16));
        } else {
          const float4 p = *reinterpret_cast<const float4*>(g.keep + keep_index(tok, col, ncc, 0));
          const float4 w = *reinterpret_cast<const float4*>(g.keep + keep_index(tok, col, ncc, 1));
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(g.out) + (size_t)tok * g.ldo + col) =
              make_uint2(pack16(s.x * p.x, s.y * p.y, g.f16), pack16(s.z * p.z, s.w * p.w, g.f16));
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(g.out2) + (size_t)tok * g.ldo + col) =
              make_uint2(pack16(s.x * w.x, s.y * w.y, g.f16), pack16(s.z * w.z, s.w * w.w, g.f16));
        }
      }
    }
  }
  if (*abort_s && threadIdx.x == 0) {
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);   // copies still in flight land before the memory is released
  }
  __syncthreads();
  if (nsplit > 1) cluster_sync_all();             // no CTA leaves while a peer may still read its sums
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)C::kTmemCols) : "memory");
  }
}

// ---------------------------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------------------------

constexpr int kMaxDevices = 64;

int current_device() {
  int dev = 0;
  return cudaGetDevice(&dev) == cudaSuccess && dev >= 0 && dev < kMaxDevices ? dev : -1;
}

// cluster size, and the permission to start before the kernel in front has ended (see wait_for_prior_kernel)
void launch_attributes(cudaLaunchAttribute (&attr)[2], int cluster) {
  attr[0] = cudaLaunchAttribute{};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1] = cudaLaunchAttribute{};
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
}

// a kernel's shared-memory limit and the number of its clusters that are resident at once, per device, looked up once
struct KernelInfo {
  std::atomic<int> resident[kMaxDevices];         // 0: not looked up; else 1 + resident CTAs (clusters of a pair)
};

template <int BN, int EPI, bool PAIR, bool MN, bool CUT, int EW, bool SUMS>
cudaError_t tile_resident(int* n) {
  static KernelInfo info;                         // zero-initialised
  using C = FfnTile<BN, PAIR, EW>;
  const int dev = current_device();
  if (dev < 0) return cudaErrorInvalidDevice;
  int r = info.resident[dev].load(std::memory_order_acquire);
  if (r == 0) {
    cudaError_t e = cudaFuncSetAttribute(k_ffn_tile<BN, EPI, PAIR, MN, CUT, EW, SUMS>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmemBytes);
    if (e != cudaSuccess) return e;
    int sms = 0, got = 0;
    if ((e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
    got = sms;
    if (PAIR) {
      cudaLaunchConfig_t cfg{};
      cfg.gridDim = dim3(sms / 2 * 2);
      cfg.blockDim = dim3(tile_threads(EW));
      cfg.dynamicSmemBytes = C::kSmemBytes;
      cudaLaunchAttribute attr{};
      attr.id = cudaLaunchAttributeClusterDimension;
      attr.val.clusterDim.x = 2; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
      cfg.attrs = &attr;
      cfg.numAttrs = 1;
      if ((e = cudaOccupancyMaxActiveClusters(&got, k_ffn_tile<BN, EPI, PAIR, MN, CUT, EW, SUMS>, &cfg)) != cudaSuccess) return e;
      got = std::min(got, sms / 2);
    }
    if (got < 1) return cudaErrorLaunchOutOfResources;
    r = got + 1;
    info.resident[dev].store(r, std::memory_order_release);
  }
  *n = r - 1;
  return cudaSuccess;
}

template <int BN, int EPI, bool PAIR, bool MN, bool CUT, int EW, bool SUMS>
cudaError_t launch_tile_t(const FfnTileArgs& g, int64_t tiles, cudaStream_t st) {
  using C = FfnTile<BN, PAIR, EW>;
  int resident = 0;
  const cudaError_t e = tile_resident<BN, EPI, PAIR, MN, CUT, EW, SUMS>(&resident);
  if (e != cudaSuccess) return e;
  const int workers = (int)std::min<int64_t>(tiles, resident);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(PAIR ? 2 * workers : workers);
  cfg.blockDim = dim3(tile_threads(EW));
  cfg.dynamicSmemBytes = C::kSmemBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  launch_attributes(attr, PAIR ? 2 : 1);
  return cudaLaunchKernelEx(&cfg, k_ffn_tile<BN, EPI, PAIR, MN, CUT, EW, SUMS>, g);
}

// where an operand lies: [rows, cols] with rows ld elements apart; K-major if K runs along the columns
struct Mat {
  const void* p;
  int64_t ld;
};

// one product's tensor maps: operand rows (M or N) by K elements, box of `box` rows (K-major) or 64 k (MN-major)
bool map_operand(CUtensorMap* tm, const Mat& m, bool f16, int64_t mn, int64_t k, bool mn_major, int box) {
  return mn_major ? make_tmap_2d(tm, m.p, f16, (uint64_t)k, (uint64_t)mn, (uint64_t)m.ld, 64)
                  : make_tmap_2d(tm, m.p, f16, (uint64_t)mn, (uint64_t)k, (uint64_t)m.ld, (uint32_t)box);
}

struct ProductSpec {
  Mat a[2], b[2];
  int nseg;
  bool a_mn;
  int M, N, K;
  void* out;
  int64_t ldo;
  int parts = 1;                                  // of K, each with its own tiles
  float* part = nullptr;
};

inline int64_t tiles_of(int64_t m, int64_t n, int tm, int tn) { return ((m + tm - 1) / tm) * ((n + tn - 1) / tn); }
inline int64_t tiles_of(const ProductSpec& s, int tm, int tn) { return tiles_of(s.M, s.N, tm, tn) * s.parts; }
inline int steps(int k) { return (k + kBK - 1) / kBK; }
inline int ksteps(const ProductSpec& s) { return (steps(s.K) * s.nseg + s.parts - 1) / s.parts; }   // of a tile

// Tile shape: single CTAs on 128 x 128 tiles while these are at most one per SM (each has an SM of its own), pairs on
// 256 x 256 tiles above that. Several products of one launch: those with the longer tiles come first; there are at most
// two lengths (specs[0] may differ from the others).
template <int EPI, bool MN, bool CUT = false, int EW = kEpiWarps, bool SUMS = false>
cudaError_t launch_tiles(const FfnArgs& a, ProductSpec* specs, int n, bool first, cudaStream_t st,
                         float* keep = nullptr, void* out2 = nullptr, bool beside = false, const LinearEpilogue* lin = nullptr) {
  constexpr int kWide = EPI == kFfnGlu ? 128 : 256, kNarrow = EPI == kFfnGlu ? 64 : 128;   // output columns of a tile
  if (n > 1 && ksteps(specs[0]) < ksteps(specs[n - 1])) std::swap(specs[0], specs[n - 1]);
  int64_t small = 0, wide = 0;
  for (int i = 0; i < n; ++i) {
    small += tiles_of(specs[i], 128, kNarrow);
    wide += tiles_of(specs[i], 256, kWide);
  }
  const bool pair = small > 148;
  // tiles of the longer class, and how many of the shorter one take as long
  int longer = 1;
  while (longer < n && ksteps(specs[longer]) == ksteps(specs[0])) ++longer;
  int64_t na = 0;
  for (int i = 0; i < longer; ++i) na += pair ? tiles_of(specs[i], 256, kWide) : tiles_of(specs[i], 128, kNarrow);
  FfnTileArgs g;
  g.np = n;
  g.na = (int)na;
  g.give = longer < n ? (ksteps(specs[0]) + ksteps(specs[n - 1]) / 2) / ksteps(specs[n - 1]) : 0;
  g.f16 = a.f16;
  g.act = a.act;
  g.nrows_dev = a.nrows_dev;
  g.keep = keep;
  g.out2 = out2;
  g.err = a.err;
  g.clear_err = first && !a.res;
  g.beside = beside;
  if (lin) g.lin = *lin;
  for (int i = 0; i < n; ++i) {
    const ProductSpec& s = specs[i];
    FfnProduct& p = g.p[i];
    p.M = s.M; p.N = s.N; p.K = s.K;
    p.nseg = s.nseg; p.a_mn = s.a_mn;
    p.out = s.out; p.ldo = s.ldo;
    p.parts = s.parts; p.part = s.part;
    p.band = (int)std::max<int64_t>(8, std::min<int64_t>(32, (32 << 20) / ((pair ? 256 : 128) * 2 * (int64_t)ksteps(s) * kBK)));
    const int box_b = EPI == kFfnGlu && !pair ? 64 : 128;
    for (int k = 0; k < (EPI == kFfnGlu ? 2 : s.nseg); ++k) {
      if (k < s.nseg && !map_operand(&p.a[k], s.a[k], a.f16 != 0, s.M, s.K, s.a_mn, 128)) return cudaErrorInvalidValue;
      if (!map_operand(&p.b[k], s.b[k], a.f16 != 0, s.N, s.K, MN, box_b)) return cudaErrorInvalidValue;
    }
  }
  if (pair) {
    const cudaError_t e = launch_tile_t<256, EPI, true, MN, CUT, EW, SUMS>(g, wide, st);
    if (e != cudaErrorLaunchOutOfResources) return e;
    // no cluster can be resident: single CTAs, whose tile of the fused projections has its own box
    for (int i = 0; EPI == kFfnGlu && i < n; ++i)
      for (int k = 0; k < 2; ++k)
        if (!map_operand(&g.p[i].b[k], specs[i].b[k], a.f16 != 0, specs[i].N, specs[i].K, MN, 64))
          return cudaErrorInvalidValue;
  }
  return launch_tile_t<128, EPI, false, MN, CUT, EW, SUMS>(g, small, st);
}

template <int BN, int EPI>
cudaError_t launch_split_t(const FfnSplitArgs& g, int tiles, int splits, cudaStream_t st) {
  using C = FfnSplit<BN, EPI>;
  static KernelInfo info;
  const int dev = current_device();
  if (dev < 0) return cudaErrorInvalidDevice;
  if (info.resident[dev].load(std::memory_order_acquire) == 0) {
    const cudaError_t e = cudaFuncSetAttribute(k_ffn_split<BN, EPI>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmemBytes);
    if (e != cudaSuccess) return e;
    info.resident[dev].store(1, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(tiles * splits, (g.rows + BN - 1) / BN);
  cfg.blockDim = dim3(kSplitThreads);
  cfg.dynamicSmemBytes = C::kSmemBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  launch_attributes(attr, splits);
  return cudaLaunchKernelEx(&cfg, k_ffn_split<BN, EPI>, g);
}

// weights [N, K] (or [K, N]: w_mn) times tokens [rows, K]
struct SplitSpec {
  Mat w[2], t[2];
  int nseg;
  bool w_mn;
  int N, K;
  void* out;
  void* out2;
  int64_t ldo;
};

inline int ksteps(const SplitSpec& s) { return (s.K + kBK - 1) / kBK * s.nseg; }
inline int split_tokens(int rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128; }
// CTAs per tile along K: until two CTAs on every SM read weights, with at least four steps of K each
inline int split_count(int rows, int tiles, int nkb) {
  const int bn = split_tokens(rows), tok = (rows + bn - 1) / bn;
  int s = 1;
  while (s < 8 && (int64_t)tiles * tok * 2 * s <= 2 * 148 && nkb / (2 * s) >= 4) s *= 2;
  return s;
}

// Which form a product of the feed-forward block takes (linear layers: linear_form), for `rows` tokens and N output columns: the shorter
// estimated time, in steps of K of one CTA (0.35 us where few CTAs run, 0.3 us for those of a full launch of pairs: the times before the
// feeding lanes were elected, kept so that a block's sums keep their order) plus what a launch and its epilogue cost. Beyond 2048 rows the few-row form has to be clearly ahead, as it is for few columns and a long K
// (3000 x 64 x 8192 forward 80 -> 53 us, 2100 x 512 x 12288 112 -> 85); close calls there went the other way
// (4096 x 128 x 512 forward 13.8 -> 17.4).
template <int EPI>
bool prefer_split(int rows, int N, int nkb) {
  constexpr int TN = EPI == kFfnGlu ? 64 : 128;
  if (rows <= 64) return true;                    // half a tile of rows and more would be empty
  if (rows > 65535 * 128) return false;           // (blocks of tokens are the grid's second dimension)
  const int tok = (rows + 127) / 128, tiles = (N + TN - 1) / TN;
  const int splits = split_count(rows, tiles, nkb);
  const int64_t ctas = (int64_t)tiles * tok * splits;
  const double split = (double)((ctas + 147) / 148) * ((nkb + splits - 1) / splits) * 0.35 + 2.0 + 0.5 * splits;
  const int64_t small = (int64_t)tok * tiles, wide = (int64_t)((rows + 255) / 256) * ((N + 2 * TN - 1) / (2 * TN));
  const double tile = small <= 148 ? nkb * 0.35 + 2.0 : (double)((wide + 73) / 74) * nkb * 0.3 + 4.0;
  return split < (rows <= 2048 ? 1.0 : 0.7) * tile;
}

template <int EPI>
cudaError_t launch_split(const FfnArgs& a, const SplitSpec& s, float* keep, bool first, cudaStream_t st,
                         const LinearEpilogue* lin = nullptr, int count = 0, int tokens = 0) {
  constexpr int TN = EPI == kFfnGlu ? 64 : 128;
  const int bn = tokens > 0 ? tokens : split_tokens(a.rows);
  FfnSplitArgs g;
  g.rows = a.rows; g.N = s.N; g.K = s.K;
  g.nseg = s.nseg; g.w_mn = s.w_mn;
  g.f16 = a.f16; g.act = a.act;
  g.keep = keep;
  g.out = s.out; g.out2 = s.out2; g.ldo = s.ldo;
  g.err = a.err;
  g.clear_err = first;
  if (lin) g.lin = *lin;
  const int nw = EPI == kFfnGlu ? 2 : s.nseg;
  for (int k = 0; k < nw; ++k)
    if (!map_operand(&g.w[k], s.w[k], a.f16 != 0, s.N, s.K, s.w_mn, EPI == kFfnGlu ? 64 : 128)) return cudaErrorInvalidValue;
  for (int k = 0; k < s.nseg; ++k)
    if (!map_operand(&g.t[k], s.t[k], a.f16 != 0, a.rows, s.K, false, bn)) return cudaErrorInvalidValue;
  const int tiles = (s.N + TN - 1) / TN;
  const int splits = count > 0 ? count : split_count(a.rows, tiles, ksteps(s));
  switch (bn) {
    case 16: return launch_split_t<16, EPI>(g, tiles, splits, st);
    case 32: return launch_split_t<32, EPI>(g, tiles, splits, st);
    case 64: return launch_split_t<64, EPI>(g, tiles, splits, st);
    default: return launch_split_t<128, EPI>(g, tiles, splits, st);
  }
}

}  // namespace

}  // namespace sds
