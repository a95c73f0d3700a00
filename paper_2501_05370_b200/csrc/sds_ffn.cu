// Gated feed-forward block, forward and backward, on the tensor cores.
//
//   forward   G = x Wg^T, U = x Wu^T, h = act(G) * U, y = h Wd^T
//   backward  dH = dy Wd, dG = dH * U act'(G), dU = dH * act(G)
//             dx = dG Wg + dU Wu, dWg = dG^T x, dWu = dU^T x, dWd = dy^T h
//
// Both projections, the activation and the product are one kernel: a tile holds the same columns of G and of U in
// one accumulator, and its epilogue writes h only. For the backward pass it also keeps the two factors
// U act'(G) and act(G) as floats (16 bits there would add an error to every gradient as large as its own rounding,
// and the activation would have to be evaluated again); they lie in the order in which the epilogue's threads
// hold them, so that every access is 512 contiguous bytes of a warp. h and dG, dU are rounded to the operand type:
// they are operands of the products that follow.
//
// Two forms of the products:
//   - k_ffn_tile: persistent CTA pairs on 256 x 256 tiles (single CTAs on 128 x 128 tiles where there are few), for
//     batches. Operands arrive by TMA in either order (K contiguous, or M / N contiguous for the transposed
//     operands of the gradients: the matrix descriptors and the instruction descriptor say which, nothing is
//     transposed in memory). Two accumulators: the epilogue of a tile runs under the next tile's products.
//   - k_ffn_split: few rows. The time is that of reading the weights once, so the weights are the 128 rows of the
//     instruction and the tokens its 16 to 128 columns; K is split over a cluster of CTAs so that all SMs
//     read, and the partial sums are added through distributed shared memory in the order of K.
// Sums are held in 32 bits (tensor memory) throughout.
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
};

constexpr int kBM = 128;                          // rows of one CTA's accumulator
constexpr int kBK = 64;                           // elements of K per stage: one 128-byte swizzle row
constexpr int kChunkBytes = 64 * kBK * 2;         // 64 x 64 elements
// Epilogue warps: one per quarter of the lanes. The main loop takes up shared memory (operand tiles written and read:
// 128 bytes per cycle), and every warp that stages and polls beside it costs; four finish a tile well within the next
// one's products. Measured at 16384 rows, d = 2048, f = 8192 in a long run: forward projections 806 us with 4 warps, 896
// with 8; dH 550 and 566; second product 430 and 447.
constexpr int kEpiWarps = 4;
constexpr int kTileThreads = 64 + 32 * kEpiWarps; // warp 0: TMA, warp 1: MMA and tensor memory, then the epilogue
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
};

// ---------------------------------------------------------------------------------------------
// the epilogues' arithmetic
// ---------------------------------------------------------------------------------------------

// a = act(g), da = act'(g). The fast exponential and division are accurate to a few units of the 24-bit
// significand, far inside the 16-bit operands' rounding.
// GELU: with z = |g| / sqrt(2), Phi(-|g|) = erfcx(z) exp(-z^2) / 2, and the exponential is that of the density. The scaled
// function is smooth in t = 1 / (1 + 0.33 z): t times a polynomial of degree 7, fitted (least squares, reweighted towards the
// smallest largest relative error) to 8.2e-8 for z up to 9.6. In floats Phi(-|g|) is off by at most 6e-7 of
// itself up to |g| = 3 and 1.3e-6 up to 6. (With erfcf and a second exponential the epilogue took longer than the
// products up to d = 2048: 16384 x 512 x 2048 forward 182 us.)
template <int ACT>
__device__ __forceinline__ void activation(float g, float& a, float& da) {
  if (ACT == SDS_ACT_SILU) {
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
__device__ __forceinline__ void store_rows64(uint4* stg, const uint32_t (&w)[16], char* out, size_t ld_bytes, int nrows,
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

// Kernels overlap their starts: one may be started when all CTAs of the one in front have said so (or ended), and waits
// for that kernel's end, and for its writes, here. Two kinds read device memory before that wait: k_ffn_split in a call's later
// products, the weights, which nothing in the call writes; and a tile launch `beside` (FfnTileArgs), all it needs, as it reads
// nothing of the kernel in front. Both are right only because the kernel directly in front is one of the same call that said so
// after its own wait: what ran before that one had then ended. So neither a norm kernel (it says so before its wait) nor
// a launch `beside` (it waits in the end) may stand there: behind these come only first kernels of calls and k_ffn_join, which
// wait before they read anything.
__device__ __forceinline__ void launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_prior_kernel() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

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

// Self-test of that report: one thread waits on a barrier that nobody arrives on, with a limit of its own.
__global__ void k_ffn_wait_selftest(uint32_t polls, int* err) {
  __shared__ uint64_t bar;
  mbar_init(&bar, 1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  *err = 0;
  bool done = false;
  for (uint32_t it = 0; it < polls && !done; ++it) done = mbar_try_wait(&bar, 0u);
  if (!done) give_up(err, 3);
}

// ---------------------------------------------------------------------------------------------
// batches: persistent tiles
// ---------------------------------------------------------------------------------------------

template <int BN, bool PAIR> struct FfnTile {
  static constexpr int kTM = PAIR ? 2 * kBM : kBM;                 // rows of a tile
  static constexpr int kBRows = PAIR ? BN / 2 : BN;                // rows of B that one CTA stages
  static constexpr int kABytes = kBM * kBK * 2;
  static constexpr int kBBytes = kBRows * kBK * 2;
  static constexpr int kStageBytes = kABytes + kBBytes;
  static constexpr int kFixedBytes = 1024 /*align*/ + 256 /*barriers*/ + kEpiWarps * kWarpStage;
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
// Bound by the tensor cores: 16384 x 2048 x 8192 forward 1280 us, 1290 TFLOP/s (92 % of the library's rate in a long run, where power
// sets the clock); 8192 rows forward and backward 2130 us, 1160 TFLOP/s beside the kept factors.
// CUT: products whose K is cut (FfnProduct::parts); its own kernel, as the others lose up to 5 % to the arithmetic.
template <int BN, int EPI, bool PAIR, bool MN, bool CUT>
__global__ void __launch_bounds__(kTileThreads, 1) k_ffn_tile(const __grid_constant__ FfnTileArgs g) {
  using C = FfnTile<BN, PAIR>;
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

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
  const int worker = PAIR ? (int)(blockIdx.x >> 1) : (int)blockIdx.x;
  const int nworkers = PAIR ? (int)(gridDim.x >> 1) : (int)gridDim.x;
  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) { mbar_init(full_bar + s, 1); mbar_init(empty_bar + s, 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(tfull_bar + s, 1); mbar_init(tempty_bar + s, PAIR ? 2 * kEpiWarps : kEpiWarps); }
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
    if (lane == 0) {
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
    if (lane == 0 && rank == 0) {
      int stage = 0, it = 0;
      uint32_t phase = 0;
      bool ok = true;
      bool more = tile_at<TM, TN, CUT>(g, M0, tile_index(g, worker, nworkers, 0), &at);
      for (; ok && more; ++it) {
        const FfnProduct& p = g.p[at.prod];
        const int all = (p.K + kBK - 1) / kBK * p.nseg;
        const int nkb = CUT ? first_step(all, p.parts, at.part + 1) - first_step(all, p.parts, at.part) : all;
        const int buf = it & 1;
        if (!mbar_wait(tempty_bar + buf, ((uint32_t)(it >> 1) & 1u) ^ 1u, abort_s)) { ok = false; break; }
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + (uint32_t)(buf * BN);
        const auto multiply = [&](auto order) {
          constexpr bool a_mn = decltype(order)::value;
          const uint32_t idesc = make_idesc(TM, BN, g.f16 != 0, a_mn, MN);
          const uint64_t adesc0 = make_sdesc(smem_u32(stages), a_mn ? (uint32_t)kChunkBytes : 0u);
          const uint64_t bdesc0 = make_sdesc(smem_u32(stages) + C::kABytes, MN ? (uint32_t)kChunkBytes : 0u);
          constexpr uint64_t a_step = a_mn ? 128u : 2u, b_step = MN ? 128u : 2u;    // 16 elements of K, in 16 bytes
          for (int kb = 0; kb < nkb; ++kb) {
            if (!mbar_wait(full_bar + stage, phase, abort_s)) { ok = false; break; }
            tc_fence_after();
            const uint64_t adesc = adesc0 + (uint64_t)(stage * (C::kStageBytes >> 4));
            const uint64_t bdesc = bdesc0 + (uint64_t)(stage * (C::kStageBytes >> 4));
#pragma unroll
            for (int k = 0; k < kBK / 16; ++k) {
              if (PAIR) umma_f16_pair(d_tmem, adesc + a_step * k, bdesc + b_step * k, idesc, (kb | k) ? 1u : 0u);
              else umma_f16(d_tmem, adesc + a_step * k, bdesc + b_step * k, idesc, (kb | k) ? 1u : 0u);
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
      if (!ok) {
        raise_abort(abort_s, PAIR);
        give_up(g.err, 2);
      }
    }
  } else {
    // ---------------- epilogue: a warp reaches the 32 tensor-memory lanes of quarter warp % 4 ----------------
    const int q = warp & 3;
    constexpr int kChunks = TN / 32;              // chunks of 32 output columns
    uint4* stg = reinterpret_cast<uint4*>(epi_stage + (warp - 2) * kWarpStage);
    const uint32_t drained0 = (PAIR && rank != 0) ? map_to_cta(smem_u32(tempty_bar), 0u) : 0u;
    const int f16 = g.f16;
    int it = 0;
    bool ok = true;
    for (; ok && tile_at<TM, TN, CUT>(g, M0, tile_index(g, worker, nworkers, it), &at); ++it) {
      const FfnProduct& p = g.p[at.prod];
      const int M = at.prod == 0 ? M0 : p.M, N = p.N;
      const int buf = it & 1;
      const int row0 = at.m * TM + (int)rank * kBM + q * 32, n0 = at.n * TN;
      const int nlive = min(32, M - row0);        // (may be negative)
      const uint32_t tbase = tmem_base + (uint32_t)(buf * BN) + ((uint32_t)(q * 32) << 16);
      const int ncc = (N + 31) >> 5;
      // the kept factors do not depend on this product: requested before its accumulator is waited for
      float4 kp[8], kq[8];
      auto keep_fetch = [&](int col) {
        const bool in = nlive > 0 && col < N;
        const float4* kp0 = reinterpret_cast<const float4*>(g.keep + (in ? keep_index(row0 + lane, col, ncc, 0) : 0));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          kp[i] = in ? __ldg(kp0 + i * 32) : make_float4(0.f, 0.f, 0.f, 0.f);
          kq[i] = in ? __ldg(kp0 + (8 + i) * 32) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
      };
      if (EPI == kFfnDGlu) keep_fetch(n0);
      if (!wait_for_sums(tfull_bar + buf, (uint32_t)(it >> 1) & 1u, abort_s, (p.K + kBK - 1) / kBK * p.nseg)) { ok = false; break; }
      tc_fence_after();
#pragma unroll 1
      for (int chunk = 0; chunk < kChunks; ++chunk) {
        const int c = chunk * 32, col = n0 + c;
        uint32_t acc[32], up[EPI == kFfnGlu ? 32 : 1];
        tmem_ld32(tbase + (uint32_t)c, acc);
        if (EPI == kFfnGlu) tmem_ld32(tbase + (uint32_t)(BN / 2 + c), reinterpret_cast<uint32_t(&)[32]>(up));
        if (chunk == kChunks - 1) {               // accumulator read: hand the buffer back
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            if (PAIR && rank != 0) mbar_arrive_cluster(drained0 + (uint32_t)buf * 8u);
            else mbar_arrive(tempty_bar + buf);
          }
        }
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
          if (chunk < kChunks - 1) keep_fetch(col + 32);
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
};

constexpr int kSplitThreads = 256;

template <int BN> struct FfnSplit {
  static constexpr int kABytes = kBM * kBK * 2, kBBytes = BN * kBK * 2, kStageBytes = kABytes + kBBytes;
  static constexpr int kFixedBytes = 1024 + 256;
  // half of an SM's shared memory, so that two CTAs share an SM: clusters of eight are then all resident at once, and
  // the CTAs of the next product request their weights while the last ones of this product finish
  static constexpr int kStages = (113 * 1024 - kFixedBytes) / kStageBytes;
  static constexpr int kSmemBytes = kStages * kStageBytes + kFixedBytes;
  static constexpr int kTmemCols = BN < 32 ? 32 : BN;
  static_assert(kStages * kStageBytes >= BN * kBM * 4, "the partial sums fit where the stages were");
};

__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}

// 2048 x 8192 bf16, both products: 1 row 24.9 us (4.0 TB/s of weights), 64 rows 31, 128 rows 34; 8 rows of 4096 x 14336 60.8 us
// (5.8 TB/s, 88 % of a copy's rate). What is left of a small call is the ramp of the requests and the exchange, once per product.
template <int BN, int EPI>
__global__ void __launch_bounds__(kSplitThreads, 2) k_ffn_split(const __grid_constant__ FfnSplitArgs g) {
  using C = FfnSplit<BN>;
  constexpr int TN = EPI == kFfnGlu ? 64 : 128;   // output columns of a CTA
  extern __shared__ uint8_t smem_raw[];
  uint8_t* stages = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(stages + C::kStages * C::kStageBytes);
  uint64_t* empty_bar = full_bar + C::kStages;
  uint64_t* tfull_bar = empty_bar + C::kStages;
  uint32_t* tmem_base_s = reinterpret_cast<uint32_t*>(tfull_bar + 1);
  volatile int* abort_s = reinterpret_cast<volatile int*>(tmem_base_s + 1);
  float* part = reinterpret_cast<float*>(stages); // [BN][128], once the products are done

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t nsplit;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(nsplit));
  const uint32_t rank = cluster_ctarank();
  const int n0 = (int)(blockIdx.x / nsplit) * TN, tok0 = (int)blockIdx.y * BN;
  const int kb_seg = (g.K + kBK - 1) / kBK, nkb = kb_seg * g.nseg;
  const int kb0 = (int)((int64_t)nkb * rank / nsplit), kb1 = (int)((int64_t)nkb * (rank + 1) / nsplit);

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

  if (warp == 0 && lane == 0) {
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
  } else if (warp == 1 && lane == 0) {
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
#pragma unroll
      for (int k = 0; k < kBK / 16; ++k)
        umma_f16(tmem_base, adesc + a_step * k, bdesc + (uint64_t)(2 * k), idesc, (kb > kb0 || k) ? 1u : 0u);
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
#pragma unroll
    for (int c = 0; c < BN / 2; ++c) part[(half * (BN / 2) + c) * kBM + q * 32 + lane] = __uint_as_float(acc[c]);
  } else if (lane == 0) {
    *abort_s = 1;
    give_up(g.err, 3);
  }
  tc_fence_before();
  if (nsplit > 1) cluster_sync_all(); else __syncthreads();

  // this CTA's share of the tokens: partial sums added in the order of K, then the epilogue; a lane holds four columns
  const int share = BN / (int)nsplit;
  const uint32_t part_a = smem_u32(part);
  const int ncc = (g.N + 31) >> 5;
  for (int i = warp; i < share; i += kSplitThreads / 32) {
    const int tk = (int)rank * share + i, tok = tok0 + tk;
    if (tok >= g.rows) break;
    const uint32_t off = (uint32_t)(tk * kBM + lane * 4) * 4u;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (nsplit == 1) {
      s = *reinterpret_cast<const float4*>(part + tk * kBM + lane * 4);
    } else {
      for (uint32_t r = 0; r < nsplit; ++r) {
        const float4 v = ld_cluster4(map_to_cta(part_a + off, r));
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
      }
    }
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

template <int BN, int EPI, bool PAIR, bool MN, bool CUT>
cudaError_t tile_resident(int* n) {
  static KernelInfo info;                         // zero-initialised
  using C = FfnTile<BN, PAIR>;
  const int dev = current_device();
  if (dev < 0) return cudaErrorInvalidDevice;
  int r = info.resident[dev].load(std::memory_order_acquire);
  if (r == 0) {
    cudaError_t e = cudaFuncSetAttribute(k_ffn_tile<BN, EPI, PAIR, MN, CUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmemBytes);
    if (e != cudaSuccess) return e;
    int sms = 0, got = 0;
    if ((e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
    got = sms;
    if (PAIR) {
      cudaLaunchConfig_t cfg{};
      cfg.gridDim = dim3(sms / 2 * 2);
      cfg.blockDim = dim3(kTileThreads);
      cfg.dynamicSmemBytes = C::kSmemBytes;
      cudaLaunchAttribute attr{};
      attr.id = cudaLaunchAttributeClusterDimension;
      attr.val.clusterDim.x = 2; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
      cfg.attrs = &attr;
      cfg.numAttrs = 1;
      if ((e = cudaOccupancyMaxActiveClusters(&got, k_ffn_tile<BN, EPI, PAIR, MN, CUT>, &cfg)) != cudaSuccess) return e;
      got = std::min(got, sms / 2);
    }
    if (got < 1) return cudaErrorLaunchOutOfResources;
    r = got + 1;
    info.resident[dev].store(r, std::memory_order_release);
  }
  *n = r - 1;
  return cudaSuccess;
}

template <int BN, int EPI, bool PAIR, bool MN, bool CUT>
cudaError_t launch_tile_t(const FfnTileArgs& g, int64_t tiles, cudaStream_t st) {
  using C = FfnTile<BN, PAIR>;
  int resident = 0;
  const cudaError_t e = tile_resident<BN, EPI, PAIR, MN, CUT>(&resident);
  if (e != cudaSuccess) return e;
  const int workers = (int)std::min<int64_t>(tiles, resident);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(PAIR ? 2 * workers : workers);
  cfg.blockDim = dim3(kTileThreads);
  cfg.dynamicSmemBytes = C::kSmemBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  launch_attributes(attr, PAIR ? 2 : 1);
  return cudaLaunchKernelEx(&cfg, k_ffn_tile<BN, EPI, PAIR, MN, CUT>, g);
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
template <int EPI, bool MN, bool CUT = false>
cudaError_t launch_tiles(const FfnArgs& a, ProductSpec* specs, int n, bool first, cudaStream_t st,
                         float* keep = nullptr, void* out2 = nullptr, bool beside = false) {
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
    const cudaError_t e = launch_tile_t<256, EPI, true, MN, CUT>(g, wide, st);
    if (e != cudaErrorLaunchOutOfResources) return e;
    // no cluster can be resident: single CTAs, whose tile of the fused projections has its own box
    for (int i = 0; EPI == kFfnGlu && i < n; ++i)
      for (int k = 0; k < 2; ++k)
        if (!map_operand(&g.p[i].b[k], specs[i].b[k], a.f16 != 0, specs[i].N, specs[i].K, MN, 64))
          return cudaErrorInvalidValue;
  }
  return launch_tile_t<128, EPI, false, MN, CUT>(g, small, st);
}

template <int BN, int EPI>
cudaError_t launch_split_t(const FfnSplitArgs& g, int tiles, int splits, cudaStream_t st) {
  using C = FfnSplit<BN>;
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

// Which form a product of `rows` tokens with N output columns takes: the shorter estimated time, in steps of K of one
// CTA (about 0.35 us where few CTAs run, 0.3 us for those of a full launch of pairs) plus what a launch and its
// epilogue cost. Beyond 2048 rows the few-row form has to be clearly ahead, as it is for few columns and a long K
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
cudaError_t launch_split(const FfnArgs& a, const SplitSpec& s, float* keep, bool first, cudaStream_t st) {
  constexpr int TN = EPI == kFfnGlu ? 64 : 128;
  const int bn = split_tokens(a.rows);
  FfnSplitArgs g;
  g.rows = a.rows; g.N = s.N; g.K = s.K;
  g.nseg = s.nseg; g.w_mn = s.w_mn;
  g.f16 = a.f16; g.act = a.act;
  g.keep = keep;
  g.out = s.out; g.out2 = s.out2; g.ldo = s.ldo;
  g.err = a.err;
  g.clear_err = first;
  const int nw = EPI == kFfnGlu ? 2 : s.nseg;
  for (int k = 0; k < nw; ++k)
    if (!map_operand(&g.w[k], s.w[k], a.f16 != 0, s.N, s.K, s.w_mn, EPI == kFfnGlu ? 64 : 128)) return cudaErrorInvalidValue;
  for (int k = 0; k < s.nseg; ++k)
    if (!map_operand(&g.t[k], s.t[k], a.f16 != 0, a.rows, s.K, false, bn)) return cudaErrorInvalidValue;
  const int tiles = (s.N + TN - 1) / TN;
  const int splits = split_count(a.rows, tiles, ksteps(s));
  switch (bn) {
    case 16: return launch_split_t<16, EPI>(g, tiles, splits, st);
    case 32: return launch_split_t<32, EPI>(g, tiles, splits, st);
    case 64: return launch_split_t<64, EPI>(g, tiles, splits, st);
    default: return launch_split_t<128, EPI>(g, tiles, splits, st);
  }
}

}  // namespace

cudaError_t ffn_gave_up(int* role, cudaStream_t st) {
  *role = 0;
  const int none = 0;
  cudaError_t e = cudaMemcpyFromSymbolAsync(role, gave_up_word, sizeof(int), 0, cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess || *role == 0) return e;
  e = cudaMemcpyToSymbolAsync(gave_up_word, &none, sizeof(int), 0, cudaMemcpyHostToDevice, st);
  return e == cudaSuccess ? cudaStreamSynchronize(st) : e;
}

cudaError_t launch_ffn_wait_selftest(uint32_t polls, int* err, cudaStream_t st) {
  k_ffn_wait_selftest<<<1, 1, 0, st>>>(polls, err);
  return cudaGetLastError();
}

size_t ffn_keep_floats(int64_t rows, int64_t f) {
  return (size_t)((rows + 31) / 32 * 32) * (size_t)((f + 31) / 32 * 32) * 2;
}

namespace {

// h = act(x Wg^T) * (x Wu^T); y = h Wd^T
ProductSpec forward_in(const FfnArgs& a) {
  ProductSpec s{};
  s.a[0] = {a.x, a.ldx}; s.b[0] = {a.wg, a.d}; s.b[1] = {a.wu, a.d};
  s.nseg = 1; s.M = a.rows; s.N = a.f; s.K = a.d; s.out = a.h; s.ldo = a.f;
  return s;
}
ProductSpec forward_out(const FfnArgs& a, void* out, int64_t ldo) {
  ProductSpec s{};
  s.a[0] = {a.h, a.f}; s.b[0] = {a.wd, a.f};
  s.nseg = 1; s.M = a.rows; s.N = a.d; s.K = a.f; s.out = out; s.ldo = ldo;
  return s;
}

// Parts into which the contractions over the rows are cut, so that the few tiles of small weights' gradients fill the
// machine: the shortest estimated time (see prefer_split) of the launch that holds them, the tiles of dx included.
int gradient_parts(int rows, int d, int f) {
  const bool dx_tiles = !prefer_split<kFfnOut>(rows, d, 2 * steps(f));
  const int k = steps(rows), kx = dx_tiles ? 2 * steps(f) : 0;
  const int64_t small = 3 * tiles_of(f, d, 128, 128), wide = 3 * tiles_of(f, d, 256, 256);
  const int64_t xs = dx_tiles ? tiles_of(rows, d, 128, 128) : 0, xw = dx_tiles ? tiles_of(rows, d, 256, 256) : 0;
  const auto time = [&](int parts) {
    const int len = (k + parts - 1) / parts;
    const double join = parts > 1 ? 4.0 + (double)parts * d * f * 24.0 / 4e6 : 0.0;
    if (xs + small * parts <= 148) return 0.35 * std::max(kx, len) + 2.0 + join;
    const double full = ((double)xw * kx + (double)wide * parts * len) / 74.0;
    return 0.3 * std::max(full + 0.5 * std::min(kx ? kx : len, len), (double)std::max(kx, len)) + 4.0 + join;
  };
  int best = 1;
  double least = time(1);
  for (int parts = 2; parts <= 64 && k / parts >= 4; ++parts)
    if (time(parts) < least) { least = time(parts); best = parts; }
  return best;
}

size_t part_floats(int m, int n, int parts) {
  return parts > 1 ? (size_t)((m + 31) / 32 * 32) * (size_t)((n + 31) / 32 * 32) * (size_t)parts : 0;
}

}  // namespace

size_t ffn_part_floats(int64_t rows, int32_t d, int32_t f) {
  return rows > 0 ? 3 * part_floats(f, d, gradient_parts((int)rows, d, f)) : 0;
}

cudaError_t launch_ffn(const FfnArgs& a, cudaStream_t st) {
  if (a.rows <= 0) return cudaMemsetAsync(a.err, 0, sizeof(int), st);
  cudaError_t e;
  if (prefer_split<kFfnGlu>(a.rows, a.f, steps(a.d))) {
    SplitSpec s{};
    s.w[0] = {a.wg, a.d}; s.w[1] = {a.wu, a.d}; s.t[0] = {a.x, a.ldx};
    s.nseg = 1; s.N = a.f; s.K = a.d; s.out = a.h; s.ldo = a.f;
    e = launch_split<kFfnGlu>(a, s, a.keep, true, st);
  } else {
    ProductSpec s = forward_in(a);
    e = launch_tiles<kFfnGlu, false>(a, &s, 1, true, st, a.keep);
  }
  if (e != cudaSuccess) return e;
  if (prefer_split<kFfnOut>(a.rows, a.d, steps(a.f))) {
    SplitSpec s{};
    s.w[0] = {a.wd, a.f}; s.t[0] = {a.h, a.f};
    s.nseg = 1; s.N = a.d; s.K = a.f; s.out = a.y; s.ldo = a.ldy;
    return launch_split<kFfnOut>(a, s, nullptr, false, st);
  }
  ProductSpec s = forward_out(a, a.y, a.ldy);
  return launch_tiles<kFfnOut, false>(a, &s, 1, false, st);
}

cudaError_t launch_ffn_hidden(const FfnArgs& a, cudaStream_t st) {
  if (a.rows <= 0) return cudaSuccess;
  ProductSpec s = forward_in(a);
  return launch_tiles<kFfnGlu, false>(a, &s, 1, true, st);
}

cudaError_t launch_ffn_residual(const FfnArgs& a, cudaStream_t st) {
  if (a.rows <= 0) return cudaSuccess;
  ProductSpec s = forward_out(a, a.res, a.d);
  return launch_tiles<kFfnAdd, false>(a, &s, 1, false, st);      // (its caller launched launch_ffn_hidden before it)
}

cudaError_t launch_ffn_backward(const FfnArgs& a, cudaStream_t st) {
  cudaError_t e = cudaSuccess;
  if (a.rows <= 0 || !(a.dx || a.dwg || a.dwu || a.dwd)) {   // an empty sum: the weights' gradients are zeros
    if ((e = cudaMemsetAsync(a.err, 0, sizeof(int), st)) != cudaSuccess) return e;
    for (void* w : {a.dwg, a.dwu, a.dwd})
      if (w && (e = cudaMemsetAsync(w, 0, (size_t)a.d * a.f * 2, st)) != cudaSuccess) return e;
    return cudaSuccess;
  }
  bool first = true;
  if (a.dx || a.dwg || a.dwu) {                   // dH = dy Wd, dG and dU
    if (prefer_split<kFfnDGlu>(a.rows, a.f, steps(a.d))) {
      SplitSpec s{};
      s.w[0] = {a.wd, a.f}; s.t[0] = {a.dy, a.lddy};
      s.nseg = 1; s.w_mn = true; s.N = a.f; s.K = a.d; s.out = a.dg; s.out2 = a.du; s.ldo = a.f;
      e = launch_split<kFfnDGlu>(a, s, a.keep, first, st);
    } else {
      ProductSpec s{};
      s.a[0] = {a.dy, a.lddy}; s.b[0] = {a.wd, a.f};
      s.nseg = 1; s.M = a.rows; s.N = a.f; s.K = a.d; s.out = a.dg; s.ldo = a.f;
      e = launch_tiles<kFfnDGlu, true>(a, &s, 1, first, st, a.keep, a.du);
    }
    if (e != cudaSuccess) return e;
    first = false;
  }
  // the gradients of x and of the weights read the same dG and dU: one launch where x's product takes tiles too
  ProductSpec w[4];
  int n = 0;
  bool beside = false;
  if (a.dx && prefer_split<kFfnOut>(a.rows, a.d, 2 * steps(a.f))) {
    SplitSpec s{};
    s.w[0] = {a.wg, a.d}; s.w[1] = {a.wu, a.d}; s.t[0] = {a.dg, a.f}; s.t[1] = {a.du, a.f};
    s.nseg = 2; s.w_mn = true; s.N = a.d; s.K = a.f; s.out = a.dx; s.ldo = a.lddx;
    beside = true;                                // (the weights' gradients, launched next, do not read dx)
    if ((e = launch_split<kFfnOut>(a, s, nullptr, false, st)) != cudaSuccess) return e;
  } else if (a.dx) {
    ProductSpec s{};
    s.a[0] = {a.dg, a.f}; s.a[1] = {a.du, a.f}; s.b[0] = {a.wg, a.d}; s.b[1] = {a.wu, a.d};
    s.nseg = 2; s.M = a.rows; s.N = a.d; s.K = a.f; s.out = a.dx; s.ldo = a.lddx;
    w[n++] = s;
  }
  const int parts = gradient_parts(a.rows, a.d, a.f);
  FfnJoinArgs join{};
  int64_t blocks = 0;
  join.parts = parts; join.f16 = a.f16;
  const auto gradient = [&](const Mat& left, const Mat& right, int M, int N, void* out) {
    ProductSpec s{};
    s.a[0] = left; s.b[0] = right;
    s.nseg = 1; s.a_mn = true; s.M = M; s.N = N; s.K = a.rows; s.out = out; s.ldo = N;
    s.parts = parts; s.part = a.part + (size_t)join.np * part_floats(M, N, parts);
    join.p[join.np].part = s.part; join.p[join.np].out = static_cast<uint16_t*>(out);
    join.p[join.np].M = M; join.p[join.np].N = N;
    blocks += (int64_t)((M + 31) / 32) * ((N + 31) / 32);
    ++join.np;
    w[n++] = s;
  };
  if (a.dwg) gradient({a.dg, a.f}, {a.x, a.ldx}, a.f, a.d, a.dwg);
  if (a.dwu) gradient({a.du, a.f}, {a.x, a.ldx}, a.f, a.d, a.dwu);
  if (a.dwd) gradient({a.dy, a.lddy}, {a.h, a.f}, a.d, a.f, a.dwd);
  if (n == 0) return cudaSuccess;
  if (join.np == 0 || parts == 1) return launch_tiles<kFfnOut, true>(a, w, n, first, st, nullptr, nullptr, beside);
  if ((e = launch_tiles<kFfnOut, true, true>(a, w, n, first, st, nullptr, nullptr, beside)) != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)blocks);           // eight warps each: the eight quads of columns of a block
  cfg.blockDim = dim3(kJoinThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  launch_attributes(attr, 1);
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, k_ffn_join, join);
}

}  // namespace sds
