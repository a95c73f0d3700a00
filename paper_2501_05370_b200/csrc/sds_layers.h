// Host-side view of the layer kernels (layer norm, gated feed-forward block): argument blocks and launchers.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace sds {

// ---- layer norm (sds_norm.cu) ----

struct NormArgs {
  const void* x;         // [rows, d] of type tx, rows ldx elements apart
  void* y;               // [rows, d] of type ty, rows ldy elements apart
  const void* dy;        // backward: [rows, d] of type ty, rows lddy elements apart
  void* dx;              // backward: [rows, d] of type tx, rows lddx elements apart (may be NULL)
  int64_t ldx, ldy, lddy, lddx;
  const void* w;         // [d] of type tw, NULL = ones
  const void* b;         // [d] of type tw, NULL = zeros
  float* mean;           // [rows], forward: written unless NULL; backward: read
  float* rstd;           // [rows]
  void* dw;              // [d] of type tw (may be NULL)
  void* db;              // [d] of type tw (may be NULL)
  int tx, ty, tw;        // SDS_F32, SDS_BF16, SDS_F16
  int rows, d;
  float eps;
  bool wide;             // w and b are 16-byte aligned (set by the launchers)
  // denoiser form (float in, 16-bit out): the row norms follow `x + temb[rowk[row]]`, which is also written to
  // res [rows, d] float; the true row count lives on the device
  const int* nrows_dev;
  const int* rowk;
  const uint16_t* temb;  // [K, d] bf16, NULL = no embedding rows
  float* res;
  // backward workspace
  float* part;           // [norm_parts(rows, d)][2][d] partial sums of dw and db
  float* shift;          // [rows] row offsets (rows longer than the register kernels hold)
};

int norm_parts(int rows, int d);                    // CTAs of a backward launch, each with its partial sums
bool norm_is_long(int d);                           // rows that no register kernel holds
cudaError_t launch_norm(const NormArgs& a, cudaStream_t st);
cudaError_t launch_norm_backward(const NormArgs& a, cudaStream_t st);

// ---- gated feed-forward block (sds_ffn.cu) ----
// h = act(x Wg^T) * (x Wu^T), y = h Wd^T with x [rows, d], Wg and Wu [f, d], Wd [d, f]; 16-bit operands (all bf16 or
// all f16), d and f multiples of 8. dG, dU: gradients of the two pre-activations, [rows, f].

struct FfnArgs {
  int rows, d, f;
  int f16;               // operands are f16 (else bf16)
  int act;               // SDS_ACT_*
  const void* x; int64_t ldx;
  const void* wg; const void* wu; const void* wd;
  void* y; int64_t ldy;
  void* h;               // [rows, f]
  float* keep;           // factors of the backward pass (ffn_keep_floats), or NULL
  // backward
  const void* dy; int64_t lddy;
  void* dx; int64_t lddx;                      // any of the four gradients may be NULL
  void* dwg; void* dwu; void* dwd;
  void* dg; void* du;    // [rows, f] workspace
  float* part;           // workspace of the weights' gradients (ffn_part_floats)
  int* err;              // device word, set non-zero if a bounded wait gave up
  // denoiser form: the true row count lives on the device, and the product with Wd is added to res [rows, d]
  const int* nrows_dev;
  float* res;
};

size_t ffn_keep_floats(int64_t rows, int64_t f);
size_t ffn_part_floats(int64_t rows, int32_t d, int32_t f);
cudaError_t launch_ffn(const FfnArgs& a, cudaStream_t st);
cudaError_t launch_ffn_backward(const FfnArgs& a, cudaStream_t st);
// the denoiser's form of the two products (row count on the device, any number of rows through the same tiles):
// h = act(x Wg^T) * (x Wu^T), then res += h Wd^T. Every output element is the same bits however many rows there are.
cudaError_t launch_ffn_hidden(const FfnArgs& a, cudaStream_t st);
cudaError_t launch_ffn_residual(const FfnArgs& a, cudaStream_t st);

// ---- linear layer with its epilogue (sds_linear.cu) ----
// y = act(x W^T + b + table[step]) + residual with x [rows, k], W [n, k]; x, W, table of one 16-bit type, k a multiple of 8.

struct LinearArgs {
  int rows, k, n;
  int f16;               // x, W and the table are f16 (else bf16)
  int act;               // SDS_ACT_*
  const void* x; int64_t ldx;
  const void* w;
  const void* bias; int tbias;                 // [n] of any type, NULL = none
  const void* table; const int* step; int steps;
  const void* residual; int64_t ldr;           // of type ty, NULL = none
  void* y; int64_t ldy; int ty;                // SDS_F32 or the operands' type
  uint16_t* factor;      // act'(z) [rows, n rounded up to 8] f16, or NULL
  // backward
  const void* dy; int64_t lddy;                // of type ty
  void* dx; int64_t lddx;                      // any of the four gradients may be NULL
  void* dw; void* db; void* dtable;
  int* err;              // status word, at the workspace's begin
};

struct LinearWorkspace { size_t dz, db, dw, begin, list, table, bytes; };   // offsets of a backward call's parts, and their end
LinearWorkspace linear_workspace(int64_t rows, int32_t k, int32_t n, int32_t nsteps, bool has_table);
size_t linear_factor_bytes(int64_t rows, int32_t n);
cudaError_t launch_linear(const LinearArgs& a, cudaStream_t st);
cudaError_t launch_linear_backward(const LinearArgs& a, cudaStream_t st);
cudaError_t linear_gave_up(int* role, cudaStream_t st);

// waits for st; *role: non-zero if a wait on the current device gave up since this was asked last
cudaError_t ffn_gave_up(int* role, cudaStream_t st);
cudaError_t launch_ffn_wait_selftest(uint32_t polls, int* err, cudaStream_t st);

}  // namespace sds
