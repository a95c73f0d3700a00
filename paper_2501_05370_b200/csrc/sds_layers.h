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
// waits for st; *role: non-zero if a wait on the current device gave up since this was asked last
cudaError_t ffn_gave_up(int* role, cudaStream_t st);
cudaError_t launch_ffn_wait_selftest(uint32_t polls, int* err, cudaStream_t st);

}  // namespace sds
