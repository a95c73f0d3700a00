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
  float* factor;         // act'(z) [rows, n rounded up to 8], or NULL
  // backward
  const void* dy; int64_t lddy;                // of type ty
  void* dx; int64_t lddx;                      // any of the four gradients may be NULL
  void* dw; void* db; void* dtable;
  int* err;              // status word, at the workspace's begin
};

struct LinearWorkspace { size_t dz, db, dw, begin, list, table, bytes; };   // offsets of a backward call's parts, and their end
LinearWorkspace linear_workspace(int64_t rows, int32_t k, int32_t n, int32_t nsteps, bool has_table);
size_t linear_factor_bytes(int64_t rows, int32_t n);   // of act'
cudaError_t launch_linear(const LinearArgs& a, cudaStream_t st);
cudaError_t launch_linear_backward(const LinearArgs& a, cudaStream_t st);
cudaError_t linear_gave_up(int* role, cudaStream_t st);

// ---- residual norm (sds_residual.cuh, sds_residual*.cu) and dropout (sds_dropout.cu) ----

// D of dropout: zero or `scale`, from the library's generator (stream kStreamDropout)
struct DropoutArgs {
  uint32_t threshold;    // of 16 random bits, out of 65536; 0 = everything is kept, and nothing is drawn
  float scale;
  uint64_t seed;
  uint32_t step;         // counter word; the value at step_dev is added to it
  const int* step_dev;
  uint64_t row0;         // global number of row 0
};

struct ResidualNormArgs {
  int rows, d, per, groups;                      // per = rows / groups: rows that share a row of gate, scale and shift
  int tr, th;                                    // types of the stream (r, out, dr, dr_in) and of the branch (h, n, dn, dh)
  bool rms, post;
  float alpha, eps;
  DropoutArgs drop;
  const void* r; int64_t ldr;
  const void* h; int64_t ldh;                    // NULL = none: out = r, and out is not written
  void* out; int64_t ldo;
  void* n; int64_t ldn;
  const void* w; const void* b; const void* wp; int tw;                            // [d] each, NULL = ones, zeros, ones
  const void* gate; const void* scale; const void* shift; int tc;                  // [groups, d] each, NULL = ones, zeros, zeros
  int64_t ldgate, ldscale, ldshift;
  float4* stats;                                 // [rows][2]: mean, its remainder, 1 / size, and the same of post; forward: may be NULL
  // backward
  const void* dn; int64_t lddn;
  const void* dr; int64_t lddr;                  // NULL = zeros
  void* dr_in; int64_t lddr_in;
  void* dh; int64_t lddh;
  void* dw; void* db; void* dwp;
  void* dgate; void* dscale; void* dshift;
  int64_t lddgate, lddscale, lddshift;
  // how the rows are dealt out, and where their sums go
  int mode, workers, share;                      // rows of a worker
  float* part;                                   // [workers][3][d]
  float* group_part;                             // [workers][2][3][d]: sums of a group that began before the worker's rows, that goes on behind them
};

constexpr int kResidualMaxD = 16384;
// how a backward call sums over rows: sets mode and workers (the most) of a; floats of the two workspaces
void residual_norm_plan(ResidualNormArgs* a, size_t* part_floats, size_t* group_floats);
cudaError_t launch_residual_norm(const ResidualNormArgs& a, cudaStream_t st);
cudaError_t launch_residual_norm_backward(const ResidualNormArgs& a, cudaStream_t st);
// y = D x + residual over [rows, d]
struct DropoutCall {
  DropoutArgs drop;
  const void* x; int64_t ldx; int tx;
  const void* residual; int64_t ldr;             // of type ty, NULL = none
  void* y; int64_t ldy; int ty;
  int64_t rows;
  int d;
};
cudaError_t launch_dropout(const DropoutCall& a, cudaStream_t st);

// waits for st; *role: non-zero if a wait on the current device gave up since this was asked last
cudaError_t ffn_gave_up(int* role, cudaStream_t st);
cudaError_t launch_ffn_wait_selftest(uint32_t polls, int* err, cudaStream_t st);

}  // namespace sds
