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
// The products (sds_tiles.cuh) take one of two forms, by their estimated time. Sums are held in 32 bits (tensor memory) throughout.
#include "sds_tiles.cuh"

namespace sds {

namespace {

// Self-test of the report of a wait that gave up: one thread waits on a barrier that nobody arrives on, with a limit of its own.
__global__ void k_ffn_wait_selftest(uint32_t polls, int* err) {
  __shared__ uint64_t bar;
  mbar_init(&bar, 1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  *err = 0;
  bool done = false;
  for (uint32_t it = 0; it < polls && !done; ++it) done = mbar_try_wait(&bar, 0u);
  if (!done) give_up(err, 3);
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
