// Layer norm of residual + dropout(x), forward: out = (z - mean) * rstd * weight + bias per row, z never stored.
//
// Bound: memory, x and residual once in and out once out.  A row stays in registers between the three steps (mean, then
// the sum of squared distances from it, then the output), so its variance is that of the definition without a
// second read and without the cancellation of E[z^2] - mean^2.
#include "rows.cuh"

namespace blossom {
namespace rows {
namespace {

constexpr int kRowsInFlight = 2;  // rows a thread loads before it works on the first

template <typename T, int W, typename P>
__global__ void __launch_bounds__(P::threads) norm_fwd_kernel(Args a, const T *__restrict__ x, const T *__restrict__ res,
                                                              const void *__restrict__ weight, const void *__restrict__ bias,
                                                              const int64_t *__restrict__ rng, T *__restrict__ out,
                                                              float2 *__restrict__ stats) {
  constexpr int TPR = P::TPR, U = kRowsInFlight;
  __shared__ float2 buf[TPR > 32 ? TPR / 16 : 1];
  grid_chain_enter();
  Generator gen;
  if (a.bar) gen.read(rng);
  const int g = (int)threadIdx.x % TPR, slot = (int)threadIdx.x / TPR, valid = a.cols - 8 * g;
  int turn = 0;
  float w[8], b[8];
  load_weights(weight, a.wide_weights, 8 * g, valid, 1.f, w);
  load_weights(bias, a.wide_weights, 8 * g, valid, 0.f, b);
  // (the bound is the same for all threads of a CTA: they meet in row_sum)
  for (int64_t r0 = (int64_t)blockIdx.x * (P::slots * U); r0 < a.rows; r0 += (int64_t)gridDim.x * (P::slots * U)) {
    float z[U][8], r[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t row = r0 + u * P::slots + slot;
      load_group<T, W>(x + row * a.sx + 8 * g, row < a.rows ? valid : 0, z[u]);
      load_group<T, W>(res + row * a.sr + 8 * g, res && row < a.rows ? valid : 0, r[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t row = r0 + u * P::slots + slot;
      if (a.bar) {
        const uint32_t m = gen.kept(a, (int)row, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) z[u][j] = m >> j & 1 ? z[u][j] * a.scale : 0.f;
      }
      float sum = 0.f, sq = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        z[u][j] += r[u][j];
        sum += z[u][j];
      }
      const float mean = row_sum<TPR>(sum, buf, turn) * a.inv_cols;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        z[u][j] = j < valid ? z[u][j] - mean : 0.f;
        sq += z[u][j] * z[u][j];
      }
      const float rstd = rsqrtf(row_sum<TPR>(sq, buf, turn) * a.inv_cols + a.eps);
      if (row < a.rows) {
#pragma unroll
        for (int j = 0; j < 8; ++j) z[u][j] = z[u][j] * rstd * w[j] + b[j];
        store_group<T, W>(out + row * a.so + 8 * g, valid, z[u]);
        if (stats && g == 0) stats[row] = make_float2(mean, rstd);
      }
    }
  }
}

}  // namespace
}  // namespace rows
}  // namespace blossom

extern "C" int blossom_add_norm_fwd(const blossom_rows_params *params, const void *x, const void *residual,
                                    const void *weight, const void *bias, const int64_t *rng, void *out, float *stats,
                                    blossom_stream_t stream) {
  using namespace blossom;
  prof_break();
  rows::Args a;
  if (int rc = rows::check(params, rows::kMaxCols, rng, &a)) return rc;
  if (a.rows == 0) return BLOSSOM_OK;
  const size_t esz = params->dtype == BLOSSOM_DTYPE_FP32 ? 4 : 2, wsz = a.wide_weights ? 4 : 2;
  if (!x || !out) return BLOSSOM_ERR_INVALID_ARG;
  for (const void *p : {x, residual, (const void *)out})
    if (reinterpret_cast<uintptr_t>(p) % esz) return BLOSSOM_ERR_INVALID_ARG;
  for (const void *p : {weight, bias})
    if (reinterpret_cast<uintptr_t>(p) % wsz) return BLOSSOM_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(stats) % 8) return BLOSSOM_ERR_INVALID_ARG;
  rows::Alignment al;
  al.rows_at(x, a.sx, esz);
  al.rows_at(residual, a.sr, esz);
  al.rows_at(out, a.so, esz);
  rows::with_plan(a.groups, [&](auto plan) {
    using P = decltype(plan);
    rows::with_type(params->dtype, al.elements(a.cols, esz), [&](auto t, auto w) {
      using T = decltype(t);
      const int64_t per = P::slots * rows::kRowsInFlight, ctas = (a.rows + per - 1) / per;
      const int64_t most = rows::kSMs * (2048 / P::threads);
      LaunchScope ls(K_NORM_FWD, (cudaStream_t)stream);
      launch_chained(rows::norm_fwd_kernel<T, decltype(w)::value, P>, dim3((unsigned)(ctas < most ? ctas : most)),
                     dim3(P::threads), 0, (cudaStream_t)stream, a, static_cast<const T *>(x),
                     static_cast<const T *>(residual), weight, bias, rng, static_cast<T *>(out),
                     reinterpret_cast<float2 *>(stats));
    });
  });
  return cudaGetLastError() == cudaSuccess ? BLOSSOM_OK : BLOSSOM_ERR_CUDA;
}
