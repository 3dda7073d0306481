// Layer norm of residual + dropout(x), backward, with the reduction of the weight's and the bias's gradient.
//
// With a = dout * weight and n = (z - mean) * rstd:  dz = rstd * (a - mean(a) - n * mean(a n)), dresidual = dz,
// dx = dz where the dropout kept, scaled; dweight = sum over rows of dout n, dbias = sum over rows of dout.
// z and the mask are formed again: reading x and residual moves the bytes that a stored z would, and z is not rounded.
//
// Bound: memory, three tensors in and two out.  Each thread owns its columns for all rows of its CTA, so the column
// sums stay in registers; a CTA leaves one partial sum a column, and a second kernel adds the CTAs up in a fixed order.
#include "rows.cuh"

namespace blossom {
namespace rows {
namespace {

template <typename T, int W, typename P>
__global__ void __launch_bounds__(P::threads) norm_bwd_kernel(Args a, const T *__restrict__ x, const T *__restrict__ res,
                                                              const void *__restrict__ weight,
                                                              const int64_t *__restrict__ rng,
                                                              const float2 *__restrict__ stats,
                                                              const T *__restrict__ dout, T *__restrict__ dx,
                                                              T *__restrict__ dres, float *__restrict__ part) {
  constexpr int TPR = P::TPR;
  __shared__ float2 buf[TPR > 32 ? TPR / 16 : 1];
  __shared__ float2 sums[TPR <= 32 ? TPR * 8 : 1];
  grid_chain_enter();
  Generator gen;
  if (a.bar) gen.read(rng);
  const int g = (int)threadIdx.x % TPR, slot = (int)threadIdx.x / TPR, valid = a.cols - 8 * g;
  int turn = 0;
  float w[8], gw[8], gb[8];
  load_weights(weight, a.wide_weights, 8 * g, valid, 1.f, w);
#pragma unroll
  for (int j = 0; j < 8; ++j) gw[j] = gb[j] = 0.f;
  // (the bound is the same for all threads of a CTA: they meet in row_sum)
  for (int64_t r0 = (int64_t)blockIdx.x * P::slots; r0 < a.rows; r0 += (int64_t)gridDim.x * P::slots) {
    const int64_t row = r0 + slot;
    const bool there = row < a.rows;
    float z[8], r[8], d[8];
    uint32_t m = 0xffu;
    float2 st = make_float2(0.f, 0.f);
    if (there) st = stats[row];
    load_group<T, W>(x + row * a.sx + 8 * g, there ? valid : 0, z);
    load_group<T, W>(res + row * a.sr + 8 * g, res && there ? valid : 0, r);
    load_group<T, W>(dout + row * a.so + 8 * g, there ? valid : 0, d);
    if (a.bar) {
      m = gen.kept(a, (int)row, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] = m >> j & 1 ? z[j] * a.scale : 0.f;
    }
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      z[j] = j < valid ? (z[j] + r[j] - st.x) * st.y : 0.f;  // n; 0 in rows and columns that are not there, like d
      gw[j] += d[j] * z[j];
      gb[j] += d[j];
      d[j] *= w[j];  // a
      s.x += d[j];
      s.y += d[j] * z[j];
    }
    s = row_sum<TPR>(s, buf, turn);
    if (!there) continue;
    const float c1 = s.x * a.inv_cols, c2 = s.y * a.inv_cols;
#pragma unroll
    for (int j = 0; j < 8; ++j) d[j] = st.y * (d[j] - c1 - z[j] * c2);
    if (dres) store_group<T, W>(dres + row * a.sdr + 8 * g, valid, d);
    if (dx) {
      if (a.bar) {
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] = m >> j & 1 ? d[j] * a.scale : 0.f;
      }
      store_group<T, W>(dx + row * a.sdx + 8 * g, valid, d);
    }
  }
  if (!part) return;
  float *mine = part + (int64_t)blockIdx.x * 2 * a.cols;
  if constexpr (TPR <= 32) {
    // over the groups of threads of a warp, which hold the same columns, then warp by warp
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int o = TPR; o < 32; o <<= 1) {
        gw[j] += __shfl_xor_sync(0xffffffffu, gw[j], o);
        gb[j] += __shfl_xor_sync(0xffffffffu, gb[j], o);
      }
    for (int warp = 0; warp < P::threads / 32; ++warp) {
      if ((int)threadIdx.x / 32 == warp && (int)threadIdx.x % 32 < TPR) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float2 &p = sums[8 * g + j];
          p = warp ? make_float2(p.x + gw[j], p.y + gb[j]) : make_float2(gw[j], gb[j]);
        }
      }
      __syncthreads();
    }
    for (int c = (int)threadIdx.x; c < a.cols; c += P::threads) {
      mine[c] = sums[c].x;
      mine[a.cols + c] = sums[c].y;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < valid) mine[8 * g + j] = gw[j], mine[a.cols + 8 * g + j] = gb[j];
  }
}

// dweight and dbias from the CTAs' partial sums: 32 columns and 32 slices of the CTAs a block.
__global__ void __launch_bounds__(1024) norm_weights_kernel(int cols, int ctas, const float *__restrict__ part, int wide,
                                                            void *__restrict__ dweight, void *__restrict__ dbias) {
  __shared__ float sums[32][33];
  grid_chain_enter();
  const int tx = (int)threadIdx.x % 32, ty = (int)threadIdx.x / 32, c = (int)blockIdx.x * 32 + tx;
  float s = 0.f;
  if (c < 2 * cols)
    for (int i = ty; i < ctas; i += 32) s += part[(int64_t)i * 2 * cols + c];
  sums[ty][tx] = s;
  __syncthreads();
  s = sums[tx][ty];  // (a warp now holds one column's slices)
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  const int col = (int)blockIdx.x * 32 + ty;
  if (tx || col >= 2 * cols) return;
  void *to = col < cols ? dweight : dbias;
  const int at = col < cols ? col : col - cols;
  if (!to) return;
  if (wide) static_cast<float *>(to)[at] = s;
  else static_cast<__nv_bfloat16 *>(to)[at] = __float2bfloat16(s);
}

}  // namespace

// CTAs of the backward: as many as run at once, fewer while they would have no rows.
int backward_ctas(const Args &a) {
  int64_t n = 0;
  with_plan(a.groups, [&](auto plan) {
    using P = decltype(plan);
    const int64_t ctas = ((int64_t)a.rows + P::slots - 1) / P::slots, most = kSMs * (P::threads < 768 ? 768 / P::threads : 1);
    n = ctas < most ? ctas : most;
  });
  return (int)n;
}

}  // namespace rows
}  // namespace blossom

extern "C" size_t blossom_add_norm_workspace_bytes(const blossom_rows_params *params) {
  using namespace blossom;
  rows::Args a;
  static const int64_t any[2] = {0, 0};
  if (rows::check(params, rows::kMaxCols, any, &a)) return 0;
  const size_t bytes = (size_t)rows::backward_ctas(a) * 2 * a.cols * sizeof(float);
  return bytes < 256 ? 256 : (bytes + 255) / 256 * 256;
}

extern "C" int blossom_add_norm_bwd(const blossom_rows_params *params, const void *x, const void *residual,
                                    const void *weight, const int64_t *rng, const float *stats, const void *dout, void *dx,
                                    void *dresidual, void *dweight, void *dbias, void *workspace, size_t workspace_bytes,
                                    blossom_stream_t stream) {
  using namespace blossom;
  prof_break();
  rows::Args a;
  if (int rc = rows::check(params, rows::kMaxCols, rng, &a)) return rc;
  const cudaStream_t st = (cudaStream_t)stream;
  const size_t esz = params->dtype == BLOSSOM_DTYPE_FP32 ? 4 : 2, wsz = a.wide_weights ? 4 : 2;
  for (const void *p : {weight, (const void *)dweight, (const void *)dbias})
    if (reinterpret_cast<uintptr_t>(p) % wsz) return BLOSSOM_ERR_INVALID_ARG;
  if (a.rows == 0) {  // sums over no rows
    for (void *p : {dweight, dbias})
      if (p && cudaMemsetAsync(p, 0, (size_t)a.cols * wsz, st) != cudaSuccess) return BLOSSOM_ERR_CUDA;
    return BLOSSOM_OK;
  }
  if (!x || !stats || !dout || !(dx || dresidual || dweight || dbias)) return BLOSSOM_ERR_INVALID_ARG;
  for (const void *p : {x, residual, dout, (const void *)dx, (const void *)dresidual})
    if (reinterpret_cast<uintptr_t>(p) % esz) return BLOSSOM_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(stats) % 8) return BLOSSOM_ERR_INVALID_ARG;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 ||
      workspace_bytes < blossom_add_norm_workspace_bytes(params))
    return BLOSSOM_ERR_WORKSPACE;
  rows::Alignment al;
  al.rows_at(x, a.sx, esz);
  al.rows_at(residual, a.sr, esz);
  al.rows_at(dout, a.so, esz);
  al.rows_at(dx, a.sdx, esz);
  al.rows_at(dresidual, a.sdr, esz);
  const int ctas = rows::backward_ctas(a);
  float *part = dweight || dbias ? static_cast<float *>(workspace) : nullptr;
  rows::with_plan(a.groups, [&](auto plan) {
    using P = decltype(plan);
    rows::with_type(params->dtype, al.elements(a.cols, esz), [&](auto t, auto w) {
      using T = decltype(t);
      LaunchScope ls(K_NORM_BWD, st);
      launch_chained(rows::norm_bwd_kernel<T, decltype(w)::value, P>, dim3((unsigned)ctas), dim3(P::threads), 0, st, a,
                     static_cast<const T *>(x), static_cast<const T *>(residual), weight, rng,
                     reinterpret_cast<const float2 *>(stats), static_cast<const T *>(dout), static_cast<T *>(dx),
                     static_cast<T *>(dresidual), part);
    });
  });
  if (part) {
    LaunchScope ls(K_NORM_WEIGHTS, st);
    launch_chained(rows::norm_weights_kernel, dim3((unsigned)((2 * a.cols + 31) / 32)), dim3(1024), 0, st, a.cols, ctas,
                   (const float *)part, a.wide_weights, dweight, dbias);
  }
  return cudaGetLastError() == cudaSuccess ? BLOSSOM_OK : BLOSSOM_ERR_CUDA;
}
