// Dropout from a counter-based generator: out = kept ? x * scale : 0, the mask a function of (seed, step, site, row,
// column) that nobody stores.  The backward is the same kernel on the upstream gradient.
//
// Bound: memory, each element once in and once out.
#include "rows.cuh"

namespace blossom {
namespace rows {

// Shared by the entry points of this file and of the layer norm: what is wrong with the params, or the kernels' arguments.
int check(const blossom_rows_params *p, int max_cols, const int64_t *rng, Args *a) {
  if (!p || p->rows < 0 || p->cols < 1) return BLOSSOM_ERR_INVALID_ARG;
  for (int t : {p->dtype, p->weight_dtype})
    if (t != BLOSSOM_DTYPE_FP32 && t != BLOSSOM_DTYPE_BF16) return BLOSSOM_ERR_INVALID_ARG;
  if (p->site < 0 || p->site > 65535) return BLOSSOM_ERR_INVALID_ARG;
  if (!(p->dropout >= 0.0 && p->dropout <= 1.0) || !(p->eps >= 0.0) || isinf(p->eps)) return BLOSSOM_ERR_INVALID_ARG;
  int64_t st[5] = {p->x_stride, p->residual_stride, p->out_stride, p->dx_stride, p->dresidual_stride};
  for (int64_t &s : st) {
    if (s == 0) s = p->cols;
    if (s < p->cols) return BLOSSOM_ERR_INVALID_ARG;
  }
  if (p->rows > 0x7fffffffLL || p->cols > max_cols) return BLOSSOM_ERR_UNSUPPORTED;
  if (p->dropout > 0.0 && (!rng || reinterpret_cast<uintptr_t>(rng) % 8)) return BLOSSOM_ERR_INVALID_ARG;
  a->rows = (int)p->rows;
  a->cols = p->cols;
  a->groups = (p->cols + 7) / 8;
  a->sx = st[0], a->sr = st[1], a->so = st[2], a->sdx = st[3], a->sdr = st[4];
  a->bar = (unsigned)floor(p->dropout * 65536.0 + 0.5);
  a->site = (unsigned)p->site;
  a->scale = a->bar < 65536u ? (float)(65536.0 / (65536.0 - a->bar)) : 0.f;
  a->eps = (float)p->eps;
  a->inv_cols = 1.f / (float)p->cols;
  a->wide_weights = p->weight_dtype == BLOSSOM_DTYPE_FP32;
  return BLOSSOM_OK;
}

namespace {

constexpr int kThreads = 256;

// A thread takes groups of 8 columns, one after another, in the order of the rows.
template <typename T, int W>
__global__ void __launch_bounds__(kThreads) dropout_kernel(Args a, const T *x, const int64_t *rng, T *out) {
  grid_chain_enter();
  Generator gen;
  if (a.bar) gen.read(rng);
  const int64_t total = (int64_t)a.rows * a.groups, step = (int64_t)gridDim.x * kThreads;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += step) {
    const int row = (int)(i / a.groups), g = (int)(i - (int64_t)row * a.groups), valid = a.cols - 8 * g;
    float v[8];
    load_group<T, W>(x + row * a.sx + 8 * g, valid, v);
    if (a.bar) {
      const uint32_t m = gen.kept(a, row, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = m >> j & 1 ? v[j] * a.scale : 0.f;
    }
    store_group<T, W>(out + row * a.so + 8 * g, valid, v);
  }
}

}  // namespace
}  // namespace rows
}  // namespace blossom

extern "C" int blossom_dropout(const blossom_rows_params *params, const void *x, const int64_t *rng, void *out,
                               blossom_stream_t stream) {
  using namespace blossom;
  prof_break();
  rows::Args a;
  if (int rc = rows::check(params, rows::kMaxCols, rng, &a)) return rc;
  if (a.rows == 0) return BLOSSOM_OK;
  const size_t esz = params->dtype == BLOSSOM_DTYPE_FP32 ? 4 : 2;
  if (!x || !out || reinterpret_cast<uintptr_t>(x) % esz || reinterpret_cast<uintptr_t>(out) % esz)
    return BLOSSOM_ERR_INVALID_ARG;
  rows::Alignment al;
  al.rows_at(x, a.sx, esz);
  al.rows_at(out, a.so, esz);
  const int64_t ctas = ((int64_t)a.rows * a.groups + rows::kThreads - 1) / rows::kThreads, most = rows::kSMs * 8;
  rows::with_type(params->dtype, al.elements(a.cols, esz), [&](auto t, auto w) {
    using T = decltype(t);
    LaunchScope ls(K_DROPOUT, (cudaStream_t)stream);
    launch_chained(rows::dropout_kernel<T, decltype(w)::value>, dim3((unsigned)(ctas < most ? ctas : most)),
                   dim3(rows::kThreads), 0, (cudaStream_t)stream, a, static_cast<const T *>(x), rng, static_cast<T *>(out));
  });
  return cudaGetLastError() == cudaSuccess ? BLOSSOM_OK : BLOSSOM_ERR_CUDA;
}
