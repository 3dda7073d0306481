// Dropout from a counter-based generator: out = kept ? x * scale : 0, the mask a function of (seed, step, site, row,
// column) that nobody stores.  The backward is the same kernel on the upstream gradient.
//
// Bound: memory, each element once in and once out, and the generator's instructions.  131072 x 64 bf16 is 33.6 MB a call, 5.2 us at
// the rate of a copy, and takes 12 us alone; 32768 x 1024 134 MB, 21 us, takes 27; in fp32 53 of 42.  Through autograd a forward
// and a backward of the former take 49 us: that is the host's part of it.  The groups of threads are as narrow as the row, so
// that a row of 64 keeps 8 threads and none idles.
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
  const double bar = floor(p->dropout * 65536.0 + 0.5);  // of 65536
  a->drop = bar == 0.0 ? 0 : bar < 65536.0 ? 1 : 2;
  a->bar = a->drop == 1 ? (unsigned)bar << 16 : 0;
  a->site = (unsigned)p->site;
  a->scale = a->drop == 0 ? 1.f : a->drop == 1 ? (float)(65536.0 / (65536.0 - bar)) : 0.f;
  a->eps = (float)p->eps;
  a->inv_cols = 1.f / (float)p->cols;
  a->wide_weights = p->weight_dtype == BLOSSOM_DTYPE_FP32;
  return BLOSSOM_OK;
}

namespace {

// A kept element times the scale, subnormal ones too: this build's arithmetic would take them for zeros.
__device__ __forceinline__ float2 scaled(float2 x, float scale) {
  const float2 s = both(scale);
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(d)
      : "l"(*reinterpret_cast<const uint64_t *>(&x)), "l"(*reinterpret_cast<const uint64_t *>(&s)));
  return *reinterpret_cast<float2 *>(&d);
}

// Rows a thread loads before it works on the first (131072 x 64, 524288 x 64 in bf16 one 11.8, 30.5 us, two 13.7, 32.5; 32768 x
// 1024 28.7, 27.0; in fp32 18.1, 57.1 and 16.1, 52.7).
template <typename T, typename P>
constexpr int kRowsInFlight = sizeof(T) == 2 && P::V == 1 ? 1 : 2;

template <typename T, int W, typename P>
__global__ void __launch_bounds__(P::threads) dropout_kernel(Args a, const T *x, const int64_t *rng, T *out) {
  constexpr int U = kRowsInFlight<T, P>, V = P::V;
  grid_chain_enter();
  Generator gen;
  if (a.drop == 1) gen.read(rng);
  const int lane = (int)threadIdx.x % P::TPR;
  const uint32_t rows = (uint32_t)a.rows, step = gridDim.x * (uint32_t)P::slots;
  uint32_t row = blockIdx.x * (uint32_t)P::slots + threadIdx.x / P::TPR;
  const T *px = x + row * a.sx + 8 * lane;
  T *po = out + row * a.so + 8 * lane;
  for (; row < rows; row += U * step, px += U * step * a.sx, po += U * step * a.so) {
    Raw<T, W> v[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int k = 0; k < V; ++k)
        v[u][k].load(px + u * step * a.sx + 8 * k * P::TPR, row + u * step < rows ? a.cols - 8 * (lane + k * P::TPR) : 0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (row + u * step >= rows) break;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int g = lane + k * P::TPR;
        Group z = v[u][k].get();
        if (a.drop) {
          if (a.drop == 1) drop(a, gen.bits(a, (int)(row + u * step), g), z);
#pragma unroll
          for (int i = 0; i < 4; ++i) z.p[i] = a.drop == 1 ? scaled(z.p[i], a.scale) : both(0.f);
        }
        store_group<T, W>(po + u * step * a.so + 8 * k * P::TPR, a.cols - 8 * g, z);
      }
    }
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
  rows::with_plan<2>(a.groups, [&](auto plan) {
    using P = decltype(plan);
    rows::with_type(params->dtype, al.elements(a.cols, esz), [&](auto t, auto w) {
      using T = decltype(t);
      const int64_t per = P::slots * rows::kRowsInFlight<T, P>, ctas = (a.rows + per - 1) / per;
      const int64_t most = rows::kSMs * (2048 / P::threads);
      LaunchScope ls(K_DROPOUT, (cudaStream_t)stream);
      launch_chained(rows::dropout_kernel<T, decltype(w)::value, P>, dim3((unsigned)(ctas < most ? ctas : most)),
                     dim3(P::threads), 0, (cudaStream_t)stream, a, static_cast<const T *>(x), rng, static_cast<T *>(out));
    });
  });
  return cudaGetLastError() == cudaSuccess ? BLOSSOM_OK : BLOSSOM_ERR_CUDA;
}
