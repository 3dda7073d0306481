// Layer norm of residual + dropout(x), forward: out = (z - mean) * rstd * weight + bias per row, z never stored.
//
// Bound: memory, x and residual once in and out once out, and the generator's and the norm's instructions.  32768 x 1024 bf16 with
// dropout: 201 MB in 36 us, 86 % of the rate of a copy, with a warp a row (with a CTA a row 46); 131072 x 64: 50 MB in 16 us.
// 12800 x 64: 5.4 us, one launch.
// A row stays in registers between the three steps (mean, then
// the sum of squared distances from it, then the output), so its variance is that of the definition without a
// second read and without the cancellation of E[z^2] - mean^2.
#include "rows.cuh"

namespace blossom {
namespace rows {
namespace {

// Rows that a thread has under way at a time: two narrow ones, or one.
template <typename P>
struct InFlight {
  static constexpr int rows = P::V == 1 ? 2 : 1;
};

// What a CTA has of its SM.
template <typename T, int W, typename P>
struct Shape {
  static constexpr int regs = P::V > 2 ? 128 : 80, resident = 65536 / regs / P::threads;
  static constexpr int weights = P::V > 1 ? P::TPR * P::V * 4 * (int)sizeof(float4) : 0;  // bytes
  static constexpr int fixed = 64;
  using Rows = Ring<2 * InFlight<P>::rows * P::V, P::threads>;
  // (not for narrow rows: 131072 x 64 18 us against 16, 12800 x 64 7.3 against 5.6; 32768 x 1024 38.5 against 41)
  static constexpr int stages = W == 8 && P::V > 1 ? Rows::stages(resident, weights + fixed) : 0;  // 0: rows in registers
  static constexpr int smem = weights + stages * Rows::kStage;
};

template <typename T, int W, typename P>
__global__ void __launch_bounds__(P::threads, Shape<T, W, P>::resident)
    norm_fwd_kernel(Args a, const T *__restrict__ x, const T *__restrict__ res, const void *__restrict__ weight,
                    const void *__restrict__ bias, const int64_t *__restrict__ rng, T *__restrict__ out,
                    float2 *__restrict__ stats) {
  // In bf16 the next rows are under way while these are worked on, wide ones by asynchronous copies; in fp32, twice the bytes a
  // column, they would take registers that the work needs.
  constexpr int STAGES = Shape<T, W, P>::stages;
  constexpr bool AHEAD = STAGES == 0 && sizeof(T) == 2;
  constexpr int TPR = P::TPR, V = P::V, U = InFlight<P>::rows, kGroups = TPR * V;
  __shared__ float buf[TPR > 32 ? TPR / 16 : 1];
  // weight and bias of wide rows: per group of columns two quarters of each, the groups side by side (so that a warp reads
  // consecutive addresses)
  extern __shared__ float4 wb[];  // [4][kGroups]
  grid_chain_enter();
  Generator gen;
  if (a.drop == 1) gen.read(rng);
  const int lane = (int)threadIdx.x % TPR, slot = (int)threadIdx.x / TPR;
  int turn = 0;
  Group w1, b1;
  if constexpr (V == 1) {
    w1 = load_weights(weight, a.wide_weights, 8 * lane, a.cols - 8 * lane, 1.f);
    b1 = load_weights(bias, a.wide_weights, 8 * lane, a.cols - 8 * lane, 0.f);
  } else {
    for (int g = (int)threadIdx.x; g < kGroups; g += P::threads) {
      const Group w = load_weights(weight, a.wide_weights, 8 * g, a.cols - 8 * g, 1.f);
      const Group b = load_weights(bias, a.wide_weights, 8 * g, a.cols - 8 * g, 0.f);
      wb[g] = make_float4(w.p[0].x, w.p[0].y, w.p[1].x, w.p[1].y);
      wb[kGroups + g] = make_float4(w.p[2].x, w.p[2].y, w.p[3].x, w.p[3].y);
      wb[2 * kGroups + g] = make_float4(b.p[0].x, b.p[0].y, b.p[1].x, b.p[1].y);
      wb[3 * kGroups + g] = make_float4(b.p[2].x, b.p[2].y, b.p[3].x, b.p[3].y);
    }
    __syncthreads();
  }
  const uint32_t rows = (uint32_t)a.rows, step = gridDim.x * (uint32_t)(P::slots * U);
  uint32_t row0 = blockIdx.x * (uint32_t)(P::slots * U) + (uint32_t)slot, left = blockIdx.x * (uint32_t)(P::slots * U);
  const T *px = x + row0 * a.sx + 8 * lane, *pr = (res ? res : x) + row0 * a.sr + 8 * lane;
  T *po = out + row0 * a.so + 8 * lane;
  Raw<T, W> xs[U][V], rs[U][V];
  const typename Shape<T, W, P>::Rows ring(wb + Shape<T, W, P>::weights / sizeof(float4));
  int stage = 0;
  auto load = [&](uint32_t row) {  // from px and pr, which go on to the next
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int valid = row + u * P::slots < rows ? a.cols - 8 * (lane + v * TPR) : 0;
        const T *x1 = px + u * P::slots * a.sx + 8 * v * TPR, *r1 = pr + u * P::slots * a.sr + 8 * v * TPR;
        if constexpr (STAGES > 0) {
          ring.copy(stage, 2 * (u * V + v), x1, a.drop < 2 && valid > 0);
          ring.copy(stage, 2 * (u * V + v) + 1, r1, res && valid > 0);
        } else {
          xs[u][v].load(x1, a.drop < 2 ? valid : 0);
          rs[u][v].load(r1, res ? valid : 0);
        }
      }
    if constexpr (STAGES > 0) {
      copies_end();
      stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    px += step * a.sx, pr += step * a.sr;
  };
  if (AHEAD) load(row0);
#pragma unroll 1
  for (int i = 0; i < STAGES; ++i) load(row0 + i * step);
  // (`left`, the CTA's first row, is the same for all of its threads: they meet in row_sum)
  for (; left < rows; left += step, row0 += step, po += step * a.so) {
    Group z[U][V];
    if constexpr (STAGES > 0) copies_wait<STAGES - 1>();
    else if (!AHEAD) load(row0);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        uint4 bits = make_uint4(0, 0, 0, 0);
        if (a.drop == 1) bits = gen.bits(a, (int)(row0 + u * P::slots), lane + v * TPR);
        if constexpr (STAGES > 0) {
          ring.get(stage, 2 * (u * V + v), xs[u][v]);
          ring.get(stage, 2 * (u * V + v) + 1, rs[u][v]);
        }
        z[u][v] = xs[u][v].get();
        if (a.drop == 1) drop(a, bits, z[u][v]);
        const Group r = rs[u][v].get();
#pragma unroll
        for (int i = 0; i < 4; ++i) z[u][v].p[i] = fma2(z[u][v].p[i], both(a.scale), r.p[i]);
      }
    if (STAGES > 0) load(row0 + STAGES * step);  // (into the stage that has just been read)
    else if (AHEAD) load(row0 + step);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float s = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) s += total(z[u][v].p);
      const float mean = row_sum<TPR>(s, buf, turn) * a.inv_cols;
      s = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Group m = spread<W>(-mean, a.cols - 8 * (lane + v * TPR));
        float2 sq[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          z[u][v].p[i] = add2(z[u][v].p[i], m.p[i]);
          sq[i] = mul2(z[u][v].p[i], z[u][v].p[i]);
        }
        s += total(sq);
      }
      const float rstd = rsqrtf(row_sum<TPR>(s, buf, turn) * a.inv_cols + a.eps);
      if (row0 + u * P::slots < rows) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int g = lane + v * TPR;
          Group w = w1, b = b1;
          if constexpr (V > 1) {
            const float4 q[4] = {wb[g], wb[kGroups + g], wb[2 * kGroups + g], wb[3 * kGroups + g]};
            w.p[0] = make_float2(q[0].x, q[0].y), w.p[1] = make_float2(q[0].z, q[0].w);
            w.p[2] = make_float2(q[1].x, q[1].y), w.p[3] = make_float2(q[1].z, q[1].w);
            b.p[0] = make_float2(q[2].x, q[2].y), b.p[1] = make_float2(q[2].z, q[2].w);
            b.p[2] = make_float2(q[3].x, q[3].y), b.p[3] = make_float2(q[3].z, q[3].w);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) z[u][v].p[i] = fma2(mul2(z[u][v].p[i], both(rstd)), w.p[i], b.p[i]);
          store_group<T, W>(po + u * P::slots * a.so + 8 * v * TPR, a.cols - 8 * g, z[u][v]);
        }
        if (stats && lane == 0) stats[row0 + u * P::slots] = make_float2(mean, rstd);
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
  if (!residual) a.sr = a.sx;  // (a copy of no bytes needs an aligned address as well: x's)
  al.rows_at(residual, a.sr, esz);
  al.rows_at(out, a.so, esz);
  bool ok = true;
  auto launch = [&](auto plan) {
    using P = decltype(plan);
    rows::with_type(params->dtype, al.elements(a.cols, esz), [&](auto t, auto w) {
      using T = decltype(t);
      if constexpr (P::V <= (sizeof(T) == 2 ? 4 : 2)) {
        const auto kern = rows::norm_fwd_kernel<T, decltype(w)::value, P>;
        const int64_t per = P::slots * rows::InFlight<P>::rows, ctas = (a.rows + per - 1) / per;
        using S = rows::Shape<T, decltype(w)::value, P>;
        const int64_t most = rows::kSMs * S::resident;  // (as many as run at once)
        ok = rows::allow_stages(kern, S::smem, S::fixed);
        if (S::stages) rows::prefer_shared(kern);
        if (!ok) return;
        LaunchScope ls(K_NORM_FWD, (cudaStream_t)stream);
        launch_chained(kern, dim3((unsigned)(ctas < most ? ctas : most)), dim3(P::threads), S::smem, (cudaStream_t)stream, a,
                       static_cast<const T *>(x), static_cast<const T *>(residual), weight, bias, rng,
                       static_cast<T *>(out), reinterpret_cast<float2 *>(stats));
      }
    });
  };
  // (half the bytes a column in bf16: twice the columns a thread for as much under way)
  if (esz == 2) rows::with_plan<4>(a.groups, launch);
  else rows::with_plan<2>(a.groups, launch);
  if (!ok) return BLOSSOM_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? BLOSSOM_OK : BLOSSOM_ERR_CUDA;
}
