// Layer norm of residual + dropout(x), backward, with the reduction of the weight's and the bias's gradient.
//
// With a = dout * weight and n = (z - mean) * rstd:  dz = rstd * (a - mean(a) - n * mean(a n)), dresidual = dz,
// dx = dz where the dropout kept, scaled; dweight = sum over rows of dout n, dbias = sum over rows of dout.
// z and the mask are formed again: reading x and residual moves the bytes that a stored z would, and z is not rounded.
//
// Bound: memory, three tensors in and two out.  32768 x 1024 bf16 with dropout: 336 MB in 66 us, 79 % of the rate of a copy;
// 131072 x 64: 84 MB in 20 us.  128 registers leave 16 warps an SM for it (20 and 24 in fewer spill: 85 and 79 us), the rows to
// come are in shared memory.
// Each thread owns its columns for all rows of its CTA, so the column
// sums stay in registers; a CTA leaves one partial sum a column, and a second kernel adds the CTAs up in a fixed order.
#include "rows.cuh"

namespace blossom {
namespace rows {
namespace {

// What a CTA has of its SM.
template <typename P>
constexpr int resident = 65536 / (P::V > 1 ? 128 : 96) / P::threads;
template <typename T, int W, typename P>
struct Shape {
  using Rows = Ring<3 * P::V, P::threads>;
  static constexpr int fixed = (P::V > 1 ? P::TPR * P::V * 32 : 0) + (P::TPR <= 32 ? P::TPR * P::V * 64 : 0) + 128;  // bytes
  static constexpr int stages = W == 8 ? Rows::stages(resident<P>, fixed) : 0;  // 0: rows in registers
  static constexpr int smem = stages * Rows::kStage;
};

template <typename T, int W, typename P>
__global__ void __launch_bounds__(P::threads, resident<P>)
    norm_bwd_kernel(Args a, const T *__restrict__ x, const T *__restrict__ res, const void *__restrict__ weight,
                    const int64_t *__restrict__ rng, const float2 *__restrict__ stats, const T *__restrict__ dout,
                    T *__restrict__ dx, T *__restrict__ dres, float *__restrict__ part) {
  constexpr int STAGES = Shape<T, W, P>::stages;
  // The next rows are under way while this one is worked on (see the forward): by asynchronous copies 33.5 M elements in rows
  // of 64, 256, 1024, 4096 take 65, 63, 69, 73 us, with the next row in registers 76, 79, 69, 85.
  constexpr bool AHEAD = STAGES == 0 && sizeof(T) == 2;
  constexpr int TPR = P::TPR, V = P::V, kGroups = TPR * V;
  __shared__ float2 buf[TPR > 32 ? TPR / 16 : 1];
  __shared__ float2 sums[TPR <= 32 ? TPR * V * 8 : 1];
  __shared__ float4 ws[V > 1 ? 2 * kGroups : 1];  // the weights of wide rows, two quarters a group, the groups side by side
  extern __shared__ float4 stages[];
  grid_chain_enter();
  Generator gen;
  if (a.drop == 1) gen.read(rng);
  const int lane = (int)threadIdx.x % TPR, slot = (int)threadIdx.x / TPR;
  int turn = 0;
  Group w1, gw[V], gb[V];
  if constexpr (V == 1) {
    w1 = load_weights(weight, a.wide_weights, 8 * lane, a.cols - 8 * lane, 1.f);
  } else {
    for (int g = (int)threadIdx.x; g < kGroups; g += P::threads) {
      const Group w = load_weights(weight, a.wide_weights, 8 * g, a.cols - 8 * g, 1.f);
      ws[g] = make_float4(w.p[0].x, w.p[0].y, w.p[1].x, w.p[1].y);
      ws[kGroups + g] = make_float4(w.p[2].x, w.p[2].y, w.p[3].x, w.p[3].y);
    }
    __syncthreads();
  }
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int i = 0; i < 4; ++i) gw[v].p[i] = gb[v].p[i] = both(0.f);
  const uint32_t rows = (uint32_t)a.rows, step = gridDim.x * (uint32_t)P::slots;
  uint32_t left = blockIdx.x * (uint32_t)P::slots, row = left + (uint32_t)slot;
  const T *px = x + row * a.sx + 8 * lane, *pr = (res ? res : x) + row * a.sr + 8 * lane, *pd = dout + row * a.so + 8 * lane;
  T *pdx = dx + row * a.sdx + 8 * lane, *pdr = dres + row * a.sdr + 8 * lane;
  Raw<T, W> xs[V], rs[V], ds[V];
  const typename Shape<T, W, P>::Rows ring(stages);
  int stage = 0;
  auto stats_of = [&](uint32_t row) { return row < rows ? stats[row] : both(0.f); };
  auto load = [&](uint32_t row) {  // from px, pr and pd, which go on to the next
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int valid = row < rows ? a.cols - 8 * (lane + v * TPR) : 0;
      const T *x1 = px + 8 * v * TPR, *r1 = pr + 8 * v * TPR, *d1 = pd + 8 * v * TPR;
      if constexpr (STAGES > 0) {
        ring.copy(stage, 3 * v, x1, a.drop < 2 && valid > 0);
        ring.copy(stage, 3 * v + 1, r1, res && valid > 0);
        ring.copy(stage, 3 * v + 2, d1, valid > 0);
      } else {
        xs[v].load(x1, a.drop < 2 ? valid : 0);
        rs[v].load(r1, res ? valid : 0);
        ds[v].load(d1, valid);
      }
    }
    if constexpr (STAGES > 0) {
      copies_end();
      stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    px += step * a.sx, pr += step * a.sr, pd += step * a.so;
  };
  if (AHEAD) load(row);
#pragma unroll 1
  for (int i = 0; i < STAGES; ++i) load(row + i * step);
  float2 next_stats = stats_of(row);
  // (`left`, the CTA's first row, is the same for all of its threads: they meet in row_sum)
  for (; left < rows; left += step, row += step, pdx += step * a.sdx, pdr += step * a.sdr) {
    if constexpr (STAGES > 0) copies_wait<STAGES - 1>();
    else if (!AHEAD) load(row);
    const float2 st = next_stats;
    next_stats = stats_of(row + step);
    Group z[V], d[V];
    uint4 bits[V];
    float2 s = both(0.f);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      bits[v] = make_uint4(0, 0, 0, 0);
      if (a.drop == 1) bits[v] = gen.bits(a, (int)row, lane + v * TPR);
      if constexpr (STAGES > 0) {
        ring.get(stage, 3 * v, xs[v]);
        ring.get(stage, 3 * v + 1, rs[v]);
        ring.get(stage, 3 * v + 2, ds[v]);
      }
      z[v] = xs[v].get();
      d[v] = ds[v].get();
      if (a.drop == 1) drop(a, bits[v], z[v]);
      const Group r = rs[v].get();
#pragma unroll
      for (int i = 0; i < 4; ++i) z[v].p[i] = fma2(z[v].p[i], both(a.scale), r.p[i]);
    }
    if (STAGES > 0) load(row + STAGES * step);  // (into the stage that has just been read)
    else if (AHEAD) load(row + step);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const Group m = spread<W>(-st.x, a.cols - 8 * (lane + v * TPR));
      Group w = w1;
      if constexpr (V > 1) {
        const float4 q0 = ws[lane + v * TPR], q1 = ws[kGroups + lane + v * TPR];
        w.p[0] = make_float2(q0.x, q0.y), w.p[1] = make_float2(q0.z, q0.w);
        w.p[2] = make_float2(q1.x, q1.y), w.p[3] = make_float2(q1.z, q1.w);
      }
      float2 s2[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // n; 0 in rows and columns that are not there, like d
        z[v].p[i] = mul2(add2(z[v].p[i], m.p[i]), both(st.y));
        gw[v].p[i] = fma2(d[v].p[i], z[v].p[i], gw[v].p[i]);
        gb[v].p[i] = add2(d[v].p[i], gb[v].p[i]);
        d[v].p[i] = mul2(d[v].p[i], w.p[i]);  // a
        s2[i] = mul2(d[v].p[i], z[v].p[i]);
      }
      s = add2(s, make_float2(total(d[v].p), total(s2)));
    }
    s = row_sum<TPR>(s, buf, turn);
    if (row >= rows) continue;
    const float2 c1 = both(-s.x * a.inv_cols), c2 = both(-s.y * a.inv_cols);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int valid = a.cols - 8 * (lane + v * TPR);
#pragma unroll
      for (int i = 0; i < 4; ++i) d[v].p[i] = mul2(fma2(z[v].p[i], c2, add2(d[v].p[i], c1)), both(st.y));
      if (dres) store_group<T, W>(pdr + 8 * v * TPR, valid, d[v]);
      if (dx) {
        if (a.drop) {
          if (a.drop == 1) drop(a, bits[v], d[v]);
#pragma unroll
          for (int i = 0; i < 4; ++i) d[v].p[i] = a.drop == 1 ? mul2(d[v].p[i], both(a.scale)) : both(0.f);
        }
        store_group<T, W>(pdx + 8 * v * TPR, valid, d[v]);
      }
    }
  }
  if (!part) return;
  float *mine = part + (int64_t)blockIdx.x * 2 * a.cols;
  if constexpr (TPR <= 32) {
    // over the groups of threads of a warp, which hold the same columns, then warp by warp
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int o = TPR; o < 32; o <<= 1) {
          gw[v].at(j) = exchange_add(gw[v].at(j), o);
          gb[v].at(j) = exchange_add(gb[v].at(j), o);
        }
    for (int warp = 0; warp < P::threads / 32; ++warp) {
      if ((int)threadIdx.x / 32 == warp && (int)threadIdx.x % 32 < TPR) {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float2 &p = sums[8 * (lane + v * TPR) + j];
            p = warp ? make_float2(p.x + gw[v].at(j), p.y + gb[v].at(j)) : make_float2(gw[v].at(j), gb[v].at(j));
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
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int c = 8 * (lane + v * TPR) + j;
        if (c < a.cols) mine[c] = gw[v].at(j), mine[a.cols + c] = gb[v].at(j);
      }
  }
}

// dweight and dbias from the CTAs' partial sums: 16 columns and 32 slices of the CTAs a block, 8 loads in flight a thread.
// Bound: latency of a few dependent loads (1184 x 2048 sums, 9.7 MB: 6 us behind the backward).
// SHARED: behind a backward that asked for all of an SM's shared memory (prefer_shared).  A function keeps that request from call
// to call; with a kernel of their own the narrow rows' launches do not depend on whether a wide call came before.
constexpr int kSumCols = 16, kSumSlices = 32;
template <bool SHARED>
__global__ void __launch_bounds__(kSumCols *kSumSlices) norm_weights_kernel(int cols, int ctas, const float *__restrict__ part,
                                                                            int wide, void *__restrict__ dweight,
                                                                            void *__restrict__ dbias) {
  __shared__ float sums[kSumSlices][kSumCols + 1];
  grid_chain_enter();
  const int tx = (int)threadIdx.x % kSumCols, ty = (int)threadIdx.x / kSumCols, c = (int)blockIdx.x * kSumCols + tx;
  float s = 0.f;
  if (c < 2 * cols)
    for (int i0 = ty; i0 < ctas; i0 += 8 * kSumSlices) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int i = i0 + k * kSumSlices;
        v[k] = i < ctas ? part[(int64_t)i * 2 * cols + c] : 0.f;
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) s += v[k];
    }
  sums[ty][tx] = s;
  __syncthreads();
  const int lane = (int)threadIdx.x % 32, warp = (int)threadIdx.x / 32;  // a warp a column
  s = sums[lane][warp];
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  const int col = (int)blockIdx.x * kSumCols + warp;
  if (lane || col >= 2 * cols) return;
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
  with_plan<2>(a.groups, [&](auto plan) {
    using P = decltype(plan);
    const int64_t ctas = ((int64_t)a.rows + P::slots - 1) / P::slots;
    const int64_t most = kSMs * resident<P>;  // (as the kernel's bounds say)
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
  if ((dweight || dbias) && (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 ||
                             workspace_bytes < blossom_add_norm_workspace_bytes(params)))
    return BLOSSOM_ERR_WORKSPACE;
  rows::Alignment al;
  al.rows_at(x, a.sx, esz);
  if (!residual) a.sr = a.sx;  // (a copy of no bytes needs an aligned address as well: x's)
  al.rows_at(residual, a.sr, esz);
  al.rows_at(dout, a.so, esz);
  al.rows_at(dx, a.sdx, esz);
  al.rows_at(dresidual, a.sdr, esz);
  const int ctas = rows::backward_ctas(a);
  float *part = dweight || dbias ? static_cast<float *>(workspace) : nullptr;
  bool ok = true, wide = false;
  rows::with_plan<2>(a.groups, [&](auto plan) {
    using P = decltype(plan);
    rows::with_type(params->dtype, al.elements(a.cols, esz), [&](auto t, auto w) {
      using T = decltype(t);
      const auto kern = rows::norm_bwd_kernel<T, decltype(w)::value, P>;
      using S = rows::Shape<T, decltype(w)::value, P>;
      ok = rows::allow_stages(kern, S::smem, S::fixed);
      wide = S::stages > 0 && P::V > 1;
      if (wide) rows::prefer_shared(kern);
      if (!ok) return;
      LaunchScope ls(K_NORM_BWD, st);
      launch_chained(kern, dim3((unsigned)ctas), dim3(P::threads), S::smem, st, a,
                     static_cast<const T *>(x), static_cast<const T *>(residual), weight, rng,
                     reinterpret_cast<const float2 *>(stats), static_cast<const T *>(dout), static_cast<T *>(dx),
                     static_cast<T *>(dresidual), part);
    });
  });
  if (!ok) return BLOSSOM_ERR_CUDA;
  if (part) {
    const auto kern = wide ? rows::norm_weights_kernel<true> : rows::norm_weights_kernel<false>;
    if (wide) rows::prefer_shared(kern);
    LaunchScope ls(K_NORM_WEIGHTS, st);
    launch_chained(kern, dim3((unsigned)((2 * a.cols + rows::kSumCols - 1) / rows::kSumCols)),
                   dim3(rows::kSumCols * rows::kSumSlices), 0, st, a.cols, ctas,
                   (const float *)part, a.wide_weights, dweight, dbias);
  }
  return cudaGetLastError() == cudaSuccess ? BLOSSOM_OK : BLOSSOM_ERR_CUDA;
}
