// A linear layer on few rows (the last positions of one or a few users): the CUDA cores, in single precision.
//
// Bound: the weight, read once for all rows (written once for dweight), and the latency of a few launches; tiles of 128 rows
// would be mostly empty and leave most SMs without one.  1 x 64 -> 256 2.4 us, 1 x 1024 -> 4096 4.1 us in bf16 (8 MB of weight).
//   forward  a warp takes kColumns outs and a share of k: its lanes run along the weight's rows, 8 numbers each, and add up the sums
//            of all rows; warps of a block that share a column's k meet in shared memory
//   dx       a thread has 4 columns and all rows, a block a share of the outs; the shares' sums are added up behind it
//   dweight  a thread has 4 columns of all rows of x in registers and goes down the outs
#include "linear.cuh"

namespace blossom {
namespace linear {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

template <typename T, int W>
__device__ __forceinline__ void load8(float (&v)[8], const T *p, int valid) {
  rows::Raw<T, W> x;
  x.load(p, valid);
  const rows::Group g = x.get();
#pragma unroll
  for (int i = 0; i < 4; ++i) v[2 * i] = g.p[i].x, v[2 * i + 1] = g.p[i].y;
}
__device__ __forceinline__ float load1(const float *p) { return *p; }
__device__ __forceinline__ float load1(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store1(float *p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16 *p, float v) { *p = __float2bfloat16(v); }

// Sums over the lanes of N numbers (a power of two): lane l is left with those of l, l + 32, ... in v[0], v[1], ...
template <int N>
__device__ __forceinline__ void scatter_sums(float (&v)[N]) {
  const int lane = (int)threadIdx.x & 31;
  int left = N;
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) {
    const bool up = lane & o;
    if (left > 1 && N >= 2) {
      const int half = left / 2;
#pragma unroll
      for (int i = 0; i < N / 2; ++i)
        if (i < half) {
          const float keep = up ? v[i + half] : v[i], give = up ? v[i] : v[i + half];
          v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
      left = half;
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    }
  }
}
// which number of N that is (halves by the lane's bits from the highest on)
template <int N>
__device__ __forceinline__ int scattered(int i) {
  const int lane = (int)threadIdx.x & 31;
  int at = 0, left = N;
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1)
    if (left > 1) {
      left /= 2;
      at += lane & o ? left : 0;
    }
  return at + i;
}

// out = act(x W^T + bias) + extra, or (SLOPE) extra * act'(x W^T + bias) in single precision.  R: rows at most.
template <typename T, int R, int W, bool SLOPE>
__global__ void __launch_bounds__(kThreads) few_rows_kernel(int rows, int cols, int outs, int wk, const T *x, int64_t ldx, const T *weight,
                                                            int64_t ldw, const T *bias, const T *extra, int64_t ld_extra, int act, void *out,
                                                            int64_t ld_out, int32_t *status) {
  constexpr int C = R <= 4 ? 4 : 2, N = C * R, LEFT = N > 32 ? N / 32 : 1;
  __shared__ float sums[kWarps][N];
  grid_chain_enter();
  x = behind_wait(x), weight = behind_wait(weight), bias = behind_wait(bias), extra = behind_wait(extra);
  if (status && blockIdx.x == 0 && threadIdx.x < 8) status[threadIdx.x] = 0;
  const int warp = (int)threadIdx.x / 32, lane = (int)threadIdx.x % 32, part = warp % wk, group = warp / wk;
  const int per = kWarps / wk, n0 = (blockIdx.x * per + group) * C;
  float v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = 0.f;
  for (int k = 8 * (part * 32 + lane); k < cols; k += 256 * wk) {
    float w[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) load8<T, W>(w[c], weight + (int64_t)(n0 + c < outs ? n0 + c : 0) * ldw + k, n0 + c < outs ? cols - k : 0);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float y[8];
      load8<T, W>(y, x + (int64_t)(r < rows ? r : 0) * ldx + k, r < rows ? cols - k : 0);
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c * R + r] = fmaf(y[i], w[c][i], v[c * R + r]);
    }
  }
  scatter_sums<N>(v);
#pragma unroll
  for (int i = 0; i < LEFT; ++i) {
    const int at = scattered<N>(i);
    sums[warp][at] = v[i];  // (lanes with the same number have the same sum)
  }
  __syncthreads();
  for (int i = (int)threadIdx.x; i < per * N; i += kThreads) {
    const int g = i / N, at = i % N, r = at % R, c = (blockIdx.x * per + g) * C + at / R;
    if (r >= rows || c >= outs) continue;
    float y = 0.f;
    for (int p = 0; p < wk; ++p) y += sums[g * wk + p][at];
    if (bias) y += load1(bias + c);
    const float e = extra ? load1(extra + (int64_t)r * ld_extra + c) : 0.f;
    with_curve(act, SLOPE, extra != nullptr, [&](auto a, auto slope, auto) {
      const Curve<decltype(a)::value, decltype(slope)::value, sizeof(T) == 4> curve;
      y = curve(make_float2(y, 0.f)).x;
    });
    if (SLOPE) static_cast<float *>(out)[(int64_t)r * ld_out + c] = y * e;
    else store1(static_cast<T *>(out) + (int64_t)r * ld_out + c, y + e);
  }
}

// part[share][r][k] = sum over the share's outs of g[r][n] weight[n][k]
template <typename T, typename G, int R, int W>
__global__ void __launch_bounds__(kThreads) few_dx_kernel(int rows, int cols, int outs, int per, const G *g, int64_t ldg, const T *weight,
                                                          int64_t ldw, float *part, int32_t *status) {
  constexpr int kDeep = 32;
  __shared__ float tile[kDeep][R];
  grid_chain_enter();
  if (status && blockIdx.x + blockIdx.y == 0 && threadIdx.x < 8) status[threadIdx.x] = 0;
  g = behind_wait(g), weight = behind_wait(weight);
  const int k = 4 * (blockIdx.x * kThreads + (int)threadIdx.x), n0 = blockIdx.y * per, n1 = min(n0 + per, outs);
  float2 acc[R][2];
#pragma unroll
  for (int r = 0; r < R; ++r) acc[r][0] = acc[r][1] = make_float2(0.f, 0.f);
  for (int n = n0; n < n1; n += kDeep) {
    __syncthreads();
    for (int i = (int)threadIdx.x; i < kDeep * R; i += kThreads) {
      const int d = i % kDeep, r = i / kDeep;
      tile[d][r] = n + d < n1 && r < rows ? load1(g + (int64_t)r * ldg + n + d) : 0.f;
    }
    __syncthreads();
    if (k < cols) {
#pragma unroll 8
      for (int d = 0; d < min(kDeep, n1 - n); ++d) {
        const T *p = weight + (int64_t)(n + d) * ldw + k;
        float w[4];
        if constexpr (W >= 4) {
          const float4 q = ld4(p);
          w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = k + i < cols ? load1(p + i) : 0.f;
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float2 s = make_float2(tile[d][r], tile[d][r]);
          acc[r][0] = fma2(s, make_float2(w[0], w[1]), acc[r][0]);
          acc[r][1] = fma2(s, make_float2(w[2], w[3]), acc[r][1]);
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (r >= rows) break;
    const float v[4] = {acc[r][0].x, acc[r][0].y, acc[r][1].x, acc[r][1].y};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (k + i < cols) part[((int64_t)blockIdx.y * rows + r) * cols + k + i] = v[i];
  }
}

// dweight[n][k] = sum_r g[r][n] x[r][k], dbias[n] = sum_r g[r][n]; either may be null.  `per` outs a block
template <typename T, typename G, int R, int W>
__global__ void __launch_bounds__(kThreads) few_dweight_kernel(int rows, int cols, int outs, int per, const G *g, int64_t ldg, const T *x,
                                                               int64_t ldx, T *dweight, int64_t ld, T *dbias, int32_t *status) {
  constexpr int kDeep = 32;
  __shared__ float tile[kDeep][R];
  grid_chain_enter();
  if (status && blockIdx.x + blockIdx.y == 0 && threadIdx.x < 8) status[threadIdx.x] = 0;
  g = behind_wait(g), x = behind_wait(x);
  const int k = 4 * (blockIdx.x * kThreads + (int)threadIdx.x), n0 = blockIdx.y * per, n1 = min(n0 + per, outs);
  float2 v[R][2];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float y[4] = {0.f, 0.f, 0.f, 0.f};
    if (dweight && r < rows) {
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = k + i < cols ? load1(x + (int64_t)r * ldx + k + i) : 0.f;
    }
    v[r][0] = make_float2(y[0], y[1]), v[r][1] = make_float2(y[2], y[3]);
  }
  for (int n = n0; n < n1; n += kDeep) {
    __syncthreads();
    for (int i = (int)threadIdx.x; i < kDeep * R; i += kThreads) {
      const int d = i % kDeep, r = i / kDeep;
      tile[d][r] = n + d < n1 && r < rows ? load1(g + (int64_t)r * ldg + n + d) : 0.f;
    }
    __syncthreads();
    if (dbias && blockIdx.x == 0 && (int)threadIdx.x < min(kDeep, n1 - n)) {
      float s = 0.f;
#pragma unroll
      for (int r = 0; r < R; ++r) s += tile[threadIdx.x][r];
      store1(dbias + n + threadIdx.x, s);
    }
    if (!dweight || k >= cols) continue;
    for (int d = 0; d < min(kDeep, n1 - n); ++d) {
      float2 s[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float2 q = make_float2(tile[d][r], tile[d][r]);
        s[0] = fma2(q, v[r][0], s[0]);
        s[1] = fma2(q, v[r][1], s[1]);
      }
      T *const to = dweight + (int64_t)(n + d) * ld + k;
      if constexpr (W >= 4) {
        st4(to, make_float4(s[0].x, s[0].y, s[1].x, s[1].y));
      } else {
        const float o[4] = {s[0].x, s[0].y, s[1].x, s[1].y};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (k + i < cols) store1(to + i, o[i]);
      }
    }
  }
}

// f(T, R): type and rows at most
template <typename F>
void with_rows(int dtype, int rows, F &&f) {
  using std::integral_constant;
  auto typed = [&](auto t) {
    if (rows <= 1) f(t, integral_constant<int, 1>());
    else if (rows <= 4) f(t, integral_constant<int, 4>());
    else if (rows <= 8) f(t, integral_constant<int, 8>());
    else f(t, integral_constant<int, 16>());
  };
  if (dtype == BLOSSOM_DTYPE_FP32) typed(float());
  else typed(__nv_bfloat16());
}

}  // namespace

// Shares of the outs for dx: a block an SM, eight outs a share at least.
int few_shares(int cols, int outs) {
  const int blocks = (cols + 4 * kThreads - 1) / (4 * kThreads), most = (outs + 7) / 8;
  int s = kSMs / blocks;
  s = s < most ? s : most;
  if (s < 1) return 1;
  const int per = (outs + s - 1) / s;
  return (outs + per - 1) / per;  // (none empty)
}

int launch_few_forward(const FewRows &f, bool slope, const void *extra, int64_t ld_extra, void *out, int64_t ld_out, int32_t *status,
                       cudaStream_t st) {
  const size_t esz = f.dtype == BLOSSOM_DTYPE_FP32 ? 4 : 2;
  rows::Alignment al;
  al.rows_at(f.x, f.ldx, esz);
  al.rows_at(f.weight, f.ldw, esz);
  const int width = al.elements(f.cols, esz);
  // warps that share a column's k: until an SM has a block, with a pass over k each at least
  with_rows(f.dtype, f.rows, [&](auto t, auto r) {
    using T = decltype(t);
    constexpr int R = decltype(r)::value, C = R <= 4 ? 4 : 2;
    int wk = 1;
    while (wk < kWarps && f.cols > 256 * wk && (int64_t)(f.outs + C - 1) / C * wk < kSMs * kWarps) wk *= 2;
    const int columns = kWarps / wk * C;
    auto go = [&](auto w) {
      constexpr int W = decltype(w)::value;
      LaunchScope ls(slope ? K_LINEAR_SLOPE : K_LINEAR_FWD, st);
      launch_chained(slope ? few_rows_kernel<T, R, W, true> : few_rows_kernel<T, R, W, false>, dim3((unsigned)((f.outs + columns - 1) / columns)),
                     dim3(kThreads), 0, st, f.rows, f.cols, f.outs, wk, static_cast<const T *>(f.x), f.ldx, static_cast<const T *>(f.weight),
                     f.ldw, static_cast<const T *>(f.bias), static_cast<const T *>(extra), ld_extra, f.act, out, ld_out, status);
    };
    if (width == (int)(16 / esz)) go(std::integral_constant<int, 16 / sizeof(T)>());
    else if (width >= 2) go(std::integral_constant<int, 2>());
    else go(std::integral_constant<int, 1>());
  });
  return cudaGetLastError() == cudaSuccess ? BLOSSOM_OK : BLOSSOM_ERR_CUDA;
}

int launch_few_backward(const FewRows &f, const void *g, int64_t ldg, bool g_wide, float *part, void *dx, int64_t ld_dx, void *dweight,
                        int64_t ld_dweight, void *dbias, int32_t *status, cudaStream_t st) {
  const size_t esz = f.dtype == BLOSSOM_DTYPE_FP32 ? 4 : 2;
  const unsigned blocks = (unsigned)((f.cols + 4 * kThreads - 1) / (4 * kThreads));
  with_rows(f.dtype, f.rows, [&](auto t, auto r) {
    using T = decltype(t);
    constexpr int R = decltype(r)::value;
    auto typed = [&](auto gt) {
      using G = decltype(gt);
      const G *const from = static_cast<const G *>(g);
      if (dx) {
        rows::Alignment al;
        al.rows_at(f.weight, f.ldw, esz);
        const int shares = few_shares(f.cols, f.outs), per = (f.outs + shares - 1) / shares;
        LaunchScope ls(K_LINEAR_DX, st);
        launch_chained(al.elements(f.cols, esz) >= 4 ? few_dx_kernel<T, G, R, 4> : few_dx_kernel<T, G, R, 1>, dim3(blocks, (unsigned)shares),
                       dim3(kThreads), 0, st, f.rows, f.cols, f.outs, per, from, ldg, static_cast<const T *>(f.weight), f.ldw, part, status);
      }
      if (dweight || dbias) {
        rows::Alignment al;
        al.rows_at(dweight, ld_dweight, esz);
        // outs a block: two blocks an SM
        const int want = 2 * kSMs / (int)blocks, shares = want < 1 ? 1 : want, per = (f.outs + shares - 1) / shares;
        LaunchScope ls(K_LINEAR_DWEIGHT, st);
        launch_chained(al.elements(f.cols, esz) >= 4 ? few_dweight_kernel<T, G, R, 4> : few_dweight_kernel<T, G, R, 1>,
                       dim3(dweight ? blocks : 1, (unsigned)((f.outs + per - 1) / per)), dim3(kThreads), 0, st, f.rows, f.cols, f.outs, per,
                       from, ldg, static_cast<const T *>(f.x), f.ldx, static_cast<T *>(dweight), ld_dweight, static_cast<T *>(dbias), dx ? nullptr : status);
      }
    };
    if (g_wide) typed(float());
    else typed(T());
  });
  if (cudaGetLastError() != cudaSuccess) return BLOSSOM_ERR_CUDA;
  if (!dx) return BLOSSOM_OK;
  return launch_join(f.dtype, part, nullptr, few_shares(f.cols, f.outs), 0, f.rows, f.cols, dx, ld_dx, nullptr, st);
}

}  // namespace linear
}  // namespace blossom
