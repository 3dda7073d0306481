// Rows in 8 bits with a power of two for every 32 columns, and back.
//
// Bound: memory, an element in and 33 / 32 bytes out, or the other way round.  Four threads hold 32 columns, 8 each, and exchange
// the largest magnitude, as bits: what is no number is the largest of all.  Powers of two make every step exact but the one
// rounding, and the values exact in bf16 too.  131072 x 256 bf16, 102 MB each way: 22 and 16 us.  A thread asks for four rows
// before it needs the first (one at a time 54 us for both, four 45; codes by whole-number addition instead of conversions 42; as
// many blocks as that takes 40; 48 registers instead of 72, 40 warps an SM, 38; 40 registers and 48 warps 39).
#include "rows.cuh"

namespace blossom {
namespace rows {
namespace {

// 8 codes from or to memory; wide: their address is a multiple of 8
__device__ __forceinline__ void store_codes(int8_t *p, int valid, bool wide, uint2 c) {
  if (wide && valid >= 8) {
    *reinterpret_cast<uint2 *>(p) = c;
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < valid) p[j] = (int8_t)((j < 4 ? c.x : c.y) >> (8 * (j % 4)));
}
__device__ __forceinline__ uint2 load_codes(const int8_t *p, int valid, bool wide) {
  if (wide && valid >= 8) return *reinterpret_cast<const uint2 *>(p);
  uint2 c = make_uint2(0, 0);
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < valid) (j < 4 ? c.x : c.y) |= (uint32_t)(uint8_t)p[j] << (8 * (j % 4));
  return c;
}
// 2^(133 - E); nothing is kept of groups of tiny numbers and of those with one that is none
__device__ __forceinline__ float code_per_value(uint32_t e) { return e <= 6 || e == 255 ? 0.f : __uint_as_float((260 - e) << 23); }

// The largest magnitude of 32 columns, as a float's bits; bf16 are compared two at a time as they come.
template <typename T, int W>
__device__ __forceinline__ uint32_t top_of_four(const Raw<T, W> &v, uint32_t four) {
  constexpr uint32_t value = sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
  auto larger = [](uint32_t a, uint32_t b) { return sizeof(T) == 4 ? max(a, b) : __vmaxu2(a, b); };
  uint32_t top = v.w[0] & value;
#pragma unroll
  for (int i = 1; i < 2 * (int)sizeof(T); ++i) top = larger(top, v.w[i] & value);
  top = larger(top, __shfl_xor_sync(four, top, 1));
  top = larger(top, __shfl_xor_sync(four, top, 2));
  return sizeof(T) == 4 ? top : max(top & 0xffff0000u, top << 16);
}
// x * f + c of subnormal x too, which this build's arithmetic would take for zeros: beside a largest magnitude below 2^-119 they
// have codes of 1
__device__ __forceinline__ float2 fma2_of_all(float2 x, float2 f, float2 c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(d)
      : "l"(*reinterpret_cast<uint64_t *>(&x)), "l"(*reinterpret_cast<uint64_t *>(&f)), "l"(*reinterpret_cast<uint64_t *>(&c)));
  return *reinterpret_cast<float2 *>(&d);
}
// 8 values' codes, f a value.  1.5 * 2^23 rounds a sum to whole numbers and leaves them in the lowest bits; the product is exact.
__device__ __forceinline__ void codes_of(Group z, float f, uint32_t top, uint32_t (&c)[2]) {
  constexpr float magic = 12582912.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) z.p[i] = fma2_of_all(z.p[i], both(f), both(magic));
  if ((top & 0x7fffffu) >= 0x7f0000u) {  // of 127.5 and more there are 128s
#pragma unroll
    for (int j = 0; j < 8; ++j) z.at(j) = fminf(fmaxf(z.at(j), magic - 127.f), magic + 127.f);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)
    c[h] = __byte_perm(__byte_perm(__float_as_uint(z.at(4 * h)), __float_as_uint(z.at(4 * h + 1)), 0x0040),
                       __byte_perm(__float_as_uint(z.at(4 * h + 2)), __float_as_uint(z.at(4 * h + 3)), 0x0040), 0x5410);
}

// rows that a thread asks for before it needs the first
template <typename P>
constexpr int U = P::V == 1 ? 4 : 2;

template <typename T, int W, typename P>
__global__ void __launch_bounds__(P::threads, sizeof(T) == 2 && P::V == 1 ? 1280 / P::threads : 1) pack_rows_kernel(Args a, const T *x, int8_t *codes, uint8_t *scales, int wide) {
  grid_chain_enter();
  x = behind_wait(x);
  const int lane = (int)threadIdx.x % P::TPR, chunks = (a.cols + 31) / 32;
  const uint32_t four = 0xfu << ((int)threadIdx.x % 32 / 4 * 4);
  const int64_t step = (int64_t)gridDim.x * P::slots;
  for (int64_t row0 = (int64_t)blockIdx.x * P::slots + threadIdx.x / P::TPR; row0 < a.rows; row0 += U<P> * step) {
    Raw<T, W> v[U<P>][P::V];
#pragma unroll
    for (int u = 0; u < U<P>; ++u) {
      const int64_t row = row0 + u * step;
#pragma unroll
      for (int k = 0; k < P::V; ++k)
        v[u][k].load(x + (row < a.rows ? row : row0) * a.sx + 8 * (lane + k * P::TPR),
                     row < a.rows ? a.cols - 8 * (lane + k * P::TPR) : 0);
    }
#pragma unroll
    for (int i = 0; i < U<P> * P::V; ++i) {
      const int u = i / P::V, k = i % P::V;
      const int64_t row = row0 + u * step;
      if (row >= a.rows) break;  // (the four that share 32 columns are of one row)
      const int g = lane + k * P::TPR;
      const uint32_t top = top_of_four(v[u][k], four), e = top >> 23;
      const float f = code_per_value(e);
      uint32_t c[2] = {0, 0};
      if (f != 0.f) codes_of(v[u][k].get(), f, top, c);
      store_codes(codes + row * a.cols + 8 * g, a.cols - 8 * g, wide, make_uint2(c[0], c[1]));
      if (g % 4 == 0 && g / 4 < chunks) scales[row * chunks + g / 4] = (uint8_t)(e <= 6 ? 0 : e);
    }
  }
}

template <typename T, int W, typename P>
__global__ void __launch_bounds__(P::threads) unpack_rows_kernel(Args a, const int8_t *codes, const uint8_t *scales, T *out,
                                                                 int wide) {
  grid_chain_enter();
  codes = behind_wait(codes), scales = behind_wait(scales);
  const int lane = (int)threadIdx.x % P::TPR, chunks = (a.cols + 31) / 32;
  const int64_t step = (int64_t)gridDim.x * P::slots;
  for (int64_t row0 = (int64_t)blockIdx.x * P::slots + threadIdx.x / P::TPR; row0 < a.rows; row0 += U<P> * step) {
    uint2 c[U<P> * P::V];
    uint32_t e[U<P> * P::V];
#pragma unroll
    for (int i = 0; i < U<P> * P::V; ++i) {
      const int g = lane + i % P::V * P::TPR;
      const int64_t row = row0 + i / P::V * step;
      const bool there = row < a.rows;
      c[i] = load_codes(codes + (there ? row : row0) * a.cols + 8 * g, there ? a.cols - 8 * g : 0, wide);
      e[i] = there && g / 4 < chunks ? scales[row * chunks + g / 4] : 0;
    }
#pragma unroll
    for (int i = 0; i < U<P> * P::V; ++i) {
      const int g = lane + i % P::V * P::TPR;
      const int64_t row = row0 + i / P::V * step;
      if (row >= a.rows) break;
      const float f = value_per_code(e[i]);
      Group z;
#pragma unroll
      for (int j = 0; j < 8; ++j) z.at(j) = (float)(int8_t)((j < 4 ? c[i].x : c[i].y) >> (8 * (j % 4))) * f;
      store_group<T, W>(out + row * a.so + 8 * g, a.cols - 8 * g, z);
    }
  }
}

int check_packed(const blossom_rows_params *p, Args *a) {
  static const int64_t any[2] = {0, 0};
  return check(p, kMaxCols, any, a);
}

template <bool PACK>
int launch_packed(const blossom_rows_params *p, const Args &a, const void *x, void *codes, void *scales, cudaStream_t st) {
  const size_t esz = p->dtype == BLOSSOM_DTYPE_FP32 ? 4 : 2;
  if (!x || !codes || !scales || reinterpret_cast<uintptr_t>(x) % esz) return BLOSSOM_ERR_INVALID_ARG;
  Alignment al;
  al.rows_at(x, PACK ? a.sx : a.so, esz);
  const int wide = (reinterpret_cast<uintptr_t>(codes) | (uintptr_t)a.cols) % 8 == 0;
  with_plan<2>(a.groups, [&](auto plan) {
    using P = decltype(plan);
    with_type(p->dtype, al.elements(a.cols, esz), [&](auto t, auto w) {
      using T = decltype(t);
      constexpr int W = decltype(w)::value;
      // a row a thread until the device is full, then U, in as many blocks as that takes (131072 x 256 and back 40 us; blocks
      // that stay and loop 42 to 47; 25597 x 50 with U rows at once 12 us instead of 8)
      const int64_t ctas = (a.rows + P::slots - 1) / P::slots, full = kSMs * (2048 / P::threads), by_u = (ctas + U<P> - 1) / U<P>;
      const dim3 grid((unsigned)(ctas < full ? ctas : by_u < full ? full : by_u)), block(P::threads);
      LaunchScope ls(PACK ? K_PACK_ROWS : K_UNPACK_ROWS, st);
      if constexpr (PACK)
        launch_chained(pack_rows_kernel<T, W, P>, grid, block, 0, st, a, static_cast<const T *>(x), static_cast<int8_t *>(codes),
                       static_cast<uint8_t *>(scales), wide);
      else
        launch_chained(unpack_rows_kernel<T, W, P>, grid, block, 0, st, a, static_cast<const int8_t *>(codes),
                       static_cast<const uint8_t *>(scales), static_cast<T *>(const_cast<void *>(x)), wide);
    });
  });
  return cudaGetLastError() == cudaSuccess ? BLOSSOM_OK : BLOSSOM_ERR_CUDA;
}

}  // namespace
}  // namespace rows
}  // namespace blossom

extern "C" int blossom_pack_rows(const blossom_rows_params *params, const void *x, int8_t *codes, uint8_t *scales,
                                 blossom_stream_t stream) {
  using namespace blossom;
  prof_break();
  rows::Args a;
  if (int rc = rows::check_packed(params, &a)) return rc;
  if (a.rows == 0) return BLOSSOM_OK;
  return rows::launch_packed<true>(params, a, x, codes, scales, (cudaStream_t)stream);
}

extern "C" int blossom_unpack_rows(const blossom_rows_params *params, const int8_t *codes, const uint8_t *scales, void *out,
                                   blossom_stream_t stream) {
  using namespace blossom;
  prof_break();
  rows::Args a;
  if (int rc = rows::check_packed(params, &a)) return rc;
  if (a.rows == 0) return BLOSSOM_OK;
  return rows::launch_packed<false>(params, a, out, const_cast<int8_t *>(codes), const_cast<uint8_t *>(scales),
                                    (cudaStream_t)stream);
}
