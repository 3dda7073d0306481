// Rows of cols elements around the attention: dropout and the residual + layer norm sub-layer.  What the kernels share:
// access to a group of 8 columns, the counter-based generator, sums over a row, and the choice of a shape.
#pragma once
#include "common.cuh"

namespace blossom {
namespace rows {

constexpr int kSMs = 148;
constexpr int kMaxCols = 8192;

struct Args {
  int rows, cols, groups;  // groups of 8 columns, the last one possibly short
  int64_t sx, sr, so, sdx, sdr;  // element strides: x, residual, out / dout, dx, dresidual
  unsigned bar, site;      // an element is kept if its 16 bits are >= bar
  float scale;             // of the kept ones
  float eps, inv_cols;
  int wide_weights;        // weight and bias are fp32 (else bf16)
};

// ---- a group of 8 columns, W elements an access -------------------------------------------------
// W is the widest of 16 bytes, two elements and one that every row's address and length is a multiple of.
template <typename T, int W>
__device__ __forceinline__ void load_group(const T *p, int valid, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; j += W) {
    if (j < valid) {
      if constexpr (sizeof(T) == 4 && W == 4) {
        const float4 q = *reinterpret_cast<const float4 *>(p + j);
        v[j] = q.x, v[j + 1] = q.y, v[j + 2] = q.z, v[j + 3] = q.w;
      } else if constexpr (sizeof(T) == 4 && W == 2) {
        const float2 q = *reinterpret_cast<const float2 *>(p + j);
        v[j] = q.x, v[j + 1] = q.y;
      } else if constexpr (sizeof(T) == 4) {
        v[j] = p[j];
      } else if constexpr (W == 8) {
        const uint4 q = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      } else if constexpr (W == 2) {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(p + j);
        v[j] = __uint_as_float(w << 16), v[j + 1] = __uint_as_float(w & 0xffff0000u);
      } else {
        v[j] = __bfloat162float(p[j]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < W; ++i) v[j + i] = 0.f;
    }
  }
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);  // round to nearest even, once
  return *reinterpret_cast<const uint32_t *>(&h);
}
template <typename T, int W>
__device__ __forceinline__ void store_group(T *p, int valid, const float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; j += W) {
    if (j < valid) {
      if constexpr (sizeof(T) == 4 && W == 4) {
        *reinterpret_cast<float4 *>(p + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
      } else if constexpr (sizeof(T) == 4 && W == 2) {
        *reinterpret_cast<float2 *>(p + j) = make_float2(v[j], v[j + 1]);
      } else if constexpr (sizeof(T) == 4) {
        p[j] = v[j];
      } else if constexpr (W == 8) {
        *reinterpret_cast<uint4 *>(p) = make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
      } else if constexpr (W == 2) {
        *reinterpret_cast<uint32_t *>(p + j) = pack2(v[j], v[j + 1]);
      } else {
        p[j] = __float2bfloat16(v[j]);
      }
    }
  }
}
// weight and bias come in either type, at any alignment of theirs, once per thread and group
__device__ __forceinline__ void load_weights(const void *p, int wide, int at, int valid, float other, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = other;
    if (p && i < valid)
      v[i] = wide ? static_cast<const float *>(p)[at + i] : __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[at + i]);
  }
}

// ---- which elements a dropout keeps ------------------------------------------------------------
// Philox 4x32, ten rounds (Salmon et al., 2011): each round multiplies two counter words by odd constants, swaps the halves of
// the products and mixes in the other words and the key, which moves on by another pair of constants.
__device__ __forceinline__ uint4 philox(uint4 c, uint2 key) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)0xD2511F53u * c.x, b = (uint64_t)0xCD9E8D57u * c.z;
    c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ key.x, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ key.y, (uint32_t)a);
    key.x += 0x9E3779B9u;
    key.y += 0xBB67AE85u;
  }
  return c;
}
struct Generator {
  uint2 key, step;
  __device__ __forceinline__ void read(const int64_t *rng) {
    const uint64_t a = (uint64_t)rng[0], b = (uint64_t)rng[1];
    key = make_uint2((uint32_t)a, (uint32_t)(a >> 32));
    step = make_uint2((uint32_t)b, (uint32_t)(b >> 32));
  }
  // bit i: column i of the group is kept.  16 bits decide an element, so that one evaluation serves the 8 elements
  // of a 16-byte access in bf16 (32 bits each would double the generator's share of the kernel's instructions)
  __device__ __forceinline__ uint32_t kept(const Args &a, int row, int group) const {
    const uint4 w = philox(make_uint4((uint32_t)group | a.site << 16, (uint32_t)row, step.x, step.y), key);
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m |= (uint32_t)((x[i] & 0xffffu) >= a.bar) << (2 * i);
      m |= (uint32_t)((x[i] >> 16) >= a.bar) << (2 * i + 1);
    }
    return m;
  }
};

// ---- sums over a row's TPR threads ---------------------------------------------------------------
// Every thread gets the same bits: within a warp by exchange, across warps added up in the order of the warps.  buf: two
// slots of TPR / 32 pairs that alternate, so that one barrier a sum suffices.
template <int TPR>
__device__ __forceinline__ float2 row_sum(float2 v, float2 *buf, int &turn) {
#pragma unroll
  for (int o = 1; o < (TPR < 32 ? TPR : 32); o <<= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
  }
  if constexpr (TPR > 32) {
    constexpr int NW = TPR / 32;
    float2 *b = buf + turn * NW;
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) b[threadIdx.x >> 5] = v;
    __syncthreads();
    v = b[0];
#pragma unroll
    for (int i = 1; i < NW; ++i) v.x += b[i].x, v.y += b[i].y;
  }
  return v;
}
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float2 *buf, int &turn) {
  if constexpr (TPR > 32) return row_sum<TPR>(make_float2(v, 0.f), buf, turn).x;
#pragma unroll
  for (int o = 1; o < (TPR < 32 ? TPR : 32); o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// ---- shapes ----------------------------------------------------------------------------------
// A thread holds one group of 8 columns of a row, TPR threads a row: groups of threads as narrow as the row, so that narrow
// rows share a warp; rows of more than 256 columns take a CTA of their own.
template <int TPR_>
struct Plan {
  static constexpr int TPR = TPR_, threads = TPR_ > 32 ? TPR_ : 256, slots = threads / TPR_;
};
template <typename F>
inline void with_plan(int groups, F &&f) {
  if (groups <= 4) f(Plan<4>());
  else if (groups <= 8) f(Plan<8>());
  else if (groups <= 16) f(Plan<16>());
  else if (groups <= 32) f(Plan<32>());
  else if (groups <= 64) f(Plan<64>());
  else if (groups <= 128) f(Plan<128>());
  else if (groups <= 256) f(Plan<256>());
  else if (groups <= 512) f(Plan<512>());
  else f(Plan<1024>());
}

// Elements an access may take: 16 bytes, two elements or one.
struct Alignment {
  uint64_t bits = 0;
  void rows_at(const void *p, int64_t stride, size_t esz) {
    if (p) bits |= reinterpret_cast<uintptr_t>(p) | (uint64_t)stride * esz;
  }
  int elements(int cols, size_t esz) const {
    const uint64_t b = bits | (uint64_t)cols * esz;
    return b % 16 == 0 ? (int)(16 / esz) : b % (2 * esz) == 0 ? 2 : 1;
  }
};

int check(const blossom_rows_params *p, int max_cols, const int64_t *rng, Args *a);
int backward_ctas(const Args &a);

// f(T, W): element type and elements an access
template <typename F>
inline void with_type(int dtype, int w, F &&f) {
  using std::integral_constant;
  if (dtype == BLOSSOM_DTYPE_FP32) {
    if (w == 4) f(float(), integral_constant<int, 4>());
    else if (w == 2) f(float(), integral_constant<int, 2>());
    else f(float(), integral_constant<int, 1>());
  } else {
    if (w == 8) f(__nv_bfloat16(), integral_constant<int, 8>());
    else if (w == 2) f(__nv_bfloat16(), integral_constant<int, 2>());
    else f(__nv_bfloat16(), integral_constant<int, 1>());
  }
}

}  // namespace rows
}  // namespace blossom
