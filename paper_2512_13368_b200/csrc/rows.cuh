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
  int drop;                // 0: everything is kept, 1: by the generator, 2: nothing is
  unsigned bar, site;      // an element is kept if its 16 bits are >= bar / 65536 (bar: those bits above 16 zeros)
  float scale;             // of the kept ones
  float eps, inv_cols;
  int wide_weights;        // weight and bias are fp32 (else bf16)
};

// ---- a group of 8 columns in four pairs, W elements an access --------------------------------------
// W is the widest of 16 bytes, 8 bytes, two elements and one that every row's address and length is a multiple of.
struct Group {
  float2 p[4];
  __device__ __forceinline__ float &at(int j) { return j & 1 ? p[j / 2].y : p[j / 2].x; }
};
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  uint64_t d;
  asm("mul.rn.ftz.f32x2 %0, %1, %2;"
      : "=l"(d)
      : "l"(*reinterpret_cast<uint64_t *>(&a)), "l"(*reinterpret_cast<uint64_t *>(&b)));
  return *reinterpret_cast<float2 *>(&d);
}
__device__ __forceinline__ float2 halves(uint32_t w) {  // two bf16
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);  // round to nearest even, once
  return *reinterpret_cast<const uint32_t *>(&h);
}
// As it comes from memory: loads that are under way hold half as many registers in bf16.
template <typename T, int W>
struct Raw {
  uint32_t w[2 * sizeof(T)];
  // the elements j .. j + W - 1 from p, or zeros
  __device__ __forceinline__ void piece(const T *p, int j, bool there) {
    constexpr int words = W * (int)sizeof(T) / 4;  // an access has (0: half a one)
    const int at = j * (int)sizeof(T) / 4;
    if (there) {
      if constexpr (words == 4) {
        const uint4 q = *reinterpret_cast<const uint4 *>(p);
        w[at] = q.x, w[at + 1] = q.y, w[at + 2] = q.z, w[at + 3] = q.w;
      } else if constexpr (words == 2) {
        const uint2 q = *reinterpret_cast<const uint2 *>(p);
        w[at] = q.x, w[at + 1] = q.y;
      } else if constexpr (words == 1) {
        w[at] = *reinterpret_cast<const uint32_t *>(p);
      } else {
        const uint32_t h = *reinterpret_cast<const uint16_t *>(p);
        w[at] = j & 1 ? w[at] | h << 16 : h;
      }
    } else if constexpr (words > 0) {
#pragma unroll
      for (int i = 0; i < words; ++i) w[at + i] = 0;
    } else if (!(j & 1)) {
      w[at] = 0;
    }
  }
  __device__ __forceinline__ void load(const T *p, int valid) {
#pragma unroll
    for (int j = 0; j < 8; j += W) piece(p + j, j, j < valid);
  }
  __device__ __forceinline__ Group get() const {
    Group v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) v.p[i] = make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
      else v.p[i] = halves(w[i]);
    }
    return v;
  }
};
// ---- bf16 rows under way in shared memory ----------------------------------------------------------
// Asynchronous copies bring the rows to come without a register for them.  A thread copies and reads its own groups of 8 columns
// alone, 16 bytes each, so that nobody meets at a barrier; the threads' groups lie side by side.  G: groups a thread and stage.
// (In fp32 the two halves of a group would come by two copies that take the same sectors from L2 twice: 32768 x 1024 forward
// 106 us instead of 70, backward 174 instead of 121.)
template <int G, int THREADS>
struct Ring {
  static constexpr int kStage = G * 16 * THREADS;
  char *mine;
  __device__ __forceinline__ explicit Ring(void *smem) : mine(static_cast<char *>(smem) + 16 * threadIdx.x) {}
  // 8 elements from p into group g; zeros if they are not there, which are not read
  __device__ __forceinline__ void copy(int stage, int g, const void *p, bool there) const {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                     (uint32_t)__cvta_generic_to_shared(mine) + stage * kStage + g * 16 * THREADS),
                 "l"(p), "r"(there ? 16 : 0)
                 : "memory");
  }
  template <typename T, int W>
  __device__ __forceinline__ void get(int stage, int g, Raw<T, W> &r) const {
    const uint4 q = *reinterpret_cast<const uint4 *>(mine + stage * kStage + g * 16 * THREADS);
    r.w[0] = q.x, r.w[1] = q.y, r.w[2] = q.z, r.w[3] = q.w;
  }
  // Stages for `resident` CTAs an SM that take `other` bytes besides: up to four.
  static constexpr int stages(int resident, int other) {
    const int n = (227 * 1024 / resident - 1024 - other) / kStage;
    return n < 0 ? 0 : n < 4 ? n : 4;
  }
};
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }  // of a stage
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }  // all but N stages

// More than 48 KB, `fixed` of them the kernel's own arrays, have to be asked for.
template <typename K>
inline bool allow_stages(K kern, int dynamic, int fixed) {
  return dynamic + fixed <= 48 * 1024 ||
         cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, dynamic) == cudaSuccess;
}

// All of an SM's shared memory for the kernels of wide rows: a CTA that starts before the kernel ahead of it has ended finds the
// split between L1 and shared memory as that one left it, and while one runs it stays so, too small for the others (32768 x
// 1024, forward and backward in turn: 141 us without, 110 with it; narrow rows, 131072 x 256: 106 without, 112 with).
template <typename K>
inline void prefer_shared(K kern) {
  (void)cudaFuncSetAttribute(kern, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
}

template <typename T, int W>
__device__ __forceinline__ void store_piece(T *p, int j, Group &v) {
  if constexpr (sizeof(T) == 4 && W == 4) {
    *reinterpret_cast<float4 *>(p) = make_float4(v.at(j), v.at(j + 1), v.at(j + 2), v.at(j + 3));
  } else if constexpr (sizeof(T) == 4 && W == 2) {
    *reinterpret_cast<float2 *>(p) = v.p[j / 2];
  } else if constexpr (sizeof(T) == 4) {
    *p = v.at(j);
  } else if constexpr (W == 8) {
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack2(v.p[0].x, v.p[0].y), pack2(v.p[1].x, v.p[1].y),
                                               pack2(v.p[2].x, v.p[2].y), pack2(v.p[3].x, v.p[3].y));
  } else if constexpr (W == 4) {
    *reinterpret_cast<uint2 *>(p) = make_uint2(pack2(v.at(j), v.at(j + 1)), pack2(v.at(j + 2), v.at(j + 3)));
  } else if constexpr (W == 2) {
    *reinterpret_cast<uint32_t *>(p) = pack2(v.at(j), v.at(j + 1));
  } else {
    *p = __float2bfloat16(v.at(j));
  }
}
template <typename T, int W>
__device__ __forceinline__ void store_group(T *p, int valid, const Group &g) {
  Group v = g;
#pragma unroll
  for (int j = 0; j < 8; j += W)
    if (j < valid) store_piece<T, W>(p + j, j, v);
}
// what is subtracted from the columns that are there, zero for the others (whose elements are zero and stay so)
template <int W>
__device__ __forceinline__ Group spread(float v, int valid) {
  Group g;
#pragma unroll
  for (int j = 0; j < 8; j += W)
#pragma unroll
    for (int i = 0; i < W; ++i) g.at(j + i) = j < valid ? v : 0.f;
  return g;
}
// weight and bias come in either type, at any alignment of theirs, once per thread and group
__device__ __forceinline__ Group load_weights(const void *p, int wide, int at, int valid, float other) {
  Group v;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v.at(i) = other;
    if (p && i < valid)
      v.at(i) = wide ? static_cast<const float *>(p)[at + i] : __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[at + i]);
  }
  return v;
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
  // 16 bits decide an element, so that one evaluation serves the 8 elements of a 16-byte access in bf16 (32 bits each would
  // double the generator's share of the kernel's instructions)
  __device__ __forceinline__ uint4 bits(const Args &a, int row, int group) const {
    return philox(make_uint4((uint32_t)group | a.site << 16, (uint32_t)row, step.x, step.y), key);
  }
};
// zero where an element is dropped, whatever it was; the kept ones are yet to be scaled
__device__ __forceinline__ void drop(const Args &a, uint4 bits, Group &v) {
  const uint32_t x[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v.p[i].x = (x[i] << 16) >= a.bar ? v.p[i].x : 0.f;  // (bar's low 16 bits are zero)
    v.p[i].y = x[i] >= a.bar ? v.p[i].y : 0.f;
  }
}

// ---- sums over a row's TPR threads ---------------------------------------------------------------
// Every thread gets the same bits: within a warp by exchange, across warps added up in the order of the warps.  buf: two
// slots of TPR / 32 sums that alternate, so that one barrier a sum suffices.
__device__ __forceinline__ float total(const float2 (&v)[4]) {
  const float2 s = add2(add2(v[0], v[1]), add2(v[2], v[3]));
  return s.x + s.y;
}
__device__ __forceinline__ float exchange_add(float v, int o) { return v + __shfl_xor_sync(0xffffffffu, v, o); }
__device__ __forceinline__ float2 exchange_add(float2 v, int o) {
  return add2(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
}
__device__ __forceinline__ float plus(float a, float b) { return a + b; }
__device__ __forceinline__ float2 plus(float2 a, float2 b) { return add2(a, b); }
template <int TPR, typename S>
__device__ __forceinline__ S row_sum(S v, S *buf, int &turn) {
#pragma unroll
  for (int o = 1; o < (TPR < 32 ? TPR : 32); o <<= 1) v = exchange_add(v, o);
  if constexpr (TPR > 32) {
    constexpr int NW = TPR / 32;
    S *b = buf + turn * NW;
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) b[threadIdx.x >> 5] = v;
    __syncthreads();
    v = b[0];
#pragma unroll
    for (int i = 1; i < NW; ++i) v = plus(v, b[i]);
  }
  return v;
}

// ---- shapes ----------------------------------------------------------------------------------
// TPR threads a row, V groups of 8 columns a thread: groups of threads as narrow as the row, so that narrow rows share a
// warp; then more columns a thread, so that a row's sums are exchanged once for all of them; then a CTA a row.
template <int TPR_, int V_>
struct Plan {
  static constexpr int TPR = TPR_, V = V_, threads = TPR_ > 32 ? TPR_ : 128, slots = threads / TPR_;
};
template <int VMAX, typename F>
inline void with_plan(int groups, F &&f) {
  if (groups <= 4) return f(Plan<4, 1>());
  if (groups <= 8) return f(Plan<8, 1>());
  if (groups <= 16) return f(Plan<16, 1>());
  if (groups <= 32) return f(Plan<32, 1>());
  constexpr int V = VMAX;
  if constexpr (VMAX > 2)
    if (groups <= 64) return f(Plan<32, 2>());
  if (groups <= 32 * V) return f(Plan<32, V>());
  if (groups <= 64 * V) return f(Plan<64, V>());
  if (groups <= 128 * V) return f(Plan<128, V>());
  if (groups <= 256 * V) return f(Plan<256, V>());
  if constexpr (VMAX < 4)
    if (groups <= 512 * V) return f(Plan<512, V>());
}

// Elements an access may take: 16 bytes, 8 bytes, two elements or one.
struct Alignment {
  uint64_t bits = 0;
  void rows_at(const void *p, int64_t stride, size_t esz) {
    if (p) bits |= reinterpret_cast<uintptr_t>(p) | (uint64_t)stride * esz;
  }
  int elements(int cols, size_t esz) const {
    const uint64_t b = bits | (uint64_t)cols * esz;
    return b % 16 == 0 ? (int)(16 / esz) : b % 8 == 0 ? (int)(8 / esz) : b % (2 * esz) == 0 ? 2 : 1;
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
    else if (w == 4) f(__nv_bfloat16(), integral_constant<int, 4>());
    else if (w == 2) f(__nv_bfloat16(), integral_constant<int, 2>());
    else f(__nv_bfloat16(), integral_constant<int, 1>());
  }
}

}  // namespace rows
}  // namespace blossom
