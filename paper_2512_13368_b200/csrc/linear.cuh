// A linear layer with what follows it: what the kernels share.
#pragma once
#include <math.h>

#include "rows.cuh"

namespace blossom {
namespace linear {

constexpr int kSMs = 148;
constexpr int kMaxWidth = 65536;

// ---- the activation and its derivative --------------------------------------------------------------------
// (what is no number stays so)
__device__ __forceinline__ float at_least(float x, float least) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(least));
  return y;
}
__device__ __forceinline__ float at_most(float x, float most) {
  float y;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(most));
  return y;
}
__device__ __forceinline__ float2 at_least(float2 x, float least) { return make_float2(at_least(x.x, least), at_least(x.y, least)); }
__device__ __forceinline__ float2 at_most(float2 x, float most) { return make_float2(at_most(x.x, most), at_most(x.y, most)); }
// Two arguments at a time.
// Phi(x) = sigmoid(x P(x^2)), P a polynomial fitted to the logit of Phi (weighted least squares, the weights moved towards the
// largest errors).  For bf16 results P has nine terms: x Phi(x) is off by 9e-4 of itself at most, from x = -6 on, a quarter of
// their half step; else seven, off by 7e-8, for whom a relative error would be asking for more than their argument is known to.
// The derivative is Phi(x) + x phi(x), Phi off by 5e-8.  (Five terms of the value are off by 4e-6, 2.6 % of it at x = -4, and four
// of a logit that serves for the derivative's polynomial as well by 4.4e-5: 131072 x 64 -> 256, forward and backward, 91 us, with
// these terms 96; 99 with seven terms and the derivative of their polynomial.)
// An exponential and a reciprocal an element (and an exponential for phi), which the unit for those gives 16 a clock and SM:
// 131072 x 256 elements 15 us, and 22; with the error function it is the FMA pipes, three times as long.  (One reciprocal for two
// elements makes both of them no number if one is, and keeps an element's bits from depending on itself alone; without that, by
// a minimum that takes what is no number for 60, 131072 x 64 -> 256 takes 98 us instead of 95.)  From |x| = 6 on the
// derivative is 0 or 1 to 4e-8, from x = -6 down the value is 0 to 6e-9: arguments are cut there, so that
// infinite ones have their limits.
constexpr float kLog2e = 1.4426950408889634f;
using rows::mul2;
// a constant in a pair of registers (which the compiler would otherwise fill anew for every use)
__device__ __forceinline__ float2 held(float v) {
  float2 p = make_float2(v, v);
  asm volatile("" : "+l"(*reinterpret_cast<uint64_t *>(&p)));
  return p;
}
__device__ __forceinline__ float reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// WIDE: the results are of single precision
template <int ACT, bool SLOPE, bool WIDE = false>
struct Curve {
  static constexpr bool kGelu = ACT == BLOSSOM_ACT_GELU, kSilu = ACT == BLOSSOM_ACT_SILU;
  static constexpr float kCut = kGelu ? 6.f : 40.f;  // (silu: from x = -40 down 0 to 2e-16)
  static constexpr bool kFar = kGelu && !SLOPE && !WIDE;  // nine terms
  // (the lowest terms are held; the others, which would not fit the registers, are one-element instructions' own)
  static constexpr int kTerms = kFar ? 9 : 7, kHeld = kGelu ? 5 : 1;
  float2 p[kHeld], half, top, one, minus;
  // Of P: the terms of a short fit and what those of the long one have besides.
  static __device__ constexpr float term(int i) {
    constexpr float value[5] = {1.5957043f, 0.072862640f, -0.00021803212f, -6.5811037e-05f, 2.4471922e-06f};
    constexpr float value_rest[9] = {6.89029694e-05f, -0.00020750612f, 0.000163902325f, -4.95181739e-05f, 6.45735508e-06f,
                                     -3.66156229e-07f, 8.67401528e-09f, -1.09854764e-10f, 5.69511343e-13f};
    constexpr float both[4] = {1.5954539f, 0.073342353f, -0.00046575911f, -2.1383154e-05f};
    constexpr float both_rest[7] = {0.000315785408f, -0.000676117837f, 0.00040095704f, -8.94888726e-05f, 7.98777546e-06f,
                                    -2.69765849e-07f, 3.67201225e-09f};
    return kFar ? (i < 5 ? value[i % 5] : 0.f) + value_rest[i] : (i < 4 ? both[i % 4] : 0.f) + both_rest[i % 7];
  }
  __device__ __forceinline__ Curve() {
    if constexpr (kGelu) {
#pragma unroll
      for (int i = 0; i < kHeld; ++i) p[i] = held(-kLog2e * term(i));
    }
    if constexpr (kGelu && SLOPE) half = held(-0.5f * kLog2e), top = held(0.3989422804014327f);
    if constexpr (kSilu) p[0] = held(-kLog2e);
    if constexpr (kGelu || kSilu) one = held(1.f);
    if constexpr (kSilu && SLOPE) minus = held(-1.f);
  }
  // -log2(e) P(t)
  __device__ __forceinline__ float2 scaled_p(float2 t) const {
    float2 s = make_float2(-kLog2e * term(kTerms - 1), -kLog2e * term(kTerms - 1));
#pragma unroll
    for (int i = kTerms - 2; i >= kHeld; --i) s = make_float2(fmaf(s.x, t.x, -kLog2e * term(i)), fmaf(s.y, t.y, -kLog2e * term(i)));
#pragma unroll
    for (int i = kHeld - 1; i >= 0; --i) s = fma2(s, t, p[i]);
    return s;
  }
  // 1 / (1 + 2^v)
  __device__ __forceinline__ float2 sigmoid2(float2 v) const {
    const float2 y = add2(make_float2(exp2f(v.x), exp2f(v.y)), one);
    return make_float2(reciprocal(y.x), reciprocal(y.y));
  }
  __device__ __forceinline__ float2 operator()(float2 x) const {
    if constexpr (ACT == BLOSSOM_ACT_NONE) return x;
    if constexpr (ACT == BLOSSOM_ACT_RELU) {
      if constexpr (SLOPE) return make_float2(x.x > 0.f ? 1.f : 0.f, x.y > 0.f ? 1.f : 0.f);
      return at_least(x, 0.f);
    }
    if constexpr (kGelu || kSilu) {
      x = at_least(x, -kCut);
      if constexpr (SLOPE) x = at_most(x, kCut);
      float2 t = x, u = p[0];
      if constexpr (kGelu) {
        t = mul2(x, x);
        u = scaled_p(t);
      }
      const float2 s = sigmoid2(mul2(x, u));
      if constexpr (!SLOPE) return mul2(x, s);
      if constexpr (kGelu) {  // Phi + x phi
        const float2 v = mul2(t, half);
        return fma2(mul2(x, top), make_float2(exp2f(v.x), exp2f(v.y)), s);
      }
      return mul2(s, add2(mul2(x, fma2(s, minus, one)), one));
    }
    return x;
  }
};
// f(activation, derivative or value, something is read) with all of it known to the compiler; a derivative always reads
template <typename F>
__device__ __forceinline__ void with_curve(int act, bool slope, bool read, F &&f) {
  using std::integral_constant;
  using Yes = integral_constant<bool, true>;
  using No = integral_constant<bool, false>;
  auto choose = [&](auto a) {
    if (slope) f(a, Yes(), Yes());
    else if (read) f(a, No(), Yes());
    else f(a, No(), No());
  };
  if (act == BLOSSOM_ACT_RELU) choose(integral_constant<int, BLOSSOM_ACT_RELU>());
  else if (act == BLOSSOM_ACT_GELU) choose(integral_constant<int, BLOSSOM_ACT_GELU>());
  else if (act == BLOSSOM_ACT_SILU) choose(integral_constant<int, BLOSSOM_ACT_SILU>());
  else if (read) f(integral_constant<int, BLOSSOM_ACT_NONE>(), No(), Yes());
  else f(integral_constant<int, BLOSSOM_ACT_NONE>(), No(), No());
}

// ---- a product C[m][n] = sum_k A(m, k) B(n, k) ------------------------------------------------------------
// Element (i, k) of an operand is at i * ld + k (k runs along a row in memory) or at k * ld + i (it runs down the rows).
struct Operand {
  const void *p;
  int64_t ld;
  bool along;
  int there = 0;  // of B: columns that are there, the others count as zeros; 0: all n
  const void *low = nullptr;  // of A: a second part of the same shape that is added to it, or null
};
// What becomes of C.
enum Mode {
  kForward,  // out = act(C + bias) + extra
  kSlope,    // out = extra * act'(C + bias)
  kPlain,    // out = C
  kPartial,  // part[split][m][n] = C in single precision over a part of k; part_bias[..][m]: shares of sum_k A(m, k)
};
struct Epilogue {
  int act = 0;
  const void *bias = nullptr, *extra = nullptr;
  int64_t ld_extra = 0;
  void *out = nullptr, *out_low = nullptr;  // out_low (kSlope): what out's rounding leaves, or null
  int64_t ld_out = 0;
  // kPartial: sums of the splits in `part`; or, of one split, the results in `out`; or neither, the sums over k alone
  float *part = nullptr, *part_bias = nullptr;
  int splits = 1;
  bool first = true;  // of a call's products: it clears the status words
};

// n / by, rounded up (n may be the largest int)
inline int parts_of(int n, int by) { return (int)(((int64_t)n + by - 1) / by); }

constexpr int kMostSlabs = 256;  // of 64 rows in one accumulator of a bf16 product over the rows
// Tensor cores, bf16, any alignment.  No split of k may be empty.
int launch_tc(int kernel_id, Mode mode, const Operand &a, const Operand &b, int m, int n, int k, const Epilogue &e, int32_t *status,
              cudaStream_t st);
// The same of single precision.
int launch_f32(int kernel_id, Mode mode, const Operand &a, const Operand &b, int m, int n, int k, const Epilogue &e, int32_t *status,
               cudaStream_t st);
int f32_splits(int m, int n, int k);
// Into how many splits k goes; parts: of A.
int tc_splits(int m, int n, int k, int parts);
int tc_bias_parts(int m, int n, int k, int parts);  // and the sums over k alone
// Few rows.
constexpr int kFewRows = 16;
struct FewRows {
  int dtype, rows, cols, outs, act;
  const void *x, *weight, *bias;
  int64_t ldx, ldw;
};
int few_shares(int cols, int outs);  // of the outs, for dx
// slope: out is in single precision
int launch_few_forward(const FewRows &f, bool slope, const void *extra, int64_t ld_extra, void *out, int64_t ld_out, int32_t *status,
                       cudaStream_t st);
// g_wide: g is in single precision; part: [shares][rows][cols].  Both clear the status words if they are given them.
int launch_few_backward(const FewRows &f, const void *g, int64_t ldg, bool g_wide, float *part, void *dx, int64_t ld_dx, void *dweight,
                        int64_t ld_dweight, void *dbias, int32_t *status, cudaStream_t st);
// The backward of a narrow layer in one kernel.
struct NarrowBackward {
  int rows, cols, outs, act;
  const void *x, *weight, *bias, *dout;  // x null: neither an activation nor dweight wants it
  const int8_t *codes;    // x in 8 bits instead (without an activation), or null
  const uint8_t *scales;
  int64_t ld_x, ld_weight, ld_dout, ld_dx;
  void *dx;               // null: not wanted, as the next two
  float *part, *part_bias;  // [splits][outs][cols] or turned, [splits][outs]
  int32_t *status;
  bool later;             // a call's first rows came before: the status words stay
};
bool narrow_takes(const NarrowBackward &n);
bool narrow_turned(const NarrowBackward &n);  // part is [splits][cols][outs]
int narrow_splits(int rows);
int launch_narrow(const NarrowBackward &n, cudaStream_t st);
// dweight and dbias (either may be null) from the partial sums of the splits; turned: those are [cols][outs].
int launch_join(int dtype, const float *part, const float *part_bias, int splits, int bias_parts, int outs, int cols, void *dweight,
                int64_t ld, void *dbias, cudaStream_t st, bool turned = false);

}  // namespace linear
}  // namespace blossom
