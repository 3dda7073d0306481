// Products on the tensor cores: what the kernel for matrices of any size and the one for narrow layers share.
#pragma once
#include "linear.cuh"
#include "tc_common.cuh"

namespace blossom {
namespace linear {

constexpr int kSlabRow = 128;  // bytes of 64 elements

// rows x cols elements, ld apart; boxes of 64 columns and box_rows rows.  False if the driver refuses.
bool make_map(CUtensorMap *map, const void *base, int64_t rows, int64_t cols, int64_t ld, int box_rows);
// TMA wants rows 16 bytes apart and less than 2^40; the extents may be odd.
inline bool tma_takes(const void *p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0 && ld < (int64_t)1 << 38; }

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1)
      : "memory");
}

__device__ __forceinline__ void tma_prefetch_2d(const CUtensorMap *map, int c0, int c1) {  // into L2
  asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1)
               : "memory");
}
// One look at a barrier, without a wait.
__device__ __forceinline__ bool mbar_done(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}

// A slab of an operand on its way to shared memory, by plain loads: along: [EXTENT rows of the operand][64 of k], else blocks of 64
// rows of k and 64 of the operand; zeros for what is not there.  A thread has N pieces of 8 numbers; put hands each with its
// place (128-byte swizzle) to f.
template <typename T, int EXTENT, int WARPS, int W>
struct Pieces {
  static constexpr int N = EXTENT * 8 / (32 * WARPS), kDeep = 64;
  rows::Raw<T, W> v[N];
  static __device__ __forceinline__ int row(int tid, int j) { return (tid + 32 * WARPS * j) >> 3; }
  __device__ __forceinline__ void ask(int tid, const T *p, int64_t ld, bool along, int at, int end, int k0, int k_end) {
    const int c = 8 * (tid & 7);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int r = row(tid, j), i = along ? at + r : at + r / kDeep * kDeep + c, k = along ? k0 + c : k0 + r % kDeep;  // the first one's
      const bool there = along ? i < end : k < k_end;
      v[j].load(p + (there ? (along ? (int64_t)i * ld + k : (int64_t)k * ld + i) : 0), there ? (along ? k_end - k : end - i) : 0);
    }
  }
  template <typename F>
  __device__ __forceinline__ void put(int tid, F &&f) const {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int r = row(tid, j);
      f(r * kSlabRow + (((tid & 7) ^ (r & 7)) << 4), v[j].w);
    }
  }
};

// ---- 32 rows x 32 columns between memory and a warp's staging, 32 rows of 64 bytes in shared memory ----
// A lane moves four times 8 columns, of row lane / 4 + 8 j.
__device__ __forceinline__ uint4 *piece(uint8_t *staging, int r, int c) {  // 16 bytes c of row r
  return reinterpret_cast<uint4 *>(staging + r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
}
// At the edges of a matrix, and rows of any alignment: w elements an access.  Out of line: the loops' own instructions have to
// fit the instruction cache.
template <int W>
__device__ __forceinline__ void read_ragged_by(uint8_t *staging, const __nv_bfloat16 *p, int64_t ld, int rows, int cols) {
  const int lane = (int)threadIdx.x & 31, c = 8 * (lane & 3);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int r = (lane >> 2) + 8 * j;
    rows::Raw<__nv_bfloat16, W> x;
    x.load(p + (int64_t)(r < rows ? r : 0) * ld + c, r < rows ? cols - c : 0);
    *piece(staging, r, lane & 3) = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
  }
}
template <int W>
__device__ __forceinline__ void write_ragged_by(uint8_t *staging, __nv_bfloat16 *p, int64_t ld, int rows, int cols) {
  const int lane = (int)threadIdx.x & 31, c = 8 * (lane & 3);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int r = (lane >> 2) + 8 * j;
    if (r >= rows) break;
    const uint4 v = *piece(staging, r, lane & 3);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    __nv_bfloat16 *q = p + (int64_t)r * ld + c;
#pragma unroll
    for (int i = 0; i < 8; i += W) {
      if (c + i >= cols) break;
      if constexpr (W == 8) *reinterpret_cast<uint4 *>(q) = v;
      else if constexpr (W == 4) *reinterpret_cast<uint2 *>(q + i) = make_uint2(w[i / 2], w[i / 2 + 1]);
      else if constexpr (W == 2) *reinterpret_cast<uint32_t *>(q + i) = w[i / 2];
      else *reinterpret_cast<uint16_t *>(q + i) = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
    }
  }
}
static __device__ __noinline__ void read_ragged(uint8_t *staging, const __nv_bfloat16 *p, int64_t ld, int rows, int cols, int w) {
  if (w == 8) read_ragged_by<8>(staging, p, ld, rows, cols);
  else if (w == 4) read_ragged_by<4>(staging, p, ld, rows, cols);
  else if (w == 2) read_ragged_by<2>(staging, p, ld, rows, cols);
  else read_ragged_by<1>(staging, p, ld, rows, cols);
}
static __device__ __noinline__ void write_ragged(uint8_t *staging, __nv_bfloat16 *p, int64_t ld, int rows, int cols, int w) {
  if (w == 8) write_ragged_by<8>(staging, p, ld, rows, cols);
  else if (w == 4) write_ragged_by<4>(staging, p, ld, rows, cols);
  else if (w == 2) write_ragged_by<2>(staging, p, ld, rows, cols);
  else write_ragged_by<1>(staging, p, ld, rows, cols);
}
// The whole block, 16 bytes an access.  p: the lane's piece of its first row; step: 8 rows
__device__ __forceinline__ void write_whole(uint8_t *staging, __nv_bfloat16 *p, int64_t step) {
  const int lane = (int)threadIdx.x & 31;
#pragma unroll
  for (int j = 0; j < 4; ++j) *reinterpret_cast<uint4 *>(p + j * step) = *piece(staging, (lane >> 2) + 8 * j, lane & 3);
}
template <typename F>
__device__ __forceinline__ void with_width(int w, F &&f) {
  using std::integral_constant;
  if (w == 8) f(integral_constant<int, 8>());
  else if (w == 4) f(integral_constant<int, 4>());
  else if (w == 2) f(integral_constant<int, 2>());
  else f(integral_constant<int, 1>());
}
// 16 columns of a warp's 32 rows in single precision to memory, by way of 32 x 17 floats
__device__ __forceinline__ void write_sums(const float (&v)[16], float *t, float *to, int64_t ld, int rows, int cols) {
  const int lane = (int)threadIdx.x & 31, c = lane & 15;
#pragma unroll
  for (int i = 0; i < 16; ++i) t[lane * 17 + i] = v[i];
  __syncwarp();
#pragma unroll
  for (int r = lane >> 4; r < 32; r += 2)
    if (r < rows && c < cols) to[(int64_t)r * ld + c] = t[r * 17 + c];
  __syncwarp();
}

// Of a load of 16 columns that is under way: nothing of them is touched before this.
__device__ __forceinline__ void wait_for(float (&v)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]),
                 "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15])
               :
               : "memory");
}
// two bf16: the curve of (v + bias), plus what was read (READ)
template <bool READ, typename C>
__device__ __forceinline__ uint32_t finish2(const C &curve, float2 v, float2 bias, uint32_t read) {
  float2 y = curve(add2(v, bias));
  if constexpr (READ) y = add2(y, rows::halves(read));
  return tc::pack_bf16(y.x, y.y);
}
// 8 columns
template <bool READ, typename C>
__device__ __forceinline__ uint4 finish8(const C &curve, const float *y, const float *bias, uint4 e) {
  const float4 b0 = *reinterpret_cast<const float4 *>(bias), b1 = *reinterpret_cast<const float4 *>(bias + 4);
  return make_uint4(finish2<READ>(curve, make_float2(y[0], y[1]), make_float2(b0.x, b0.y), e.x),
                    finish2<READ>(curve, make_float2(y[2], y[3]), make_float2(b0.z, b0.w), e.y),
                    finish2<READ>(curve, make_float2(y[4], y[5]), make_float2(b1.x, b1.y), e.z),
                    finish2<READ>(curve, make_float2(y[6], y[7]), make_float2(b1.z, b1.w), e.w));
}
// No further from 0 than 2^120, which no remainder is; what is no number (an infinity's remainder) counts as that as well.
__device__ __forceinline__ uint32_t remainders(uint32_t two) {
  uint32_t r;
  asm("{\n\t.reg .b32 t;\n\tmin.bf16x2 t, %1, %2;\n\tmax.bf16x2 %0, t, %3;\n\t}" : "=r"(r) : "r"(two), "r"(0x7b807b80u), "r"(0xfb80fb80u));
  return r;
}
// 8 columns of dout o act'(v + bias) as a sum of two bf16: the first is returned, `low` is what it leaves
template <typename C>
__device__ __forceinline__ uint4 finish8_parts(const C &curve, const float *y, const float *bias, uint4 read, uint4 &low) {
  const uint32_t d[4] = {read.x, read.y, read.z, read.w};
  uint32_t h[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 b = *reinterpret_cast<const float2 *>(bias + 2 * i);
    const float2 g = mul2(curve(add2(make_float2(y[2 * i], y[2 * i + 1]), b)), rows::halves(d[i]));
    h[i] = tc::pack_bf16(g.x, g.y);
    const float2 f = rows::halves(h[i]);
    l[i] = remainders(tc::pack_bf16(g.x - f.x, g.y - f.y));
  }
  low = make_uint4(l[0], l[1], l[2], l[3]);
  return make_uint4(h[0], h[1], h[2], h[3]);
}

}  // namespace linear
}  // namespace blossom
