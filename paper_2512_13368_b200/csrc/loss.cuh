// Sampled softmax loss: what the kernels over positions (loss_rows.cu) and over items (loss_items.cu) share.
#pragma once
#include "rows.cuh"

namespace blossom {
namespace loss {

using rows::kSMs;
using rows::both;
using rows::Group;
using rows::mul2;

// A row's candidates: numbers of them, and where the strides behind the last one lead, stay far from 2^31, and a running sum of
// exponentials in single precision still grows (it takes no more ones from 2^24 on).
constexpr int kMaxNegatives = (1 << 24) - 1;
constexpr int kMaxCols = 1024, kMaxRowCtas = kSMs * 16, kMmaThreads = 128;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Args {
  int rows, cols, groups, items, n;
  int64_t ignore, sh, st, sdh, sdt;  // strides: hidden, table, dhidden, dtable
  uint32_t sn;                       // negatives
  int idx8, hits;
  const void *targets, *negatives;
};

// LAST: nobody reads it again, and it is the first to leave L2, where the sort's lists stay (131072 x 128 entries: the first
// pass's counts and moves 72 and 125 us, with it 68 and 96).  The forward's reads stay, as the backward comes back for them
// (51200 x 32 entries: counts 15 us against 19).
template <bool LAST = false>
__device__ __forceinline__ int64_t load_id(const void *p, int64_t i, int idx8) {
  const int64_t *wide = static_cast<const int64_t *>(p) + i;
  const int32_t *narrow = static_cast<const int32_t *>(p) + i;
  if (LAST) return idx8 ? __ldcs(reinterpret_cast<const long long *>(wide)) : __ldcs(narrow);
  return idx8 ? *wide : *narrow;
}
// the row's target, or -1 if the row takes no part
__device__ __forceinline__ int valid_target(const Args &a, int64_t t) {
  return (uint64_t)t < (uint64_t)a.items && t != a.ignore ? (int)t : -1;
}
__device__ __forceinline__ int row_target(const Args &a, int row) { return valid_target(a, load_id(a.targets, row, a.idx8)); }
// candidate j >= 1 of a row that takes part, or -1 if it is none
template <bool LAST = false>
__device__ __forceinline__ int64_t load_negative(const Args &a, int row, int j) {
  return load_id<LAST>(a.negatives, (int64_t)((uint64_t)(uint32_t)row * a.sn + (uint32_t)(j - 1)), a.idx8);
}
__device__ __forceinline__ int valid_negative(const Args &a, int target, int64_t i) {
  return (uint64_t)i < (uint64_t)a.items && !(a.hits && i == target) ? (int)i : -1;
}
// candidate j of a row that takes part (j = 0: its target)
template <bool LAST = false>
__device__ __forceinline__ int candidate(const Args &a, int row, int target, int j) {
  return j == 0 ? target : valid_negative(a, target, load_negative<LAST>(a, row, j));
}
// the lane's share of <a, b>
template <int V>
__device__ __forceinline__ float dot(const Group (&a)[V], const Group (&b)[V]) {
  float2 s[2] = {both(0.f), both(0.f)};
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i & 1] = fma2(a[v].p[i], b[v].p[i], s[i & 1]);
  const float2 t = add2(s[0], s[1]);
  return t.x + t.y;
}

// A row over LPC lanes, V times 8 columns a lane: access by access the lanes lie side by side (which columns are whose does not
// matter here), so that narrow accesses of odd rows still touch whole sectors.
template <typename T, int W, typename P>
struct Strip {
  static __device__ __forceinline__ int column(int lane, int v, int j) { return W * (lane + P::LPC * (j / W + v * (8 / W))); }
  static __device__ __forceinline__ rows::Raw<T, W> raw(const T *row, int lane, int v, int cols, bool there = true) {
    rows::Raw<T, W> r;
#pragma unroll
    for (int j = 0; j < 8; j += W) r.piece(row + column(lane, v, j), j, there && column(lane, v, j) < cols);
    return r;
  }
  static __device__ __forceinline__ Group load(const T *row, int lane, int v, int cols, bool there = true) {
    return raw(row, lane, v, cols, there).get();
  }
  static __device__ __forceinline__ void store(T *row, int lane, int v, int cols, const Group &g) {
    Group x = g;
#pragma unroll
    for (int j = 0; j < 8; j += W)
      if (column(lane, v, j) < cols) rows::store_piece<T, W>(row + column(lane, v, j), j, x);
  }
};

// Single-precision sums in the columns that a strip of W elements an access has (of 8: two accesses).
template <int W, typename P>
__device__ __forceinline__ void store_sums(float *row, int lane, int v, int cols, const Group &g) {
  Group x = g;
  constexpr int WF = W < 4 ? W : 4;
#pragma unroll
  for (int j = 0; j < 8; j += WF) {
    const int c = Strip<float, W, P>::column(lane, v, j / W * W) + j % W;
    if (c < cols) rows::store_piece<float, WF>(row + c, j, x);
  }
}
template <int W, typename P>
__device__ __forceinline__ Group load_sums(const float *row, int lane, int v, int cols) {
  rows::Raw<float, (W < 4 ? W : 4)> r;
  constexpr int WF = W < 4 ? W : 4;
#pragma unroll
  for (int j = 0; j < 8; j += WF) {
    const int c = Strip<float, W, P>::column(lane, v, j / W * W) + j % W;
    r.piece(row + c, j, c < cols);
  }
  return r.get();
}

// LPC lanes hold a row, V groups of 8 columns each
template <int LPC_, int V_>
struct Plan {
  static constexpr int LPC = LPC_, V = V_;
};
template <typename F>
inline void with_plan(int groups, F &&f) {
  if (groups <= 4) f(Plan<4, 1>());
  else if (groups <= 8) f(Plan<8, 1>());
  else if (groups <= 16) f(Plan<16, 1>());
  else if (groups <= 32) f(Plan<32, 1>());
  else if (groups <= 64) f(Plan<32, 2>());
  else f(Plan<32, 4>());
}
inline int lanes_of(int groups) { return groups <= 4 ? 4 : groups <= 8 ? 8 : groups <= 16 ? 16 : 32; }

// ---- bf16 rows of up to 64 NL columns on the matrix units ---------------------------------------------
// A warp scores 16 rows against one vector.  L lanes hold a row, kParts times 16 bytes each (side by side: a load takes 64 or 128
// bytes of a row), and of every kStep-th row of the 16.  As the order in which a product's columns are added up is free, a load's
// four registers are the first operand of an m16n8k16 product as they come, without a detour through shared memory or other
// registers: the first and third word are the columns of the product's row lane / 4, the second and fourth those of the row
// 8 behind it.  The vector's words are the second operand, the first and third in even columns, the others in odd ones, so
// that the two sums a lane wants are its first and its last.  With 8 lanes a row its two quads have different columns; the
// vector's then alternate by twos, and what counts is fetched from a lane of either quad.
// (With words of two loads in one operand, which the compiler had to move together, positions of 131072 x 128 x 64 took 285 us
// instead of 271, of 32768 x 128 x 128 140 instead of 128.)
template <int NL, int L>
struct Rows16 {
  static constexpr int kLanes = L, kStep = 32 / L, kRows = L / 2, kParts = 8 * NL / L;  // kRows: of a lane
  uint4 w[kRows][kParts];
};
// Where a lane finds its columns of a row.  Columns that are not there are read as the row's first ones and meet a zero of the
// vector (a row that is no number somewhere is none in its product anyway).
template <int NL, int L, bool FULL>
struct Lanes16 {
  using R = Rows16<NL, L>;
  const char *base;
  uint32_t stride;  // bytes
  uint32_t off[R::kParts];
  __device__ __forceinline__ Lanes16(const __nv_bfloat16 *p, int64_t elements, int cols)
      : base(reinterpret_cast<const char *>(p)), stride((uint32_t)(elements * 2)) {
    const int t = (int)threadIdx.x % L;
    if (FULL) base += 16 * t;
#pragma unroll
    for (int e = 0; e < R::kParts; ++e) off[e] = FULL ? 16 * L * e : 8 * (L * e + t) < cols ? 16 * (L * e + t) : 0;
  }
  __device__ __forceinline__ void load(uint32_t row, uint4 (&w)[R::kParts]) const {
    const char *p = base + (uint64_t)row * stride;
#pragma unroll
    for (int e = 0; e < R::kParts; ++e) w[e] = *reinterpret_cast<const uint4 *>(p + off[e]);
  }
  // rows named by one lane each, `from` on
  __device__ __forceinline__ void load16(uint32_t rows, int from, R &w) const {
    const int q = ((int)threadIdx.x % 32) / L;
#pragma unroll
    for (int j = 0; j < R::kRows; ++j) load(__shfl_sync(0xffffffffu, rows, from + R::kStep * j + q), w.w[j]);
  }
  // the second operand: the lane's words of the vector, zero where there are no columns
  __device__ __forceinline__ void vector(uint32_t row, int cols, uint2 (&w)[R::kParts]) const {
    const int lane = (int)threadIdx.x % 32, t = L == 4 ? lane % 4 : lane / 8 % 2 * 4 + lane % 4, own = FULL ? lane % L : 0;
    const char *p = base + (uint64_t)row * stride - 16 * own;
#pragma unroll
    for (int e = 0; e < R::kParts; ++e) {
      w[e] = make_uint2(0, 0);
      if (FULL || 8 * (L * e + t) < cols) {
        const uint4 q = *reinterpret_cast<const uint4 *>(p + 16 * (L * e + t));
        w[e] = lane & 4 ? make_uint2(q.y, q.w) : make_uint2(q.x, q.z);
      }
    }
  }
};
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                               uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// l[j] = <the lane's row j, v>
template <int NL, int L>
__device__ __forceinline__ void dots16(const Rows16<NL, L> &r, const uint2 (&v)[8 * NL / L], float (&l)[L / 2]) {
  const int from = (int)threadIdx.x & 24;
#pragma unroll
  for (int j = 0; j < r.kRows; ++j) {
    float d[4];
#pragma unroll
    for (int e = 0; e < r.kParts; ++e) {
      const uint4 x = r.w[j][e];
      if (e == 0) mma16816_first(d, x.x, x.y, x.z, x.w, v[e].x, v[e].y);
      else mma16816(d, x.x, x.y, x.z, x.w, v[e].x, v[e].y);
    }
    l[j] = d[0] + d[3];
    if (L == 8) l[j] = __shfl_sync(0xffffffffu, l[j], from) + __shfl_sync(0xffffffffu, l[j], from + 5);
  }
}
// acc += sum_j p[j] * the lane's row j, in single precision (the weights keep their 24 bits)
template <int NL, int L>
__device__ __forceinline__ void weigh16(const Rows16<NL, L> &r, const float (&p)[L / 2], float2 (&acc)[8 * NL / L][4]) {
#pragma unroll
  for (int j = 0; j < r.kRows; ++j) {
    const float2 pp = make_float2(p[j], p[j]);
#pragma unroll
    for (int e = 0; e < r.kParts; ++e) {
      const uint32_t x[4] = {r.w[j][e].x, r.w[j][e].y, r.w[j][e].z, r.w[j][e].w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        acc[e][i] = fma2(pp, make_float2(__uint_as_float(x[i] << 16), __uint_as_float(x[i] & 0xffff0000u)), acc[e][i]);
    }
  }
}
// The sum over the groups of lanes, scattered: two columns a lane and line are left (scattered_column).
template <int NL, int L>
__device__ __forceinline__ void scatter16(const float2 (&acc)[8 * NL / L][4], float2 (&out)[NL]) {
  const bool b4 = threadIdx.x & 16, b3 = threadIdx.x & 8, b2 = threadIdx.x & 4;
  auto exchange = [](bool second, float2 a, float2 b, int o) {  // of two sums one is kept
    const float2 keep = second ? b : a, give = second ? a : b;
    return make_float2(keep.x + __shfl_xor_sync(0xffffffffu, give.x, o), keep.y + __shfl_xor_sync(0xffffffffu, give.y, o));
  };
  if constexpr (L == 4) {
    static_assert(NL == 1, "4 lanes hold a line");
    float2 s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = exchange(b4, acc[0][i], acc[1][i], 16);
    out[0] = exchange(b2, exchange(b3, s[0], s[2], 8), exchange(b3, s[1], s[3], 8), 4);
  } else {
#pragma unroll
    for (int c = 0; c < NL; ++c)
      out[c] = exchange(b3, exchange(b4, acc[c][0], acc[c][2], 16), exchange(b4, acc[c][1], acc[c][3], 16), 8);
  }
}
// the first of the two columns
template <int L>
__device__ __forceinline__ int scattered_column(int c) {
  const int lane = (int)threadIdx.x % 32;
  return L == 4 ? 32 * (lane / 16) + 8 * (lane % 4) + 2 * (lane / 4 % 4) : 64 * c + 8 * (lane % 8) + 2 * (lane / 8);
}
// Lines of 64 columns where the matrix units take the rows (bf16, 16-byte aligned rows of up to 128 columns less than 4 GiB
// apart), else 0.  Against groups of lanes, 131072 x 128 x 64: positions 252 us to 419, items 293 to 589; 32768 x 128 x 128:
// 117 to 204, 211 to 283.
inline int mma_lines(const Args &a, int dtype, int width) {
  if (dtype != BLOSSOM_DTYPE_BF16 || width != 8 || a.cols > 128 || a.sh > 0x7fffffffLL || a.st > 0x7fffffffLL) return 0;
  return a.cols <= 64 ? 1 : 2;
}
// f(lines, all of their columns are there)
template <typename F>
inline void with_lines(int lines, int cols, F &&f) {
  using std::integral_constant;
  auto full = [&](auto n) {
    if (cols == 64 * decltype(n)::value) f(n, integral_constant<bool, true>());
    else f(n, integral_constant<bool, false>());
  };
  if (lines == 1) full(integral_constant<int, 1>());
  else full(integral_constant<int, 2>());
}

// Device scratch; the forward uses `sums` alone.
struct Scratch {
  double2 *sums;                 // [kMaxRowCtas] loss and number of rows of a CTA
  uint32_t *keys[2], *vals[2];   // [entries] item and position (top bit: it is the target) of every candidate, being sorted
  uint32_t *hist, *totals;       // [digits][tiles], [digits]
  uint32_t *range;               // [2][items] where an item's entries start and end in the sorted list; not written for others
  float *part;                   // [spans][2][cols] sums of items that reach over the end of a span
  size_t bytes;
};
constexpr size_t kForwardBytes = BLOSSOM_LOSS_FORWARD_BYTES;
static_assert(kMaxRowCtas * sizeof(double2) <= kForwardBytes, "a sum per CTA");

// The sort's shape: digits of up to 9 bits, the fewest passes that cover every item and the mark of what is none.
struct SortPlan {
  int passes, bits;
  int64_t entries, tiles;
  int chunk;  // sorted entries that a warp or a group of lanes adds up
  int span;   // that a block does
  int64_t spans;
};
constexpr int kSortThreads = 256, kSortPerThread = 16, kTile = kSortThreads * kSortPerThread, kMaxDigits = 512;

SortPlan sort_plan(const Args &a, int lanes, int threads);  // lanes of a group that walks a chunk, threads of a block
Scratch carve(const Args &a, void *base);
// dtable from the candidates, sorted by item; dhidden from grad_hidden; either may be null
int launch_items(const Args &a, int dtype, const void *hidden, const void *table, const float *lse, const float *grad_hidden,
                 const float *grad_loss, void *dhidden, void *dtable, int width, const Scratch &s, cudaStream_t st);

// g / count, the factor of every gradient
__device__ __forceinline__ float grad_scale(const Args &a, const float *lse, const float *grad_loss) {
  const float count = lse[a.rows];
  return count > 0.f ? (grad_loss ? *grad_loss : 1.f) / count : 0.f;
}

}  // namespace loss
}  // namespace blossom
