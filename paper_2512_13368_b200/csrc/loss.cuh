// Sampled softmax loss: what the kernels over positions (loss_rows.cu) and over items (loss_items.cu) share.
#pragma once
#include "rows.cuh"

namespace blossom {
namespace loss {

using rows::kSMs;
using rows::load_group;
using rows::store_group;

constexpr int kMaxCols = 1024, kMaxRowCtas = kSMs * 8;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Args {
  int rows, cols, groups, items, n;
  int64_t ignore, sh, st, sn, sdh, sdt;  // strides: hidden, table, negatives, dhidden, dtable
  int idx8, hits;
  const void *targets, *negatives;
};

__device__ __forceinline__ int64_t load_id(const void *p, int64_t i, int idx8) {
  return idx8 ? static_cast<const int64_t *>(p)[i] : static_cast<const int32_t *>(p)[i];
}
// the row's target, or -1 if the row takes no part
__device__ __forceinline__ int row_target(const Args &a, int row) {
  const int64_t t = load_id(a.targets, row, a.idx8);
  return t >= 0 && t < a.items && t != a.ignore ? (int)t : -1;
}
// candidate j of a row that takes part (j = 0: its target), or -1 if it is none
__device__ __forceinline__ int candidate(const Args &a, int row, int target, int j) {
  if (j == 0) return target;
  const int64_t i = load_id(a.negatives, row * a.sn + (j - 1), a.idx8);
  return i >= 0 && i < a.items && !(a.hits && i == target) ? (int)i : -1;
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

// Device scratch; the forward uses `sums` alone.
struct Scratch {
  double2 *sums;                 // [kMaxRowCtas] loss and number of rows of a CTA
  uint32_t *keys[2], *vals[2];   // [entries] item and position (top bit: it is the target) of every candidate, being sorted
  uint32_t *hist, *totals;       // [digits][tiles], [digits]
  float *part;                   // [chunks][2][cols] sums of items that reach over the end of a chunk
  size_t bytes;
};
constexpr size_t kForwardBytes = BLOSSOM_LOSS_FORWARD_BYTES;
static_assert(kMaxRowCtas * sizeof(double2) <= kForwardBytes, "a sum per CTA");

// The sort's shape: digits of up to 9 bits, the fewest passes that cover every item and the mark of what is none.
struct SortPlan {
  int passes, bits;
  int64_t entries, tiles;
  int chunk;  // sorted entries that a group of lanes adds up
  int64_t chunks;
};
constexpr int kSortThreads = 512, kSortPerThread = 16, kTile = kSortThreads * kSortPerThread, kMaxDigits = 512;

SortPlan sort_plan(const Args &a);
Scratch carve(const Args &a, void *base);
// dtable from the candidates, sorted by item
int launch_items(const Args &a, int dtype, const void *hidden, const void *table, const float *lse, const float *grad_loss,
                 void *dtable, int width, const Scratch &s, cudaStream_t st);

// g / count, the factor of every gradient
__device__ __forceinline__ float grad_scale(const Args &a, const float *lse, const float *grad_loss) {
  const float count = lse[a.rows];
  return count > 0.f ? (grad_loss ? *grad_loss : 1.f) / count : 0.f;
}

}  // namespace loss
}  // namespace blossom
