// Sampled softmax loss, the part over items: dtable[i] = g / count * sum over the candidates (t, j) that are item i of
// (p_tj - [j is the target]) * hidden_t.
//
// The candidates are sorted by item (a stable radix sort of (item, position) pairs, so that an item's positions come in
// the same order every time), then groups of lanes walk equal chunks of the sorted list: the item's row of the table stays
// in registers, each position's hidden row is read once for both the logit that is formed again and the sum.  An item
// whose entries lie in one chunk is written there and then; the sums of others go to scratch, one a chunk, and are
// added up in order.  No atomics on sums: every one has a fixed order whatever the popularity of the items.
#include <float.h>

#include "loss.cuh"

namespace blossom {
namespace loss {
namespace {

// Up to so many tiles a block of the second kernel adds their counts up itself, instead of a kernel in between (whole step at 4
// tiles 46 us against 51, at 16 58 against 56, at 64 120 against 76).
constexpr int kTilesWithoutScan = 8;

// ---- the sort ------------------------------------------------------------------------------------
// Bound: each pass reads the keys twice and the list once and writes it once: 131072 x 128 entries of 50001 items, two passes,
// 0.9 GB, 140 us at the rate of a copy.  It takes 310 us: counts 68 (with the keys made from 134 MB of ids) and 23, scans 10,
// moves 97 each (issue slots 55 - 61 % busy: eight ballots an entry find the lanes of the same digit, and 64 registers leave
// half of an SM's warps; a warp's match instruction took longer than the ballots).  Tiles of 4096 entries in 256 threads.
// Entry e of the unsorted list is candidate e % (n + 1) of position e / (n + 1); what is no candidate gets the item
// number `items` and ends up behind all others.
struct Split {  // e / (n + 1) for e < 2^31: a product and a shift
  uint32_t mul, shift;
  __device__ __forceinline__ uint32_t operator()(uint32_t e) const { return (uint32_t)((uint64_t)e * mul >> shift); }
};
inline Split split_by(uint32_t d) {
  int l = 0;
  while (((uint64_t)1 << l) < d) ++l;
  return Split{(uint32_t)((((uint64_t)1 << (31 + l)) + d - 1) / d), (uint32_t)(31 + l)};
}
__device__ __forceinline__ uint32_t entry_val(const Args &a, const Split &by, uint32_t e) {
  const uint32_t t = by(e);
  return t | (e == t * (uint32_t)(a.n + 1) ? 0x80000000u : 0u);
}

// Counts of a tile's digits, to hist[digit][tile].  The first pass makes the keys.  Issue slots 66 - 72 % busy.
template <bool FIRST>
__global__ void __launch_bounds__(kSortThreads, 8) sort_count_kernel(Args a, Split by, uint32_t *__restrict__ keys, uint32_t entries,
                                                                  int shift, int bits, uint32_t *__restrict__ hist) {
  __shared__ uint32_t count[kMaxDigits];
  __shared__ int targets[FIRST ? kTile + 1 : 1];  // of the positions that the tile belongs to
  grid_chain_enter();
  const int digits = 1 << bits, tid = (int)threadIdx.x;
  const uint32_t mask = (uint32_t)digits - 1, none = (uint32_t)a.items, tile0 = blockIdx.x * (uint32_t)kTile;
  for (int d = tid; d < digits; d += kSortThreads) count[d] = 0;
  uint32_t t0 = 0;
  if (FIRST) {
    t0 = by(tile0);
    const uint32_t last = by((entries - tile0 < (uint32_t)kTile ? entries : tile0 + kTile) - 1);
    for (uint32_t t = t0 + (uint32_t)tid; t <= last; t += kSortThreads) targets[t - t0] = row_target(a, (int)t);
  }
  __syncthreads();
  uint32_t key[kSortPerThread];
#pragma unroll
  for (int r = 0; r < kSortPerThread; ++r) {
    const uint32_t e = tile0 + (uint32_t)tid + kSortThreads * r;
    key[r] = none;
    if (e < entries) {
      if (FIRST) {
        const uint32_t t = by(e);
        const int target = targets[t - t0];
        if (target >= 0) key[r] = (uint32_t)candidate<true>(a, (int)t, target, (int)(e - t * (uint32_t)(a.n + 1)));
        key[r] = min(key[r], none);  // (-1: no candidate)
      } else {
        key[r] = keys[e];
      }
    }
  }
#pragma unroll
  for (int r = 0; r < kSortPerThread; ++r) {
    const uint32_t e = tile0 + (uint32_t)tid + kSortThreads * r;
    const bool there = e < entries, padding = there && key[r] == none;
    if (FIRST && there) keys[e] = key[r];
    // (padding comes in long runs of one key: one addition a warp; items are mostly different ones)
    const uint32_t pads = __ballot_sync(0xffffffffu, padding);
    if (padding && tid % 32 == __ffs(pads) - 1) atomicAdd(&count[none >> shift & mask], (uint32_t)__popc(pads));
    if (there && !padding) atomicAdd(&count[key[r] >> shift & mask], 1u);
  }
  __syncthreads();
  for (int d = tid; d < digits; d += kSortThreads) hist[(size_t)d * gridDim.x + blockIdx.x] = count[d];
}

// Sum over the threads before this one of a block of kSortThreads, and the block's total.
__device__ __forceinline__ uint32_t block_prefix(uint32_t v, uint32_t *warp_totals, uint32_t *total) {
  const int lane = (int)threadIdx.x % 32, warp = (int)threadIdx.x / 32;
  uint32_t s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t x = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += x;
  }
  if (lane == 31) warp_totals[warp] = s;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kSortThreads / 32; ++i) {
    const uint32_t x = warp_totals[i];
    before += i < warp ? x : 0;
    all += x;
  }
  __syncthreads();
  *total = all;
  return before + s - v;
}

// hist[digit][*] becomes the number of the digit's entries in the tiles before; totals[digit] that in all of them.
__global__ void __launch_bounds__(kSortThreads) sort_scan_kernel(uint32_t *__restrict__ hist, int tiles,
                                                                 uint32_t *__restrict__ totals) {
  constexpr int PER = 8;  // counts a thread, one after another
  __shared__ uint32_t warp_totals[kSortThreads / 32];
  grid_chain_enter();
  uint32_t *h = hist + (size_t)blockIdx.x * tiles, carry = 0, total;
  for (int i0 = 0; i0 < tiles; i0 += kSortThreads * PER) {
    const int i = i0 + (int)threadIdx.x * PER;
    uint32_t v[PER], sum = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      v[k] = i + k < tiles ? h[i + k] : 0;
      sum += v[k];
    }
    uint32_t before = carry + block_prefix(sum, warp_totals, &total);
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      if (i + k < tiles) h[i + k] = before;
      before += v[k];
    }
    carry += total;
  }
  if (threadIdx.x == 0) totals[blockIdx.x] = carry;
}

// Lanes that hold the same digit as this one, among those that hold any: one ballot a bit.
template <int BITS>
__device__ __forceinline__ uint32_t same_digit(uint32_t d, bool there) {
  uint32_t peers = __ballot_sync(0xffffffffu, there);
#pragma unroll
  for (int b = 0; b < BITS; ++b) {
    const bool bit = d >> b & 1;
    const uint32_t v = __ballot_sync(0xffffffffu, bit);
    peers &= bit ? v : ~v;
  }
  return peers;
}

// A tile's entries to their places, in order: ranks within a warp by matching digits, then warps, then digits; the tile is put
// in order in shared memory first, so that it leaves in runs.  FIRST: the values are made here.  totals null: there are
// few tiles, whose counts are added up here instead of by a kernel in between.
template <int BITS, bool FIRST>
__global__ void __launch_bounds__(kSortThreads, 4) sort_move_kernel(Args a, Split by, const uint32_t *__restrict__ keys,
                                                                    const uint32_t *__restrict__ vals, uint32_t entries,
                                                                    int shift, const uint32_t *__restrict__ hist,
                                                                    const uint32_t *__restrict__ totals,
                                                                    uint32_t *__restrict__ keys_out,
                                                                    uint32_t *__restrict__ vals_out) {
  constexpr int NW = kSortThreads / 32, digits = 1 << BITS, DPT = digits > kSortThreads ? digits / kSortThreads : 1;
  constexpr uint32_t mask = (uint32_t)digits - 1;
  extern __shared__ uint32_t sm[];
  uint32_t *sk = sm, *sv = sm + kTile, *offset = sm + 2 * kTile;
  uint16_t *count = reinterpret_cast<uint16_t *>(offset + digits);  // [warp][digit]
  __shared__ uint32_t warp_totals[NW];
  grid_chain_enter();
  const int tid = (int)threadIdx.x, lane = tid % 32, warp = tid / 32;
  for (int i = tid; i < NW * digits; i += kSortThreads) count[i] = 0;
  __syncthreads();
  const uint32_t tile0 = blockIdx.x * (uint32_t)kTile, e0 = tile0 + (uint32_t)warp * (32 * kSortPerThread) + (uint32_t)lane;
  uint32_t key[kSortPerThread], rank[kSortPerThread / 2];  // (two ranks a word)
#pragma unroll
  for (int r = 0; r < kSortPerThread; ++r) {
    const uint32_t e = e0 + 32 * r;  // (read for the last time, see load_id)
    key[r] = e < entries ? __ldcs(keys + e) : 0;
  }
  uint16_t *mine = count + warp * digits;
#pragma unroll
  for (int r = 0; r < kSortPerThread; ++r) {
    const bool there = e0 + 32 * r < entries;
    const uint32_t d = key[r] >> shift & mask;
    const uint32_t peers = same_digit<BITS>(d, there), below = peers & ((1u << lane) - 1);
    const uint32_t at = there ? mine[d] + (uint32_t)__popc(below) : 0;
    rank[r / 2] = r % 2 ? rank[r / 2] | at << 16 : at;
    __syncwarp();
    if (there && below == 0) mine[d] = (uint16_t)(at + __popc(peers));
    __syncwarp();
  }
  __syncthreads();
  // the thread's digits: their entries in the warps before, in the tile, and where they go
  const int d0 = tid * DPT;
  uint32_t in_tile[DPT], sum = 0, all;
#pragma unroll
  for (int k = 0; k < DPT; ++k) {
    in_tile[k] = 0;
    if (d0 < digits)
      for (int w = 0; w < NW; ++w) {
        const uint32_t c = count[w * digits + d0 + k];
        count[w * digits + d0 + k] = (uint16_t)in_tile[k];
        in_tile[k] += c;
      }
    sum += in_tile[k];
  }
  uint32_t tile_base = block_prefix(sum, warp_totals, &all);
  uint32_t total[DPT], before[DPT];  // in all tiles, in the tiles before
  sum = 0;
#pragma unroll
  for (int k = 0; k < DPT; ++k) {
    total[k] = before[k] = 0;
    if (d0 < digits) {
      const uint32_t *h = hist + (size_t)(d0 + k) * gridDim.x;
      if (totals) {
        total[k] = totals[d0 + k], before[k] = h[blockIdx.x];
      } else {
#pragma unroll 8
        for (unsigned i = 0; i < gridDim.x; ++i) {
          const uint32_t c = h[i];
          total[k] += c;
          before[k] += i < blockIdx.x ? c : 0;
        }
      }
    }
    sum += total[k];
  }
  uint32_t global_base = block_prefix(sum, warp_totals, &all);
  if (d0 < digits)
#pragma unroll
    for (int k = 0; k < DPT; ++k) {
      const int d = d0 + k;
      for (int w = 0; w < NW; ++w) count[w * digits + d] += (uint16_t)tile_base;
      offset[d] = global_base + before[k] - tile_base;
      tile_base += in_tile[k];
      global_base += total[k];
    }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kSortPerThread; ++r)
    if (e0 + 32 * r < entries) {
      const uint32_t at = mine[key[r] >> shift & mask] + (r % 2 ? rank[r / 2] >> 16 : rank[r / 2] & 0xffffu);
      sk[at] = key[r];
      sv[at] = FIRST ? e0 + 32 * r : __ldcs(vals + e0 + 32 * r);
    }
  __syncthreads();
  const uint32_t here = entries - tile0 < (uint32_t)kTile ? entries - tile0 : (uint32_t)kTile;
  for (uint32_t i = (uint32_t)tid; i < here; i += kSortThreads) {
    const uint32_t k = sk[i], at = offset[k >> shift & mask] + i;
    keys_out[at] = k;
    vals_out[at] = FIRST ? entry_val(a, by, sv[i]) : sv[i];
  }
}

// Few entries: the whole sort in one block, in shared memory, instead of in four launches and more (up to 8192: 25 us against
// 45; 4096: 19 against 42; 256: 15 against 35).  Bound: the latency of its steps.
constexpr int kSmallThreads = 1024, kSmallPerThread = 8, kSmallEntries = kSmallThreads * kSmallPerThread, kSmallBits = 8;
constexpr size_t kSmallSmem = 2 * kSmallEntries * sizeof(uint32_t) + ((kSmallThreads / 32) << kSmallBits) * sizeof(uint16_t);
__global__ void __launch_bounds__(kSmallThreads) sort_small_kernel(Args a, Split by, uint32_t entries, int passes,
                                                                   uint32_t *__restrict__ keys_out,
                                                                   uint32_t *__restrict__ vals_out) {
  constexpr int digits = 1 << kSmallBits;
  extern __shared__ uint32_t sm[];
  uint32_t *sk = sm, *sv = sm + kSmallEntries;
  uint16_t *count = reinterpret_cast<uint16_t *>(sm + 2 * kSmallEntries);  // [warp][digit]
  __shared__ uint32_t warp_totals[digits / 32];
  grid_chain_enter();
  const int tid = (int)threadIdx.x, lane = tid % 32, warp = tid / 32;
  const uint32_t e0 = (uint32_t)warp * (32 * kSmallPerThread) + (uint32_t)lane, none = (uint32_t)a.items;
  uint32_t key[kSmallPerThread], val[kSmallPerThread], rank[kSmallPerThread];
#pragma unroll
  for (int r = 0; r < kSmallPerThread; ++r) {
    const uint32_t e = e0 + 32 * r;
    key[r] = none, val[r] = 0;
    if (e < entries) {
      const uint32_t t = by(e);
      const int target = row_target(a, (int)t);
      if (target >= 0) key[r] = min((uint32_t)candidate<true>(a, (int)t, target, (int)(e - t * (uint32_t)(a.n + 1))), none);
      val[r] = entry_val(a, by, e);
    }
  }
  uint16_t *mine = count + warp * digits;
  const int nw = (int)((entries + 32 * kSmallPerThread - 1) / (32 * kSmallPerThread));  // warps that have entries
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * kSmallBits;
    for (int i = tid; i < nw * digits; i += kSmallThreads) count[i] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSmallPerThread; ++r) {
      if (warp >= nw) break;
      const bool there = e0 + 32 * r < entries;
      const uint32_t d = key[r] >> shift & (digits - 1);
      const uint32_t peers = same_digit<kSmallBits>(d, there), below = peers & ((1u << lane) - 1);
      rank[r] = mine[d] + (uint32_t)__popc(below);
      __syncwarp();
      if (there && below == 0) mine[d] = (uint16_t)(rank[r] + __popc(peers));
      __syncwarp();
    }
    __syncthreads();
    // a digit's entries in the warps before, and in the digits before
    uint32_t sum = 0, s = 0;
    if (tid < digits) {
      for (int w = 0; w < nw; ++w) {
        const uint32_t c = count[w * digits + tid];
        count[w * digits + tid] = (uint16_t)sum;
        sum += c;
      }
      s = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += x;
      }
      if (lane == 31) warp_totals[warp] = s;
    }
    __syncthreads();
    if (tid < digits) {
      s -= sum;
      for (int w = 0; w < warp; ++w) s += warp_totals[w];
      for (int w = 0; w < nw; ++w) count[w * digits + tid] += (uint16_t)s;  // (at most kSmallEntries)
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSmallPerThread; ++r)
      if (e0 + 32 * r < entries) {
        const uint32_t at = mine[key[r] >> shift & (digits - 1)] + rank[r];
        sk[at] = key[r];
        sv[at] = val[r];
      }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSmallPerThread; ++r)
      if (e0 + 32 * r < entries) key[r] = sk[e0 + 32 * r], val[r] = sv[e0 + 32 * r];
  }
#pragma unroll
  for (int r = 0; r < kSmallPerThread; ++r)
    if (e0 + 32 * r < entries) keys_out[e0 + 32 * r] = key[r], vals_out[e0 + 32 * r] = val[r];
}

using MoveKernel = void (*)(Args, Split, const uint32_t *, const uint32_t *, uint32_t, int, const uint32_t *, const uint32_t *,
                            uint32_t *, uint32_t *);
template <bool FIRST>
MoveKernel move_kernel(int bits) {
  static const MoveKernel k[9] = {sort_move_kernel<1, FIRST>, sort_move_kernel<2, FIRST>, sort_move_kernel<3, FIRST>,
                                  sort_move_kernel<4, FIRST>, sort_move_kernel<5, FIRST>, sort_move_kernel<6, FIRST>,
                                  sort_move_kernel<7, FIRST>, sort_move_kernel<8, FIRST>, sort_move_kernel<9, FIRST>};
  return k[bits - 1];
}
constexpr size_t move_smem(int bits) {
  return 2 * kTile * sizeof(uint32_t) + ((size_t)1 << bits) * (sizeof(uint32_t) + kSortThreads / 32 * sizeof(uint16_t));
}

// ---- sums over an item's entries ---------------------------------------------------------------
// Bound: the hidden rows come from L2, one an entry.  131072 x 128 entries x 64 bf16: 2.1 GB in 290 us, 7.4 TB/s, with 65 % of the
// issue slots busy; 32768 x 128 x 128 with 25 entries an item: 211 us; fp32, 12795 x 100 x 50: 68 us.
// A block's groups of lanes (or warps) walk consecutive chunks, together a span of the list.  An item whose entries lie in one
// chunk is written there and then.  The others' sums meet in shared memory: a group leaves that of its first item there if
// the item began before its chunk, and the group in whose chunk an item began adds up those of the groups behind it.
// What reaches over the span's ends goes to scratch, at most two sums a span: [0] of the span's first item if it began
// before the span or at its start, [1] of its last item if that began inside.
constexpr int kThreads = 256, kItemsPerGroup = 2, kDense = 12;

template <int NG>
struct Ends {  // of every group's chunk
  uint32_t first[NG];  // its first item
  bool through[NG];    // that is its only one and goes on behind it
};
// Adds the sums of the groups g, g + 1, ... that belong to `item`; true if the item ends in one of them.
template <int NG, typename ADD>
__device__ __forceinline__ bool add_groups(const Ends<NG> &ends, int g, uint32_t item, ADD &&add) {
  for (; g < NG; ++g) {
    if (ends.first[g] != item) return true;
    add(g);
    if (!ends.through[g]) return true;
  }
  return false;
}

template <typename T, int W, typename P>
__global__ void __launch_bounds__(kThreads, P::V == 1 ? (sizeof(T) == 2 ? 4 : 3) : P::V == 2 ? 2 : 1)
    loss_items_kernel(Args a, const T *__restrict__ hidden, const T *__restrict__ table, const float *__restrict__ lse,
                      const float *__restrict__ grad_loss, const uint32_t *__restrict__ keys, const uint32_t *__restrict__ vals,
                      uint32_t entries, int chunk, T *__restrict__ dtable, float *__restrict__ part,
                      uint32_t *__restrict__ range) {
  using S = Strip<T, W, P>;
  constexpr int LPC = P::LPC, V = P::V, NG = kThreads / LPC;
  __shared__ float shared_sums[NG][V * 8][LPC];
  __shared__ Ends<NG> ends;
  grid_chain_enter();
  const int col = (int)threadIdx.x % LPC, base = (int)threadIdx.x % 32 / LPC * LPC;
  const uint32_t lanes = LPC == 32 ? 0xffffffffu : ((1u << LPC) - 1) << base;
  const int grp = (int)threadIdx.x / LPC;
  const uint32_t none = (uint32_t)a.items;
  const uint64_t start = ((uint64_t)blockIdx.x * NG + grp) * (uint32_t)chunk;
  const uint32_t s = start < entries ? (uint32_t)start : entries, e = entries - s < (uint32_t)chunk ? entries : s + (uint32_t)chunk;
  const float scale = grad_scale(a, lse, grad_loss);
  uint32_t cur = s < entries ? keys[s] : none;
  const uint32_t before = s > 0 ? keys[s - 1] : none;
  const bool open = cur < none && before == cur;  // the first item's entries began in a chunk before
  bool first = true, closed = cur >= none;         // closed: what follows is no candidate
  const bool writer = col == 0;
  Group acc[V], own[V];
  auto begin = [&](uint32_t item) {
    cur = item;
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[v].p[i] = both(0.f);
    }
  };
  auto write = [&](uint32_t item) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[v].p[i] = mul2(acc[v].p[i], both(scale));
      S::store(dtable + item * a.sdt, col, v, a.cols, acc[v]);
    }
  };
  auto leave = [&](int slot) {
#pragma unroll
    for (int v = 0; v < V; ++v) store_sums<W, P>(part + ((int64_t)blockIdx.x * 2 + slot) * a.cols, col, v, a.cols, acc[v]);
  };
  auto share = [&]() {
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) shared_sums[grp][8 * v + i][col] = acc[v].at(i);
  };
  auto add = [&](int g) {
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[v].at(i) += shared_sums[g][8 * v + i][col];
  };
  if (writer) {
    if (s > 0 && s < entries && !open && before < none) range[none + before] = s;
    if (!closed && !open) range[cur] = s;
    ends.first[grp] = cur;
  }
  if (!closed) begin(cur);
  // LPC entries, one a lane: the positions' log-sum-exps are asked for LPC entries after the positions (whoever asks at once
  // waits for the positions to come)
  struct Entries {
    uint32_t key, val;
    float top;
    __device__ __forceinline__ void ask(const float *lse) { top = lse[val & 0x7fffffffu]; }
  };
  auto entries_from = [&](uint32_t i) {
    Entries x = {none, 0, 0.f};
    if (i + col < e) x.key = keys[i + col], x.val = vals[i + col];
    return x;
  };
  // The next entry's hidden row is under way, and with it the table's where a new item begins: one that waited for its item would
  // be a memory latency in front of every item.  (More rows ahead in more registers were slower than more warps: 51180 x 100
  // candidates x 64 fp32 313 us with four rows and 16 warps an SM, 203 with one and 32.)
  rows::Raw<T, W> h[V], w[V];
  bool fresh;
  uint32_t last = none;  // the item of the entry loaded last
  auto load = [&](uint32_t key, uint32_t val) {
    fresh = key != last && key < none;
    last = key;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      h[v] = S::raw(hidden + (int64_t)(val & 0x7fffffffu) * a.sh, col, v, a.cols, key < none);
      if (fresh) w[v] = S::raw(table + key * a.st, col, v, a.cols);
    }
  };
  Entries x = entries_from(s), next = entries_from(s + LPC);
  x.ask(lse);
  load(__shfl_sync(lanes, x.key, base), __shfl_sync(lanes, x.val, base));
  for (uint32_t i0 = s; i0 < e && !closed; i0 += LPC) {
    next.ask(lse);
    const Entries third = entries_from(i0 + 2 * LPC);
#pragma unroll 1
    for (int k = 0; k < LPC && i0 + k < e; ++k) {
      const uint32_t key = __shfl_sync(lanes, x.key, base + k), val = __shfl_sync(lanes, x.val, base + k);
      const float top = __shfl_sync(lanes, x.top, base + k);
      if (key != cur) {
        if (first && open) share();
        else write(cur);
        first = false;
        if (writer) range[none + cur] = i0 + k;
        closed = key >= none;
        if (closed) break;
        if (writer) range[key] = i0 + k;
        begin(key);
      }
      Group hg[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (fresh) own[v] = w[v].get();
        hg[v] = h[v].get();
      }
      const bool wrap = k + 1 == LPC;
      load(__shfl_sync(lanes, wrap ? next.key : x.key, base + (wrap ? 0 : k + 1)),
           __shfl_sync(lanes, wrap ? next.val : x.val, base + (wrap ? 0 : k + 1)));
      float l = dot<V>(own, hg);
#pragma unroll
      for (int o = 1; o < LPC; o <<= 1) l += __shfl_xor_sync(lanes, l, o);
      const float coef = exp2f((l - top) * kLog2e) - (val >> 31 ? 1.f : 0.f);
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[v].p[j] = fma2(both(coef), hg[v].p[j], acc[v].p[j]);
    }
    x = next;
    next = third;
  }
  const bool goes_on = !closed && e < entries && keys[e] == cur;
  if (!closed) {
    if (first && open) share();
    else if (!goes_on) write(cur);
    if (writer && e == entries) range[none + cur] = e;
  }
  if (writer) ends.through[grp] = first && goes_on;
  __syncthreads();
  if (goes_on && !(first && open)) {  // the item began in this chunk
    if (add_groups<NG>(ends, grp + 1, cur, add)) write(cur);
    else leave(grp == 0 && first ? 0 : 1);
  }
  if (grp == 0 && open) {  // the span's first item began before it
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[v].p[i] = both(0.f);
    add_groups<NG>(ends, 0, ends.first[0], add);
    leave(0);
  }
}

// The same on the matrix units: a warp walks a chunk 16 entries at a time, their hidden rows the first operand, the item's
// row the second.  Sixteen entries of more than one item go through once an item, so it pays from kDense entries an item on
// (16384 x 64 entries, against entry by entry: 8 an item 66 us to 57, with 128 columns 113 to 89; 16 an item 49 to 55, 78 to
// 82; 32 an item 39 to 54, 60 to 80).  Blocks an SM: 7 and, with 128 columns, 4 (8 and 5: 291 us as with 7, 254 against 223).
template <int NL, bool FULL>
__global__ void __launch_bounds__(kMmaThreads, NL == 1 ? 7 : 4)
    loss_items_mma_kernel(Args a, const __nv_bfloat16 *__restrict__ hidden, const __nv_bfloat16 *__restrict__ table,
                          const float *__restrict__ lse, const float *__restrict__ grad_loss, const uint32_t *__restrict__ keys,
                          const uint32_t *__restrict__ vals, uint32_t entries, int chunk, __nv_bfloat16 *__restrict__ dtable,
                          float *__restrict__ part, uint32_t *__restrict__ range) {
  constexpr int L = 8;  // lanes a row (4 of 64 columns in 80 registers: 295 us as well)
  using R = Rows16<NL, L>;
  constexpr int NG = kMmaThreads / 32;
  __shared__ float2 shared_sums[NG][NL][32];
  __shared__ Ends<NG> ends;
  grid_chain_enter();
  const int lane = (int)threadIdx.x % 32, group = lane / R::kLanes, warp = (int)threadIdx.x / 32;
  const uint32_t none = (uint32_t)a.items;
  const uint64_t start = ((uint64_t)blockIdx.x * NG + warp) * (uint32_t)chunk;
  const uint32_t s = start < entries ? (uint32_t)start : entries, e = entries - s < (uint32_t)chunk ? entries : s + (uint32_t)chunk;
  const Lanes16<NL, L, FULL> from_hidden(hidden, a.sh, a.cols), from_table(table, a.st, a.cols);
  const float scale = grad_scale(a, lse, grad_loss);
  // 32 entries, one a lane; what lies behind the chunk is no candidate of the first position.  The positions' log-sum-exps are
  // asked for 32 entries after the positions (whoever asks at once waits for the positions to come).
  struct Entries {
    uint32_t key, val;
    float top;
    __device__ __forceinline__ void ask(const float *lse) { top = lse[val & 0x7fffffffu]; }
  };
  auto entries_from = [&](uint32_t i) {
    Entries x = {none, 0, 0.f};
    if (i + lane < e) x.key = keys[i + lane], x.val = vals[i + lane];
    return x;
  };
  uint2 w[R::kParts];
  float2 acc[R::kParts][4];
  uint32_t cur = s < entries ? keys[s] : none, before = s > 0 ? keys[s - 1] : 0xffffffffu;
  const bool open = cur < none && before == cur;  // the first item's entries began in a chunk before
  bool first = true;
  auto begin = [&](uint32_t item) {
    cur = item;
    from_table.vector(item, a.cols, w);
#pragma unroll
    for (int e = 0; e < R::kParts; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[e][i] = make_float2(0.f, 0.f);
  };
  auto write = [&](const float2 (&sum)[NL]) {
#pragma unroll
    for (int c = 0; c < NL; ++c) {
      const int col = scattered_column<L>(c);
      if (FULL || col < a.cols)
        *reinterpret_cast<uint32_t *>(dtable + cur * a.sdt + col) = rows::pack2(sum[c].x * scale, sum[c].y * scale);
    }
  };
  auto leave = [&](const float2 (&sum)[NL], int slot) {
#pragma unroll
    for (int c = 0; c < NL; ++c) {
      const int col = scattered_column<L>(c);
      if (FULL || col < a.cols) *reinterpret_cast<float2 *>(part + ((int64_t)blockIdx.x * 2 + slot) * a.cols + col) = sum[c];
    }
  };
  auto share = [&](const float2 (&sum)[NL]) {
#pragma unroll
    for (int c = 0; c < NL; ++c) shared_sums[warp][c][lane] = sum[c];
  };
  auto finish = [&]() {
    float2 sum[NL];
    scatter16<NL, L>(acc, sum);
    if (first && open) share(sum);
    else write(sum);
    first = false;
  };
  // where items start and end, from 32 entries and the key before them
  auto mark = [&](const Entries &x, uint32_t i) {
    uint32_t left = __shfl_up_sync(0xffffffffu, x.key, 1);
    if (lane == 0) left = before;
    if (i + lane < e) {
      if (x.key != left) {
        if (x.key < none) range[x.key] = i + lane;
        if (left < none) range[none + left] = i + lane;
      }
      if (i + lane + 1 == entries && x.key < none) range[none + x.key] = entries;
    }
    before = __shfl_sync(0xffffffffu, x.key, 31);
  };
  auto walk = [&](const R &h, const Entries &x, int half) {
    const float minus = -x.top * kLog2e;
    float shift[R::kRows];
#pragma unroll
    for (int j = 0; j < R::kRows; ++j) shift[j] = __shfl_sync(0xffffffffu, minus, half + R::kStep * j + group);
    const uint32_t targets = __ballot_sync(0xffffffffu, x.val >> 31) >> half & 0xffffu;
    for (;;) {
      float p[R::kRows];
      dots16<NL, L>(h, w, p);
#pragma unroll
      for (int j = 0; j < R::kRows; ++j) p[j] = exp2f(fmaf(p[j], kLog2e, shift[j]));
      if (targets) {  // (the same for the warp)
#pragma unroll
        for (int j = 0; j < R::kRows; ++j) p[j] -= targets >> (R::kStep * j + group) & 1 ? 1.f : 0.f;
      }
      uint32_t others = __ballot_sync(0xffffffffu, x.key != cur) >> half & 0xffffu;
      if (!others) {
        weigh16<NL, L>(h, p, acc);
        return;
      }
      // (a weight of zero would not do: another item's row may hold what is no number)
      others >>= group;
      R own = h;
#pragma unroll
      for (int j = 0; j < R::kRows; ++j)
        if (others >> (R::kStep * j) & 1) {
          p[j] = 0.f;
#pragma unroll
          for (int e = 0; e < R::kParts; ++e) own.w[j][e] = make_uint4(0, 0, 0, 0);
        }
      weigh16<NL, L>(own, p, acc);
      // the next item among the 16, if there is one (they are sorted)
      const uint32_t later = __ballot_sync(0xffffffffu, (lane & 16) == half && x.key > cur && x.key < none);
      if (!later) return;
      finish();
      begin(__shfl_sync(0xffffffffu, x.key, __ffs(later) - 1));
    }
  };
  const bool some = cur < none;  // (else there is no candidate here)
  if (lane == 0) ends.first[warp] = cur;
  Entries x = entries_from(s), next = entries_from(s + 32);
  x.ask(lse);
  mark(x, s);
  float2 sum[NL];
  bool goes_on = false;
  if (some) {
    begin(cur);
    R h;
    for (uint32_t i = s; i < e; i += 32) {
      from_hidden.load16(x.val & 0x7fffffffu, 0, h);
      next.ask(lse);
      const Entries after = entries_from(i + 64);
      walk(h, x, 0);
      if (i + 16 < e) {
        from_hidden.load16(x.val & 0x7fffffffu, 16, h);
        walk(h, x, 16);
      }
      if (i + 32 < e) mark(next, i + 32);
      x = next;
      next = after;
    }
    goes_on = e < entries && keys[e] == cur;
    scatter16<NL, L>(acc, sum);
    if (first && open) share(sum);
    else if (!goes_on) write(sum);
  }
  if (lane == 0) ends.through[warp] = first && goes_on;
  __syncthreads();
  auto add = [&](int g) {
#pragma unroll
    for (int c = 0; c < NL; ++c) sum[c] = add2(sum[c], shared_sums[g][c][lane]);
  };
  if (goes_on && !(first && open)) {  // the item began in this chunk
    if (add_groups<NG>(ends, warp + 1, cur, add)) write(sum);
    else leave(sum, warp == 0 && first ? 0 : 1);
  }
  if (warp == 0 && open && some) {  // the span's first item began before it
#pragma unroll
    for (int c = 0; c < NL; ++c) sum[c] = make_float2(0.f, 0.f);
    add_groups<NG>(ends, 0, ends.first[0], add);
    leave(sum, 0);
  }
}

// The last kernel: blocks up to `join_ctas` finish the table's gradient, those behind them scale that of the hidden rows
// (g / count * grad_hidden, rounded once).  Bound: memory and the latency of the ranges' checks; 131072 positions and 50001 items
// of 64 columns (50 MB in, 23 MB out) 14 us, 32768 and 165001 of 128: 22 us.
// Table: items without entries (zeros) and those whose entries reach over a span's end: their spans' sums, in order.  A
// group of lanes takes two items one after another; items of many spans are left to the whole block.
template <typename T, int W, typename P>
__global__ void __launch_bounds__(kThreads) loss_join_kernel(Args a, const float *__restrict__ lse,
                                                             const float *__restrict__ grad_loss,
                                                             const uint32_t *__restrict__ keys,
                                                             const uint32_t *__restrict__ ranges, uint32_t entries, int span,
                                                             const float *__restrict__ part, T *__restrict__ dtable,
                                                             unsigned join_ctas, const float *__restrict__ grad_hidden,
                                                             T *__restrict__ dhidden) {
  constexpr int LPC = P::LPC, V = P::V, NG = kThreads / LPC, CPW = 32 / LPC;
  using S = Strip<T, W, P>;
  constexpr int kRounds = kItemsPerGroup, kItems = NG * kRounds;  // of a block
  constexpr uint32_t kAlone = 16;  // spans that a group of lanes adds up by itself
  __shared__ uint2 popular[kItems];  // their first and last span
  __shared__ int popular_item[kItems];  // and which they are, bit 30: as `inside` below
  __shared__ int populars;
  __shared__ float sums[NG][LPC * V * 8];
  grid_chain_enter();
  const int lane = (int)threadIdx.x % 32, col = lane % LPC, sub = lane / LPC, grp = (int)threadIdx.x / LPC;
  if (blockIdx.x >= join_ctas) {
    const float scale = grad_scale(a, lse, grad_loss);
    const bool number = fabsf(scale) <= FLT_MAX;
    const int64_t step = (int64_t)(gridDim.x - join_ctas) * NG;
    for (int64_t row = (int64_t)(blockIdx.x - join_ctas) * NG + grp; row < a.rows; row += step) {
      // (padding has zeros there, which stay zeros in a product with any number: the targets are read only if it is none)
      const bool part = number || row_target(a, (int)row) >= 0;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        Group x = load_sums<W, P>(grad_hidden + row * a.cols, col, v, a.cols);
#pragma unroll
        for (int i = 0; i < 4; ++i) x.p[i] = part ? mul2(x.p[i], both(scale)) : both(0.f);
        S::store(dhidden + row * a.sdh, col, v, a.cols, x);
      }
    }
    return;
  }
  if (threadIdx.x == 0) populars = 0;
  __syncthreads();
  const float scale = grad_scale(a, lse, grad_loss);
  const int64_t item0 = (int64_t)blockIdx.x * kItems + threadIdx.x / 32 * (CPW * kRounds);  // of the warp, one a lane
  uint2 range = make_uint2(0, 0);
  if (lane < CPW * kRounds && item0 + lane < a.items && entries) {
    // (nobody has cleared the ranges: what stands at an item without entries is checked against the list)
    const uint32_t item = (uint32_t)(item0 + lane), from = ranges[item], to = ranges[a.items + item];
    if (from < to && to <= entries && keys[from] == item && keys[to - 1] == item && (from == 0 || keys[from - 1] != item) &&
        (to == entries || keys[to] != item))
      range = make_uint2(from, to);
  }
  const uint32_t c0 = range.x / (uint32_t)span, c1 = range.y ? (range.y - 1) / (uint32_t)span : 0;
  const uint32_t n = range.x == range.y ? 0 : c1 - c0 + 1;
  // the sum of every `step`-th span's share, from the `from`-th on
  auto add_up = [&](uint32_t c0, uint32_t c1, bool inside, uint32_t from, uint32_t step, Group (&acc)[V]) {
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[v].p[i] = both(0.f);
#pragma unroll(V == 1 ? 8 : 2)
    for (uint32_t c = c0 + from; c <= c1; c += step) {
      const int64_t slot = (int64_t)c * 2 + (c == c0 && inside ? 1 : 0);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Group x = load_sums<W, P>(part + slot * a.cols, col, v, a.cols);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[v].p[i] = add2(acc[v].p[i], x.p[i]);
      }
    }
  };
  auto write = [&](int64_t to, Group (&acc)[V], bool some = true) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[v].p[i] = some ? mul2(acc[v].p[i], both(scale)) : both(0.f);
      S::store(dtable + to * a.sdt, col, v, a.cols, acc[v]);
    }
  };
  const bool inside = range.x % (uint32_t)span != 0;  // the first span's share is that of its last item
  Group acc[V];
#pragma unroll 1
  for (int k = 0; k < kRounds; ++k) {
    const int from = k * CPW + sub;
    const uint32_t many = __shfl_sync(0xffffffffu, n, from);
    const uint32_t b0 = __shfl_sync(0xffffffffu, c0, from), b1 = __shfl_sync(0xffffffffu, c1, from);
    const bool in = __shfl_sync(0xffffffffu, (int)inside, from);
    if (item0 + from >= a.items || many == 1 || many > kAlone) continue;  // (one span: written by the kernel before)
    if (many) add_up(b0, b1, in, 0, 1, acc);
    write(item0 + from, acc, many > 0);  // (nobody's candidate: zeros whatever the upstream gradient is)
  }
  if (n > kAlone) {  // (in which order they are noted does not matter: each is summed by itself)
    const int at = atomicAdd(&populars, 1);
    popular[at] = make_uint2(c0, c1);
    popular_item[at] = (int)threadIdx.x / 32 * (CPW * kRounds) + lane + (inside ? 1 << 30 : 0);
  }
  __syncthreads();
  const int count = populars;
  for (int k = 0; k < count; ++k) {
    const uint2 r = popular[k];
    add_up(r.x, r.y, popular_item[k] >> 30 & 1, (uint32_t)grp, NG, acc);
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) sums[grp][8 * (col + v * LPC) + i] = acc[v].at(i);
    __syncthreads();
    if (grp == 0) {
      for (int g = 1; g < NG; ++g)
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[v].at(i) += sums[g][8 * (col + v * LPC) + i];
      write((int64_t)blockIdx.x * kItems + (popular_item[k] & 0xffff), acc);
    }
    __syncthreads();
  }
}

}  // namespace

SortPlan sort_plan(const Args &a, int lanes, int threads) {
  SortPlan p;
  int bits = 1;
  while (bits < 31 && (int64_t)1 << bits <= a.items) ++bits;  // numbers 0 .. items
  p.passes = (bits + 8) / 9;
  p.bits = (bits + p.passes - 1) / p.passes;
  p.entries = (int64_t)a.rows * (a.n + 1);
  p.tiles = (p.entries + kTile - 1) / kTile;
  // enough groups of lanes for 1024 threads an SM twice over, if there are that many entries
  p.chunk = 512;
  while (p.chunk > (threads == kMmaThreads ? 32 : 8) && p.entries / p.chunk * lanes < 2LL * kSMs * 1024) p.chunk /= 2;
  p.span = p.chunk * (threads / lanes);
  p.spans = (p.entries + p.span - 1) / p.span;
  return p;
}

Scratch carve(const Args &a, void *base) {
  Scratch s;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char *r = base ? static_cast<char *>(base) + off : nullptr;
    off += (bytes + 255) / 256 * 256;
    return r;
  };
  const SortPlan p = sort_plan(a, lanes_of(a.groups), kThreads), m = sort_plan(a, 32, kMmaThreads);
  const size_t list = (size_t)p.entries * sizeof(uint32_t);
  s.sums = reinterpret_cast<double2 *>(take(kForwardBytes));
  for (int i = 0; i < 2; ++i) {
    s.keys[i] = reinterpret_cast<uint32_t *>(take(list));
    s.vals[i] = reinterpret_cast<uint32_t *>(take(list));
  }
  s.hist = reinterpret_cast<uint32_t *>(take((size_t)p.tiles * ((size_t)1 << p.bits) * sizeof(uint32_t)));
  s.totals = reinterpret_cast<uint32_t *>(take(kMaxDigits * sizeof(uint32_t)));
  s.range = reinterpret_cast<uint32_t *>(take((size_t)a.items * 2 * sizeof(uint32_t)));
  s.part = reinterpret_cast<float *>(take((size_t)(p.spans > m.spans ? p.spans : m.spans) * 2 * a.cols * sizeof(float)));
  s.bytes = off;
  return s;
}

int launch_items(const Args &a, int dtype, const void *hidden, const void *table, const float *lse, const float *grad_hidden,
                 const float *grad_loss, void *dhidden, void *dtable, int width, const Scratch &s, cudaStream_t st) {
  const bool dense = (int64_t)a.rows * (a.n + 1) / a.items >= kDense;  // (sixteen entries at a time want several an item)
  const int lines = dense ? mma_lines(a, dtype, width) : 0;
  const SortPlan p = lines ? sort_plan(a, 32, kMmaThreads) : sort_plan(a, lanes_of(a.groups), kThreads);
  const uint32_t entries = dtable ? (uint32_t)p.entries : 0;
  const Split by = split_by((uint32_t)a.n + 1);
  int at = 1;  // the buffer that holds the list
  if (entries && entries <= (uint32_t)kSmallEntries) {
    if (!allow_smem(sort_small_kernel, kSmallSmem)) return BLOSSOM_ERR_CUDA;
    LaunchScope ls(K_LOSS_SORT, st);
    launch_chained(sort_small_kernel, dim3(1), dim3(kSmallThreads), kSmallSmem, st, a, by, entries,
                   (p.passes * p.bits + kSmallBits - 1) / kSmallBits, s.keys[at], s.vals[at]);
  } else if (entries) {
    const MoveKernel moves[2] = {move_kernel<true>(p.bits), move_kernel<false>(p.bits)};
    const size_t smem = move_smem(p.bits);
    const bool scan = p.tiles > kTilesWithoutScan;
    const dim3 grid((unsigned)p.tiles), block(kSortThreads);
    if (!allow_smem(moves[0], smem) || !allow_smem(moves[1], smem)) return BLOSSOM_ERR_CUDA;
    for (int i = 0; i < p.passes; ++i) {
      const int shift = i * p.bits, to = at ^ 1;
      {
        LaunchScope ls(K_LOSS_SORT, st);
        launch_chained(i ? sort_count_kernel<false> : sort_count_kernel<true>, grid, block, 0, st, a, by, s.keys[at], entries,
                       shift, p.bits, s.hist);
      }
      if (scan) {
        LaunchScope ls(K_LOSS_SORT, st);
        launch_chained(sort_scan_kernel, dim3(1u << p.bits), block, 0, st, s.hist, (int)p.tiles, s.totals);
      }
      LaunchScope ls(K_LOSS_SORT, st);
      launch_chained(moves[i > 0], grid, block, smem, st, a, by, (const uint32_t *)s.keys[at], (const uint32_t *)s.vals[at],
                     entries, shift, (const uint32_t *)s.hist, scan ? (const uint32_t *)s.totals : (const uint32_t *)nullptr,
                     s.keys[to], s.vals[to]);
      at = to;
    }
  }
  const uint32_t *keys = s.keys[at], *vals = s.vals[at];
  if (entries && lines) {
    with_lines(lines, a.cols, [&](auto n, auto all) {
      constexpr int NL = decltype(n)::value;
      LaunchScope ls(K_LOSS_ITEMS, st);
      launch_chained(loss_items_mma_kernel<NL, decltype(all)::value>, dim3((unsigned)p.spans),
                     dim3(kMmaThreads), 0, st, a, static_cast<const __nv_bfloat16 *>(hidden),
                     static_cast<const __nv_bfloat16 *>(table), lse, grad_loss, keys, vals, entries, p.chunk,
                     static_cast<__nv_bfloat16 *>(dtable), s.part, s.range);
    });
  }
  with_plan(a.groups, [&](auto plan) {
    using P = decltype(plan);
    rows::with_type(dtype, width, [&](auto t, auto w) {
      using T = decltype(t);
      constexpr int W = decltype(w)::value, per = kThreads / P::LPC;
      if (entries && !lines) {
        LaunchScope ls(K_LOSS_ITEMS, st);
        launch_chained(loss_items_kernel<T, W, P>,
                       dim3((unsigned)p.spans), dim3(kThreads), 0, st, a, static_cast<const T *>(hidden),
                       static_cast<const T *>(table), lse, grad_loss, keys, vals, entries, p.chunk, static_cast<T *>(dtable),
                       s.part, s.range);
      }
      const int64_t items = per * kItemsPerGroup, join = dtable ? (a.items + items - 1) / items : 0;
      const int64_t rows = dhidden ? ((int64_t)a.rows + per - 1) / per : 0, most = kSMs * 8;
      const int64_t ctas = join + (rows < most ? rows : most);
      if (ctas == 0) return;
      LaunchScope ls(K_LOSS_JOIN, st);
      launch_chained(loss_join_kernel<T, W, P>, dim3((unsigned)ctas), dim3(kThreads), 0, st, a, lse, grad_loss,
                     keys, (const uint32_t *)s.range, entries, p.span, (const float *)s.part, static_cast<T *>(dtable),
                     (unsigned)join, grad_hidden, static_cast<T *>(dhidden));
    });
  });
  return cudaGetLastError() == cudaSuccess ? BLOSSOM_OK : BLOSSOM_ERR_CUDA;
}

}  // namespace loss
}  // namespace blossom
