// Sampled softmax loss, the part over items: dtable[i] = g / count * sum over the candidates (t, j) that are item i of
// (p_tj - [j is the target]) * hidden_t.
//
// The candidates are sorted by item (a stable radix sort of (item, position) pairs, so that an item's positions come in
// the same order every time), then groups of lanes walk equal chunks of the sorted list: the item's row of the table stays
// in registers, each position's hidden row is read once for both the logit that is formed again and the sum.  An item
// whose entries lie in one chunk is written there and then; the sums of others go to scratch, one a chunk, and are
// added up in order.  No atomics: every sum has a fixed order whatever the popularity of the items.
#include "loss.cuh"

namespace blossom {
namespace loss {
namespace {

// ---- the sort ------------------------------------------------------------------------------------
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
__device__ __forceinline__ uint32_t entry_key(const Args &a, const Split &by, uint32_t e) {
  const uint32_t t = by(e), j = e - t * (uint32_t)(a.n + 1);
  const int target = row_target(a, (int)t);
  const int c = target >= 0 ? candidate(a, (int)t, target, (int)j) : -1;
  return c >= 0 ? (uint32_t)c : (uint32_t)a.items;
}
__device__ __forceinline__ uint32_t entry_val(const Args &a, const Split &by, uint32_t e) {
  const uint32_t t = by(e);
  return t | (e == t * (uint32_t)(a.n + 1) ? 0x80000000u : 0u);
}

// Counts of a tile's digits, to hist[digit][tile].  The first pass makes the keys.
template <bool FIRST>
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(Args a, Split by, uint32_t *__restrict__ keys, uint32_t entries,
                                                                  int shift, int bits, uint32_t *__restrict__ hist,
                                                                  uint32_t *__restrict__ range) {
  __shared__ uint32_t count[kMaxDigits];
  grid_chain_enter();
  const int digits = 1 << bits;
  const uint32_t mask = (uint32_t)digits - 1, none = (uint32_t)a.items;
  if ((int)threadIdx.x < digits) count[threadIdx.x] = 0;
  if (FIRST)
    for (int64_t i = (int64_t)blockIdx.x * kSortThreads + threadIdx.x; i < 2 * (int64_t)a.items; i += (int64_t)gridDim.x * kSortThreads)
      range[i] = 0;
  __syncthreads();
  const uint32_t e0 = blockIdx.x * (uint32_t)kTile + threadIdx.x;
  uint32_t key[kSortPerThread];
#pragma unroll
  for (int r = 0; r < kSortPerThread; ++r) {
    const uint32_t e = e0 + kSortThreads * r;
    key[r] = 0;
    if (e < entries) key[r] = FIRST ? entry_key(a, by, e) : keys[e];
  }
#pragma unroll
  for (int r = 0; r < kSortPerThread; ++r) {
    const uint32_t e = e0 + kSortThreads * r;
    const bool there = e < entries, padding = there && key[r] == none;
    if (FIRST && there) keys[e] = key[r];
    // (padding comes in long runs of one key: one addition a warp; items are mostly different ones)
    const uint32_t pads = __ballot_sync(0xffffffffu, padding);
    if (padding && threadIdx.x % 32 == __ffs(pads) - 1) atomicAdd(&count[none >> shift & mask], (uint32_t)__popc(pads));
    if (there && !padding) atomicAdd(&count[key[r] >> shift & mask], 1u);
  }
  __syncthreads();
  if ((int)threadIdx.x < digits) hist[(size_t)threadIdx.x * gridDim.x + blockIdx.x] = count[threadIdx.x];
}

// Sum over the threads before this one of a 512-thread block, and the block's total.
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
  __shared__ uint32_t warp_totals[kSortThreads / 32];
  grid_chain_enter();
  uint32_t *h = hist + (size_t)blockIdx.x * tiles, carry = 0, total;
  for (int i0 = 0; i0 < tiles; i0 += kSortThreads) {
    const int i = i0 + (int)threadIdx.x;
    const uint32_t before = block_prefix(i < tiles ? h[i] : 0, warp_totals, &total);
    if (i < tiles) h[i] = carry + before;
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
// in order in shared memory first, so that it leaves in runs.  FIRST: the values are made here.  hist null: there is one tile,
// whose own counts are all.
template <int BITS, bool FIRST>
__global__ void __launch_bounds__(kSortThreads, 2) sort_move_kernel(Args a, Split by, const uint32_t *__restrict__ keys,
                                                                    const uint32_t *__restrict__ vals, uint32_t entries,
                                                                    int shift, const uint32_t *__restrict__ hist,
                                                                    const uint32_t *__restrict__ totals,
                                                                    uint32_t *__restrict__ keys_out,
                                                                    uint32_t *__restrict__ vals_out) {
  constexpr int NW = kSortThreads / 32;
  extern __shared__ uint32_t sm[];
  uint32_t *sk = sm, *sv = sm + kTile, *offset = sm + 2 * kTile, *count = offset + kMaxDigits;  // count[warp][digit]
  __shared__ uint32_t warp_totals[NW];
  grid_chain_enter();
  constexpr int digits = 1 << BITS;
  constexpr uint32_t mask = (uint32_t)digits - 1;
  const int tid = (int)threadIdx.x, lane = tid % 32, warp = tid / 32;
  for (int i = tid; i < NW * digits; i += kSortThreads) count[i] = 0;
  __syncthreads();
  const uint32_t tile0 = blockIdx.x * (uint32_t)kTile, e0 = tile0 + (uint32_t)warp * (32 * kSortPerThread) + (uint32_t)lane;
  uint32_t key[kSortPerThread], rank[kSortPerThread / 2];  // (two ranks a word)
#pragma unroll
  for (int r = 0; r < kSortPerThread; ++r) {
    const uint32_t e = e0 + 32 * r;
    key[r] = 0;
    if (e < entries) key[r] = keys[e];
  }
  uint32_t *mine = count + warp * digits;
#pragma unroll
  for (int r = 0; r < kSortPerThread; ++r) {
    const bool there = e0 + 32 * r < entries;
    const uint32_t d = key[r] >> shift & mask;
    const uint32_t peers = same_digit<BITS>(d, there), below = peers & ((1u << lane) - 1);
    const uint32_t at = there ? mine[d] + (uint32_t)__popc(below) : 0;
    rank[r / 2] = r % 2 ? rank[r / 2] | at << 16 : at;
    __syncwarp();
    if (there && below == 0) mine[d] += (uint32_t)__popc(peers);
    __syncwarp();
  }
  __syncthreads();
  uint32_t in_tile = 0, all;
  if (tid < digits)
    for (int w = 0; w < NW; ++w) {
      const uint32_t c = count[w * digits + tid];
      count[w * digits + tid] = in_tile;  // of the warps before
      in_tile += c;
    }
  const uint32_t tile_base = block_prefix(in_tile, warp_totals, &all);
  uint32_t global_base = tile_base;
  if (hist) {
    const uint32_t total = tid < digits ? totals[tid] : 0;
    global_base = block_prefix(total, warp_totals, &all);
    if (tid < digits) global_base += hist[(size_t)tid * gridDim.x + blockIdx.x];
  }
  if (tid < digits) {
    for (int w = 0; w < NW; ++w) count[w * digits + tid] += tile_base;
    offset[tid] = global_base - tile_base;
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kSortPerThread; ++r)
    if (e0 + 32 * r < entries) {
      const uint32_t at = mine[key[r] >> shift & mask] + (r % 2 ? rank[r / 2] >> 16 : rank[r / 2] & 0xffffu);
      sk[at] = key[r];
      sv[at] = FIRST ? e0 + 32 * r : vals[e0 + 32 * r];
    }
  __syncthreads();
  const uint32_t here = entries - tile0 < (uint32_t)kTile ? entries - tile0 : (uint32_t)kTile;
  for (uint32_t i = (uint32_t)tid; i < here; i += kSortThreads) {
    const uint32_t k = sk[i], at = offset[k >> shift & mask] + i;
    keys_out[at] = k;
    vals_out[at] = FIRST ? entry_val(a, by, sv[i]) : sv[i];
  }
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
constexpr size_t kMoveSmem = (2 * kTile + kMaxDigits + kSortThreads / 32 * kMaxDigits) * sizeof(uint32_t);

// ---- sums over an item's entries ---------------------------------------------------------------
constexpr int kThreads = 256;

template <typename T, int W, typename P>
__global__ void __launch_bounds__(kThreads) loss_items_kernel(Args a, const T *__restrict__ hidden, const T *__restrict__ table,
                                                              const float *__restrict__ lse, const float *__restrict__ grad_loss,
                                                              const uint32_t *__restrict__ keys, const uint32_t *__restrict__ vals,
                                                              uint32_t entries, int chunk, T *__restrict__ dtable,
                                                              float *__restrict__ part, uint32_t *__restrict__ range) {
  constexpr int LPC = P::LPC, V = P::V, U = V == 1 ? 4 : 1;
  grid_chain_enter();
  const int col = (int)threadIdx.x % LPC;
  const uint32_t lanes = LPC == 32 ? 0xffffffffu : ((1u << LPC) - 1) << ((threadIdx.x % 32) / LPC * LPC);
  const int64_t c = (int64_t)blockIdx.x * (kThreads / LPC) + threadIdx.x / LPC;
  if (c * chunk >= entries) return;
  const uint32_t s = (uint32_t)(c * chunk), e = entries - s < (uint32_t)chunk ? entries : s + (uint32_t)chunk;
  const float scale = grad_scale(a, lse, grad_loss);
  uint32_t cur = keys[s];
  bool open = s > 0 && keys[s - 1] == cur;  // the item's entries began in a chunk before
  bool first = true;
  Group w[V], acc[V];
  auto begin = [&](uint32_t item) {
    cur = item;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int g = col + v * LPC;
      w[v] = load_group<T, W>(table + cur * a.st + 8 * g, a.cols - 8 * g);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[v].p[i] = both(0.f), w[v].p[i] = mul2(w[v].p[i], both(kLog2e));
    }
  };
  auto finish = [&](bool whole) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int g = col + v * LPC, valid = a.cols - 8 * g;
      if (whole) {
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[v].p[i] = mul2(acc[v].p[i], both(scale));
        store_group<T, W>(dtable + cur * a.sdt + 8 * g, valid, acc[v]);
      } else {
        store_group<float, (W < 4 ? W : 4)>(part + (c * 2 + (first ? 0 : 1)) * a.cols + 8 * g, valid, acc[v]);
      }
    }
  };
  const bool writer = col == 0;
  if (writer && s > 0 && !open && keys[s - 1] < (uint32_t)a.items) range[a.items + keys[s - 1]] = s;
  if (cur >= (uint32_t)a.items) return;
  if (writer && !open) range[cur] = s;
  begin(cur);
  for (uint32_t i = s; i < e; i += U) {
    uint32_t key[U], val[U];
    Group h[U][V];
    float top[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      key[u] = i + u < e ? keys[i + u] : (uint32_t)a.items;
      val[u] = i + u < e ? vals[i + u] : 0;
      const bool there = key[u] < (uint32_t)a.items;
      const int64_t t = val[u] & 0x7fffffffu;
      top[u] = there ? lse[t] * kLog2e : 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int g = col + v * LPC;
        h[u][v] = load_group<T, W>(hidden + t * a.sh + 8 * g, there ? a.cols - 8 * g : 0);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u >= e) break;
      if (key[u] != cur) {
        finish(!open);
        open = first = false;
        if (writer) range[a.items + cur] = i + u;
        if (key[u] >= (uint32_t)a.items) return;  // (what follows is no candidate)
        if (writer) range[key[u]] = i + u;
        begin(key[u]);
      }
      float l = dot<V>(w, h[u]);
#pragma unroll
      for (int o = 1; o < LPC; o <<= 1) l += __shfl_xor_sync(lanes, l, o);
      const float coef = exp2f(l - top[u]) - (val[u] >> 31 ? 1.f : 0.f);
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[v].p[j] = fma2(both(coef), h[u][v].p[j], acc[v].p[j]);
    }
  }
  finish(!open && !(e < entries && keys[e] == cur));
  if (writer && e == entries) range[a.items + cur] = e;
}

// The same on the matrix units: a warp walks a chunk 16 entries at a time, their hidden rows the first operand, the item's
// row the second; the next 16 rows are under way meanwhile.  Sixteen entries of more than one item go through once an item.
template <int NL, bool FULL>
__global__ void __launch_bounds__(kMmaThreads, NL == 1 ? 6 : 3)
    loss_items_mma_kernel(Args a, const __nv_bfloat16 *__restrict__ hidden, const __nv_bfloat16 *__restrict__ table,
                          const float *__restrict__ lse, const float *__restrict__ grad_loss, const uint32_t *__restrict__ keys,
                          const uint32_t *__restrict__ vals, uint32_t entries, int chunk, __nv_bfloat16 *__restrict__ dtable,
                          float *__restrict__ part, uint32_t *__restrict__ range) {
  grid_chain_enter();
  const int lane = (int)threadIdx.x % 32, group = lane / 8;
  const int64_t c0 = (int64_t)blockIdx.x * (kMmaThreads / 32) + threadIdx.x / 32;
  if (c0 * chunk >= entries) return;
  const uint32_t none = (uint32_t)a.items, s = (uint32_t)(c0 * chunk);
  const uint32_t e = entries - s < (uint32_t)chunk ? entries : s + (uint32_t)chunk;
  const Lanes16<NL, FULL> from_hidden(hidden, a.sh, a.cols), from_table(table, a.st, a.cols);
  struct Entries {  // 32 of them, one a lane; what lies behind the chunk is no candidate of the first position
    uint32_t key, val;
    float top;
  };
  auto entries_from = [&](uint32_t i) {
    Entries x = {none, 0, 0.f};
    if (i + lane < e) {
      x.key = keys[i + lane], x.val = vals[i + lane];
      x.top = lse[x.val & 0x7fffffffu] * kLog2e;
    }
    return x;
  };
  uint4 w[NL];
  float2 acc[NL][4];
  uint32_t cur = keys[s], before = s > 0 ? keys[s - 1] : 0xffffffffu;
  bool open = before == cur, first = true;  // open: the item's entries began in a chunk before
  auto begin = [&](uint32_t item) {
    cur = item;
    from_table.vector(item, a.cols, w);
#pragma unroll
    for (int c = 0; c < NL; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[c][i] = make_float2(0.f, 0.f);
  };
  auto finish = [&](bool whole) {
    float2 sum[NL];
    scatter16<NL>(acc, sum);
    const float scale = whole ? grad_scale(a, lse, grad_loss) : 1.f;
#pragma unroll
    for (int c = 0; c < NL; ++c) {
      const int col = scattered_column(c);
      if (!FULL && col >= a.cols) continue;
      if (whole) *reinterpret_cast<uint32_t *>(dtable + cur * a.sdt + col) = rows::pack2(sum[c].x * scale, sum[c].y * scale);
      else *reinterpret_cast<float2 *>(part + (c0 * 2 + (first ? 0 : 1)) * a.cols + col) = sum[c];
    }
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
  auto walk = [&](const Rows16<NL> &h, const Entries &x, int half) {
    float top[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) top[j] = __shfl_sync(0xffffffffu, x.top, half + 4 * j + group);
    const uint32_t targets = __ballot_sync(0xffffffffu, x.val >> 31) >> (half + group);
    for (;;) {
      float p[4];
      dots16<NL>(h, w, p);
#pragma unroll
      for (int j = 0; j < 4; ++j) p[j] = exp2f(p[j] * kLog2e - top[j]) - (targets >> (4 * j) & 1 ? 1.f : 0.f);
      uint32_t others = __ballot_sync(0xffffffffu, x.key != cur) >> half & 0xffffu;
      if (!others) {
        weigh16<NL>(h, p, acc);
        return;
      }
      // (a weight of zero would not do: another item's row may hold what is no number)
      others >>= group;
      Rows16<NL> own = h;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (others >> (4 * j) & 1) {
          p[j] = 0.f;
#pragma unroll
          for (int c = 0; c < NL; ++c) own.w[j][c] = make_uint4(0, 0, 0, 0);
        }
      weigh16<NL>(own, p, acc);
      // the next item among the 16, if there is one (they are sorted)
      const uint32_t later = __ballot_sync(0xffffffffu, (lane & 16) == half && x.key > cur && x.key < none);
      if (!later) return;
      finish(!open);
      open = first = false;
      begin(__shfl_sync(0xffffffffu, x.key, __ffs(later) - 1));
    }
  };
  Entries x = entries_from(s);
  mark(x, s);
  if (cur >= none) return;
  begin(cur);
  Rows16<NL> h[2];
  from_hidden.load16(x.val & 0x7fffffffu, 0, h[0]);
  for (uint32_t i = s; i < e; i += 32) {
    const bool second = i + 16 < e, third = i + 32 < e;
    Entries next = {none, 0, 0.f};
    if (third) next = entries_from(i + 32);
    if (second) from_hidden.load16(x.val & 0x7fffffffu, 16, h[1]);
    walk(h[0], x, 0);
    if (third) {
      mark(next, i + 32);
      from_hidden.load16(next.val & 0x7fffffffu, 0, h[0]);
    }
    if (second) walk(h[1], x, 16);
    x = next;
  }
  finish(!open && !(e < entries && keys[e] == cur));
}

// Items without entries (zeros) and those whose entries reach over a chunk's end: their chunks' sums, in order.  A group of
// lanes an item; popular items are left to the whole block.
template <typename T, int W, typename P>
__global__ void __launch_bounds__(kThreads) loss_join_kernel(Args a, const float *__restrict__ lse,
                                                             const float *__restrict__ grad_loss,
                                                             const uint32_t *__restrict__ ranges, uint32_t entries, int chunk,
                                                             const float *__restrict__ part, T *__restrict__ dtable) {
  constexpr int LPC = P::LPC, V = P::V, NG = kThreads / LPC, WF = W < 4 ? W : 4;
  constexpr uint32_t kAlone = 16;  // chunks that a group of lanes adds up by itself
  __shared__ uint2 range[NG];
  __shared__ float sums[NG][LPC * V * 8];
  grid_chain_enter();
  const int col = (int)threadIdx.x % LPC, grp = (int)threadIdx.x / LPC;
  const float scale = grad_scale(a, lse, grad_loss);
  const int64_t item = (int64_t)blockIdx.x * NG + grp;
  if (col == 0) {
    uint2 r = make_uint2(0, 0);
    if (item < a.items && entries) r = make_uint2(ranges[item], ranges[a.items + item]);
    range[grp] = r;
  }
  __syncthreads();
  // the sum of every `step`-th chunk of a range, from its `from`-th on
  auto add_up = [&](uint2 r, uint32_t from, uint32_t step, Group (&acc)[V]) {
    const uint32_t c0 = r.x / (uint32_t)chunk, c1 = (r.y - 1) / (uint32_t)chunk;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[v].p[i] = both(0.f);
#pragma unroll 4
    for (uint32_t c = c0 + from; c <= c1; c += step) {
      const int64_t slot = (int64_t)c * 2 + (c == c0 && r.x % (uint32_t)chunk ? 1 : 0);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int g = col + v * LPC;
        const Group x = load_group<float, WF>(part + slot * a.cols + 8 * g, a.cols - 8 * g);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[v].p[i] = add2(acc[v].p[i], x.p[i]);
      }
    }
  };
  auto chunks_of = [&](uint2 r) { return r.x == r.y ? 0u : (r.y - 1) / (uint32_t)chunk - r.x / (uint32_t)chunk + 1; };
  auto write = [&](int64_t to, Group (&acc)[V]) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int g = col + v * LPC;
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[v].p[i] = mul2(acc[v].p[i], both(scale));
      store_group<T, W>(dtable + to * a.sdt + 8 * g, a.cols - 8 * g, acc[v]);
    }
  };
  Group acc[V];
  {
    const uint2 r = range[grp];
    const uint32_t n = chunks_of(r);
    if (item < a.items && n != 1 && n <= kAlone) {  // (one chunk: written by the kernel before)
      if (n == 0) {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[v].p[i] = both(0.f);
      } else {
        add_up(r, 0, 1, acc);
      }
      write(item, acc);
    }
  }
  for (int k = 0; k < NG; ++k) {
    const uint2 r = range[k];
    if (chunks_of(r) <= kAlone) continue;  // (the same for the whole block)
    add_up(r, (uint32_t)grp, NG, acc);
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
      write((int64_t)blockIdx.x * NG + k, acc);
    }
    __syncthreads();
  }
}

}  // namespace

SortPlan sort_plan(const Args &a, int lanes) {
  SortPlan p;
  int bits = 1;
  while (bits < 31 && (int64_t)1 << bits <= a.items) ++bits;  // numbers 0 .. items
  p.passes = (bits + 8) / 9;
  p.bits = (bits + p.passes - 1) / p.passes;
  p.entries = (int64_t)a.rows * (a.n + 1);
  p.tiles = (p.entries + kTile - 1) / kTile;
  // long chunks leave fewer sums to join, short ones make more groups of lanes: enough for 1024 threads an SM twice over, if
  // there are that many
  p.chunk = 128;
  while (p.chunk > 32 && p.entries / p.chunk * lanes < 2LL * kSMs * 1024) p.chunk /= 2;
  p.chunks = (p.entries + p.chunk - 1) / p.chunk;
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
  const SortPlan p = sort_plan(a, lanes_of(a.groups));  // (narrow groups take the shortest chunks)
  const size_t list = (size_t)p.entries * sizeof(uint32_t);
  s.sums = reinterpret_cast<double2 *>(take(kForwardBytes));
  for (int i = 0; i < 2; ++i) {
    s.keys[i] = reinterpret_cast<uint32_t *>(take(list));
    s.vals[i] = reinterpret_cast<uint32_t *>(take(list));
  }
  s.hist = reinterpret_cast<uint32_t *>(take((size_t)p.tiles * ((size_t)1 << p.bits) * sizeof(uint32_t)));
  s.totals = reinterpret_cast<uint32_t *>(take(kMaxDigits * sizeof(uint32_t)));
  s.range = reinterpret_cast<uint32_t *>(take((size_t)a.items * 2 * sizeof(uint32_t)));
  s.part = reinterpret_cast<float *>(take((size_t)p.chunks * 2 * a.cols * sizeof(float)));
  s.bytes = off;
  return s;
}

int launch_items(const Args &a, int dtype, const void *hidden, const void *table, const float *lse, const float *grad_loss,
                 void *dtable, int width, const Scratch &s, cudaStream_t st) {
  const int lines = mma_lines(a, dtype, width);
  const SortPlan p = sort_plan(a, lines ? 32 : lanes_of(a.groups));
  const uint32_t entries = (uint32_t)p.entries;
  const Split by = split_by((uint32_t)a.n + 1);
  int at = 1;  // the buffer that holds the list
  const MoveKernel moves[2] = {move_kernel<true>(p.bits), move_kernel<false>(p.bits)};
  if (!allow_smem(moves[0], kMoveSmem) || !allow_smem(moves[1], kMoveSmem)) return BLOSSOM_ERR_CUDA;
  for (int i = 0; entries && i < p.passes; ++i) {
    const int shift = i * p.bits, to = at ^ 1;
    uint32_t *hist = p.tiles > 1 ? s.hist : nullptr;
    const dim3 grid((unsigned)p.tiles), block(kSortThreads);
    if (hist || i == 0) {  // (the first makes the keys too)
      LaunchScope ls(K_LOSS_SORT, st);
      launch_chained(i ? sort_count_kernel<false> : sort_count_kernel<true>, grid, block, 0, st, a, by, s.keys[at], entries,
                     shift, p.bits, s.hist, s.range);
    }
    if (hist) {
      LaunchScope ls(K_LOSS_SORT, st);
      launch_chained(sort_scan_kernel, dim3(1u << p.bits), block, 0, st, hist, (int)p.tiles, s.totals);
    }
    LaunchScope ls(K_LOSS_SORT, st);
    launch_chained(moves[i > 0], grid, block, kMoveSmem, st, a, by, (const uint32_t *)s.keys[at],
                   (const uint32_t *)s.vals[at], entries, shift, (const uint32_t *)hist,
                   (const uint32_t *)s.totals, s.keys[to], s.vals[to]);
    at = to;
  }
  const uint32_t *keys = s.keys[at], *vals = s.vals[at];
  if (entries && lines) {
    with_lines(lines, a.cols, [&](auto n, auto all) {
      constexpr int NL = decltype(n)::value, per = kMmaThreads / 32;
      LaunchScope ls(K_LOSS_ITEMS, st);
      launch_chained(loss_items_mma_kernel<NL, decltype(all)::value>, dim3((unsigned)((p.chunks + per - 1) / per)), dim3(kMmaThreads), 0, st,
                     a, static_cast<const __nv_bfloat16 *>(hidden), static_cast<const __nv_bfloat16 *>(table), lse, grad_loss,
                     keys, vals, entries, p.chunk, static_cast<__nv_bfloat16 *>(dtable), s.part, s.range);
    });
  }
  with_plan(a.groups, [&](auto plan) {
    using P = decltype(plan);
    rows::with_type(dtype, width, [&](auto t, auto w) {
      using T = decltype(t);
      constexpr int W = decltype(w)::value, per = kThreads / P::LPC;
      if (entries && !lines) {
        LaunchScope ls(K_LOSS_ITEMS, st);
        launch_chained(loss_items_kernel<T, W, P>, dim3((unsigned)((p.chunks + per - 1) / per)), dim3(kThreads), 0, st, a,
                       static_cast<const T *>(hidden), static_cast<const T *>(table), lse, grad_loss, keys, vals, entries,
                       p.chunk, static_cast<T *>(dtable), s.part, s.range);
      }
      LaunchScope ls(K_LOSS_ITEMS, st);
      launch_chained(loss_join_kernel<T, W, P>, dim3((unsigned)(((int64_t)a.items + per - 1) / per)), dim3(kThreads), 0, st, a,
                     lse, grad_loss, (const uint32_t *)s.range, entries, p.chunk, (const float *)s.part,
                     static_cast<T *>(dtable));
    });
  });
  return cudaGetLastError() == cudaSuccess ? BLOSSOM_OK : BLOSSOM_ERR_CUDA;
}

}  // namespace loss
}  // namespace blossom
