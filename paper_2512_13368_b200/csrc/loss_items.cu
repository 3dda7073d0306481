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
__device__ __forceinline__ void make_entry(const Args &a, uint32_t e, uint32_t *key, uint32_t *val) {
  const uint32_t t = e / (uint32_t)(a.n + 1), j = e - t * (uint32_t)(a.n + 1);
  const int target = row_target(a, (int)t);
  const int c = target >= 0 ? candidate(a, (int)t, target, (int)j) : -1;
  *key = c >= 0 ? (uint32_t)c : (uint32_t)a.items;
  *val = t | (j == 0 ? 0x80000000u : 0u);
}

// Counts of a tile's digits, to hist[digit][tile].
template <bool FIRST>
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(Args a, const uint32_t *__restrict__ keys, uint32_t entries,
                                                                  int shift, int bits, uint32_t *__restrict__ hist) {
  __shared__ uint32_t count[kMaxDigits];
  grid_chain_enter();
  const int digits = 1 << bits;
  if ((int)threadIdx.x < digits) count[threadIdx.x] = 0;
  __syncthreads();
  const uint32_t lane = threadIdx.x % 32, e0 = blockIdx.x * (uint32_t)kTile + threadIdx.x / 32 * (32 * kSortPerThread) + lane;
#pragma unroll 4
  for (int r = 0; r < kSortPerThread; ++r) {
    const uint32_t e = e0 + 32 * r;
    uint32_t key = 0, val, d = 0xffffffffu;
    if (e < entries) {
      if (FIRST) make_entry(a, e, &key, &val);
      else key = keys[e];
      d = key >> shift & (uint32_t)(digits - 1);
    }
    // (one addition for the lanes that share a digit: a batch of padding is one digit throughout)
    const uint32_t peers = __match_any_sync(0xffffffffu, d);
    if (e < entries && (peers & ((1u << lane) - 1)) == 0) atomicAdd(&count[d], (uint32_t)__popc(peers));
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

// A tile's entries to their places, in order: ranks within a warp by matching digits, then warps, then digits; the tile is put
// in order in shared memory first, so that it leaves in runs.  hist null: there is one tile, whose own counts are all.
template <bool FIRST>
__global__ void __launch_bounds__(kSortThreads) sort_move_kernel(Args a, const uint32_t *__restrict__ keys,
                                                                 const uint32_t *__restrict__ vals, uint32_t entries, int shift,
                                                                 int bits, const uint32_t *__restrict__ hist,
                                                                 const uint32_t *__restrict__ totals,
                                                                 uint32_t *__restrict__ keys_out, uint32_t *__restrict__ vals_out) {
  constexpr int NW = kSortThreads / 32;
  extern __shared__ uint32_t sm[];
  uint32_t *sk = sm, *sv = sm + kTile, *offset = sm + 2 * kTile, *count = offset + kMaxDigits;  // count[warp][digit]
  __shared__ uint32_t warp_totals[NW];
  grid_chain_enter();
  const int digits = 1 << bits, tid = (int)threadIdx.x, lane = tid % 32, warp = tid / 32;
  const uint32_t mask = (uint32_t)digits - 1;
  for (int i = tid; i < NW * digits; i += kSortThreads) count[i] = 0;
  __syncthreads();
  const uint32_t tile0 = blockIdx.x * (uint32_t)kTile, e0 = tile0 + (uint32_t)warp * (32 * kSortPerThread) + (uint32_t)lane;
  uint32_t key[kSortPerThread], val[kSortPerThread], rank[kSortPerThread];
#pragma unroll
  for (int r = 0; r < kSortPerThread; ++r) {
    const uint32_t e = e0 + 32 * r;
    key[r] = val[r] = 0;
    if (e < entries) {
      if (FIRST) make_entry(a, e, &key[r], &val[r]);
      else key[r] = keys[e], val[r] = vals[e];
    }
  }
  uint32_t *mine = count + warp * digits;
#pragma unroll
  for (int r = 0; r < kSortPerThread; ++r) {
    const bool there = e0 + 32 * r < entries;
    const uint32_t d = there ? key[r] >> shift & mask : 0xffffffffu;
    const uint32_t peers = __match_any_sync(0xffffffffu, d), below = peers & ((1u << lane) - 1);
    rank[r] = there ? mine[d] + (uint32_t)__popc(below) : 0;
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
      const uint32_t at = mine[key[r] >> shift & mask] + rank[r];
      sk[at] = key[r];
      sv[at] = val[r];
    }
  __syncthreads();
  const uint32_t here = entries - tile0 < (uint32_t)kTile ? entries - tile0 : (uint32_t)kTile;
  for (uint32_t i = (uint32_t)tid; i < here; i += kSortThreads) {
    const uint32_t k = sk[i], at = offset[k >> shift & mask] + i;
    keys_out[at] = k;
    vals_out[at] = sv[i];
  }
}
constexpr size_t kMoveSmem = (2 * kTile + kMaxDigits + kSortThreads / 32 * kMaxDigits) * sizeof(uint32_t);

// ---- sums over an item's entries ---------------------------------------------------------------
constexpr int kThreads = 256;

template <typename T, int W, typename P>
__global__ void __launch_bounds__(kThreads) loss_items_kernel(Args a, const T *__restrict__ hidden, const T *__restrict__ table,
                                                              const float *__restrict__ lse, const float *__restrict__ grad_loss,
                                                              const uint32_t *__restrict__ keys, const uint32_t *__restrict__ vals,
                                                              uint32_t entries, int chunk, T *__restrict__ dtable,
                                                              float *__restrict__ part) {
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
  float w[V][8], acc[V][8];
  auto begin = [&](uint32_t item) {
    cur = item;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int g = col + v * LPC;
      load_group<T, W>(table + cur * a.st + 8 * g, a.cols - 8 * g, w[v]);
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[v][i] = 0.f, w[v][i] *= kLog2e;
    }
  };
  auto finish = [&](bool whole) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int g = col + v * LPC, valid = a.cols - 8 * g;
      if (whole) {
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[v][i] *= scale;
        store_group<T, W>(dtable + cur * a.sdt + 8 * g, valid, acc[v]);
      } else {
        store_group<float, (W < 4 ? W : 4)>(part + (c * 2 + (first ? 0 : 1)) * a.cols + 8 * g, valid, acc[v]);
      }
    }
  };
  if (cur >= (uint32_t)a.items) return;
  begin(cur);
  for (uint32_t i = s; i < e; i += U) {
    uint32_t key[U], val[U];
    float h[U][V][8], top[U];
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
        load_group<T, W>(hidden + t * a.sh + 8 * g, there ? a.cols - 8 * g : 0, h[u][v]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u >= e) break;
      if (key[u] != cur) {
        finish(!open);
        open = first = false;
        if (key[u] >= (uint32_t)a.items) return;  // (what follows is no candidate)
        begin(key[u]);
      }
      float l = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j) l += w[v][j] * h[u][v][j];
#pragma unroll
      for (int o = 1; o < LPC; o <<= 1) l += __shfl_xor_sync(lanes, l, o);
      const float coef = exp2f(l - top[u]) - (val[u] >> 31 ? 1.f : 0.f);
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[v][j] += coef * h[u][v][j];
    }
  }
  finish(!open && !(e < entries && keys[e] == cur));
}

__device__ __forceinline__ uint32_t lower_bound(const uint32_t *keys, uint32_t n, uint32_t key) {
  uint32_t lo = 0, len = n;
  while (len) {
    const uint32_t half = len / 2;
    if (keys[lo + half] < key) lo += half + 1, len -= half + 1;
    else len = half;
  }
  return lo;
}

// Items without entries (zeros) and those whose entries reach over a chunk's end: their chunks' sums, in order.  A group of
// lanes an item; popular items are left to the whole block.
template <typename T, int W, typename P>
__global__ void __launch_bounds__(kThreads) loss_join_kernel(Args a, const float *__restrict__ lse,
                                                             const float *__restrict__ grad_loss,
                                                             const uint32_t *__restrict__ keys, uint32_t entries, int chunk,
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
    if (item < a.items) r = make_uint2(lower_bound(keys, entries, (uint32_t)item), lower_bound(keys, entries, (uint32_t)item + 1));
    range[grp] = r;
  }
  __syncthreads();
  // the sum of every `step`-th chunk of a range, from its `from`-th on
  auto add_up = [&](uint2 r, uint32_t from, uint32_t step, float (&acc)[V][8]) {
    const uint32_t c0 = r.x / (uint32_t)chunk, c1 = (r.y - 1) / (uint32_t)chunk;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[v][i] = 0.f;
#pragma unroll 4
    for (uint32_t c = c0 + from; c <= c1; c += step) {
      const int64_t slot = (int64_t)c * 2 + (c == c0 && r.x % (uint32_t)chunk ? 1 : 0);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int g = col + v * LPC;
        float x[8];
        load_group<float, WF>(part + slot * a.cols + 8 * g, a.cols - 8 * g, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[v][i] += x[i];
      }
    }
  };
  auto chunks_of = [&](uint2 r) { return r.x == r.y ? 0u : (r.y - 1) / (uint32_t)chunk - r.x / (uint32_t)chunk + 1; };
  auto write = [&](int64_t to, float (&acc)[V][8]) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int g = col + v * LPC;
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[v][i] *= scale;
      store_group<T, W>(dtable + to * a.sdt + 8 * g, a.cols - 8 * g, acc[v]);
    }
  };
  float acc[V][8];
  {
    const uint2 r = range[grp];
    const uint32_t n = chunks_of(r);
    if (item < a.items && n != 1 && n <= kAlone) {  // (one chunk: written by the kernel before)
      if (n == 0) {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[v][i] = 0.f;
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
      for (int i = 0; i < 8; ++i) sums[grp][8 * (col + v * LPC) + i] = acc[v][i];
    __syncthreads();
    if (grp == 0) {
      for (int g = 1; g < NG; ++g)
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[v][i] += sums[g][8 * (col + v * LPC) + i];
      write((int64_t)blockIdx.x * NG + k, acc);
    }
    __syncthreads();
  }
}

}  // namespace

SortPlan sort_plan(const Args &a) {
  SortPlan p;
  int bits = 1;
  while (bits < 31 && (int64_t)1 << bits <= a.items) ++bits;  // numbers 0 .. items
  p.passes = (bits + 8) / 9;
  p.bits = (bits + p.passes - 1) / p.passes;
  p.entries = (int64_t)a.rows * (a.n + 1);
  p.tiles = (p.entries + kTile - 1) / kTile;
  // long chunks leave fewer sums to join, short ones make more groups of lanes: twice as many as run at a time, if there
  // are that many
  const int64_t at_once = kSMs * 2048LL / lanes_of(a.groups);
  p.chunk = 128;
  while (p.chunk > 16 && p.entries / p.chunk < 2 * at_once) p.chunk /= 2;
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
  const SortPlan p = sort_plan(a);
  const size_t list = (size_t)p.entries * sizeof(uint32_t);
  s.sums = reinterpret_cast<double2 *>(take(kForwardBytes));
  for (int i = 0; i < 2; ++i) {
    s.keys[i] = reinterpret_cast<uint32_t *>(take(list));
    s.vals[i] = reinterpret_cast<uint32_t *>(take(list));
  }
  s.hist = reinterpret_cast<uint32_t *>(take((size_t)p.tiles * ((size_t)1 << p.bits) * sizeof(uint32_t)));
  s.totals = reinterpret_cast<uint32_t *>(take(kMaxDigits * sizeof(uint32_t)));
  s.part = reinterpret_cast<float *>(take((size_t)p.chunks * 2 * a.cols * sizeof(float)));
  s.bytes = off;
  return s;
}

int launch_items(const Args &a, int dtype, const void *hidden, const void *table, const float *lse, const float *grad_loss,
                 void *dtable, int width, const Scratch &s, cudaStream_t st) {
  const SortPlan p = sort_plan(a);
  const uint32_t entries = (uint32_t)p.entries;
  int at = 1;  // the buffer that holds the list
  if (!allow_smem(sort_move_kernel<true>, kMoveSmem) || !allow_smem(sort_move_kernel<false>, kMoveSmem)) return BLOSSOM_ERR_CUDA;
  for (int i = 0; entries && i < p.passes; ++i) {
    const int shift = i * p.bits, to = at ^ 1;
    uint32_t *hist = p.tiles > 1 ? s.hist : nullptr;
    const dim3 grid((unsigned)p.tiles), block(kSortThreads);
    if (hist) {
      {
        LaunchScope ls(K_LOSS_SORT, st);
        launch_chained(i ? sort_count_kernel<false> : sort_count_kernel<true>, grid, block, 0, st, a,
                       (const uint32_t *)s.keys[at], entries, shift, p.bits, hist);
      }
      LaunchScope ls(K_LOSS_SORT, st);
      launch_chained(sort_scan_kernel, dim3(1u << p.bits), block, 0, st, hist, (int)p.tiles, s.totals);
    }
    LaunchScope ls(K_LOSS_SORT, st);
    launch_chained(i ? sort_move_kernel<false> : sort_move_kernel<true>, grid, block, kMoveSmem, st, a,
                   (const uint32_t *)s.keys[at], (const uint32_t *)s.vals[at], entries, shift, p.bits, (const uint32_t *)hist,
                   (const uint32_t *)s.totals, s.keys[to], s.vals[to]);
    at = to;
  }
  with_plan(a.groups, [&](auto plan) {
    using P = decltype(plan);
    rows::with_type(dtype, width, [&](auto t, auto w) {
      using T = decltype(t);
      constexpr int W = decltype(w)::value, per = kThreads / P::LPC;
      if (entries) {
        LaunchScope ls(K_LOSS_ITEMS, st);
        launch_chained(loss_items_kernel<T, W, P>, dim3((unsigned)((p.chunks + per - 1) / per)), dim3(kThreads), 0, st, a,
                       static_cast<const T *>(hidden), static_cast<const T *>(table), lse, grad_loss,
                       (const uint32_t *)s.keys[at], (const uint32_t *)s.vals[at], entries, p.chunk, static_cast<T *>(dtable),
                       s.part);
      }
      LaunchScope ls(K_LOSS_ITEMS, st);
      launch_chained(loss_join_kernel<T, W, P>, dim3((unsigned)(((int64_t)a.items + per - 1) / per)), dim3(kThreads), 0, st, a,
                     lse, grad_loss, (const uint32_t *)s.keys[at], entries, p.chunk, (const float *)s.part,
                     static_cast<T *>(dtable));
    });
  });
  return cudaGetLastError() == cudaSuccess ? BLOSSOM_OK : BLOSSOM_ERR_CUDA;
}

}  // namespace loss
}  // namespace blossom
