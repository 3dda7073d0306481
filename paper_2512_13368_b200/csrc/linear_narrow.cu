// Backward of a linear layer whose weight stays in shared memory (bf16): all of it in one pass over the rows.
//
// Bound: memory.  dout and x are read once and dx is written once, where three products after one another would write and
// read the upstream gradient behind the activation (G) as well, and x and dout twice.  131072 x 64 -> 192 21 us, 84 MB at 4.0 TB/s;
// 131072 x 64 -> 256 with GELU 67 us, 101 MB: there it is forming G, an exponential, a reciprocal and an exponential an element (22 us
// of the special function units) and what is around them, by warps that empty the dx of the tile before as well (schedulers issue in
// 49 % of the cycles, the first stall is the wait for loads).  (Forward and backward 41 and 97 us; with three products, and a
// shorter polynomial for GELU, 49 and 152 where this took 93.)
//
// A CTA an SM walks tiles of 128 rows.  x and dout of a tile come by TMA (or x from its 8 bits, see below), the weight once.  Per tile
//   pre = x W^T           (with an activation)   128 x outs   rows of x and of the weight along k
//   G = dout o act'(pre + bias) as a sum of two bf16, the first in place of dout in shared memory (rounded to one, its
//       error would be as large as that of the results' own rounding); 128 columns of outs at a time
//   dx = G W              128 x cols             the weight as it lies: k runs down its rows
//   dW += G^T x or x^T G  k runs down the rows of both; stays in tensor memory to the end
//   db += 1^T G or G^T 1  ones in the lanes behind those of x where there are 64 left, else with 16 columns of them
// so that every product finds its operands where they lie.  (A product of 16 steps takes 43 clocks and half a clock a column, mostly
// its first operand's way from shared memory: few columns are dear.)  At its end a CTA leaves its sums for the join.
// Warps 0 - 15 form G (or bring x from its 8 bits, where there is no activation) and empty the dx of the tile before, 16 loads, 17
// issues the products: the next step's pre among this one's dx and dW, as soon as its rows are there, so that the next G is formed
// beside them.  (Shared memory holds two steps of wide layers: a step's rows are asked for when the products of the one before
// the last have ended, and into L2 a step earlier.)
#include "linear_tc.cuh"

namespace blossom {
namespace linear {
namespace {

using namespace tc;

constexpr int kRows = 128, kBlock = kRows * kSlabRow;  // a tile's rows; bytes of 64 columns of them
constexpr int kWarps = 16, kThreads = 32 * (kWarps + 4);
constexpr int kPieces = 4;  // of 16 codes a thread and tile: 128 rows of 16 pieces at most
constexpr int kStaging = 32 * 64, kSums = 32 * 17 * 4;  // of a warp: for dx, and for the sums at the end (in place of the ring)
constexpr int kOnes = 16 * kSlabRow;

int up(int n, int to) { return (n + to - 1) / to * to; }

// Where everything is; the same for the host and the kernel.
struct Plan {
  int cols16, outs16;        // rounded to 16: widths of the products
  int xb, gb;                // blocks of 64 columns of x and of dout
  int gw, nb;                // those of dout that are worked on at a time, and how often that is a tile
  int parts;                 // of G
  int wide_outs;             // the lanes of dW are outs (else cols)
  int ones_in_lanes;         // the last block of 64 of the lanes is ones: db
  int mb, gmb;               // blocks of 128 of the wider side, and of outs
  int narrow16, narrow32;    // columns of dW in tensor memory, of a block
  int t_pre, t_dx, t_dw, t_db, t_cols;  // columns of tensor memory
  int drains;                // groups of four warps that empty dx (three of the four leave room for two tiles of 320 columns)
  int stages, w_bytes, smem;
};

bool make_plan(int cols, int outs, bool act, Plan *p) {
  if (cols > 256 || outs > 256) return false;
  p->cols16 = up(cols, 16), p->outs16 = up(outs, 16);
  p->xb = (cols + 63) / 64, p->gb = (outs + 63) / 64;
  p->ones_in_lanes = p->xb % 2;
  p->wide_outs = !p->ones_in_lanes && outs >= cols;
  const int wide = p->wide_outs ? outs : cols;
  p->narrow16 = p->wide_outs ? p->cols16 : p->outs16, p->narrow32 = up(p->narrow16, 32);
  p->mb = (wide + 127) / 128, p->gmb = (outs + 127) / 128;
  p->t_pre = 0;
  p->gw = act && p->gb > 2 ? 2 : p->gb, p->nb = (p->gb + p->gw - 1) / p->gw, p->parts = act ? 2 : 1;
  p->t_dx = act ? up(outs < 128 ? outs : 128, 32) : 0;
  p->t_dw = p->t_dx + up(cols, 32);
  p->t_db = p->t_dw + p->mb * p->narrow32;
  const int n = p->t_db + (p->ones_in_lanes ? 0 : 16 * p->gmb);
  if (n > 512) return false;
  p->t_cols = n <= 128 ? 128 : n <= 256 ? 256 : 512;
  p->w_bytes = p->xb * p->outs16 * kSlabRow;
  // (a product's blocks of 128 may reach past the last block of 64, into the next tile or what lies behind the ring: lanes that
  // nobody reads)
  p->drains = cols <= 32 ? 1 : cols <= 64 ? 2 : 3;
  const int behind = up(p->w_bytes, 1024) + kOnes + 4 * p->drains * kStaging, rest = 1024 + (behind > kBlock ? behind : kBlock);
  const int stage = (p->xb + p->gw * p->parts) * kBlock, most = 227 * 1024 - 3 * 1024;
  p->stages = (most - rest) / stage;
  if (p->stages > 4) p->stages = 4;
  p->smem = rest + p->stages * stage;
  return p->stages >= 2;
}

struct Params {
  Plan plan;
  int rows, cols, outs, tiles, act;
  int load_x;                    // x comes by TMA
  const __nv_bfloat16 *bias;
  __nv_bfloat16 *dx;
  int64_t ld_dx;
  int wo;                        // elements a store
  const int8_t *codes;           // x in 8 bits, or null
  const uint8_t *scales;
  float *part, *part_bias;       // of this CTA on: [gridDim][wide][narrow], [gridDim][outs]; null: not wanted
  int32_t *status;
  int clear;                     // the status words first
};

// f(activation), known to the compiler; none of them without ACT
template <bool ACT, typename F>
__device__ __forceinline__ void with_slope(int act, F &&f) {
  using std::integral_constant;
  if constexpr (!ACT) f(integral_constant<int, BLOSSOM_ACT_NONE>());
  else if (act == BLOSSOM_ACT_RELU) f(integral_constant<int, BLOSSOM_ACT_RELU>());
  else if (act == BLOSSOM_ACT_GELU) f(integral_constant<int, BLOSSOM_ACT_GELU>());
  else f(integral_constant<int, BLOSSOM_ACT_SILU>());
}

template <bool ACT>
__global__ void __launch_bounds__(kThreads, 1)
    narrow_bwd_kernel(const __grid_constant__ CUtensorMap tx, const __grid_constant__ CUtensorMap tg,
                      const __grid_constant__ CUtensorMap tw, const __grid_constant__ Params p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[20];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  __shared__ __align__(16) float bias[2][256];  // [1]: zeros, for rows that are not there (a bias may be no number)
  grid_chain_enter();
  const Plan &q = p.plan;
  const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
  const uint32_t raw = smem_u32(smem_raw);
  uint8_t *const ring = smem_raw + (((raw + 1023u) & ~1023u) - raw);
  const int stage_bytes = (q.xb + q.gw * q.parts) * kBlock, stages = q.stages;
  uint8_t *const w_tile = ring + stages * stage_bytes, *const ones = w_tile + (q.w_bytes + 1023) / 1024 * 1024,
          *const staging0 = ones + kOnes;
  const uint32_t b_full = smem_u32(&bars[0]), b_empty = smem_u32(&bars[4]), b_w = smem_u32(&bars[8]), b_pre = smem_u32(&bars[9]),
                 b_g = smem_u32(&bars[14]), b_dx = smem_u32(&bars[11]), b_free = smem_u32(&bars[12]), b_all = smem_u32(&bars[13]);
  const bool packed = p.codes != nullptr;
  if (tid == 0) {
    abort_flag = 0;
    if (p.clear && blockIdx.x == 0)
      for (int i = 0; i < 8; ++i) p.status[i] = 0;  // (a wait that runs out does so long after this)
    for (int i = 0; i < stages; ++i) {
      mbar_init(b_full + 8 * i, packed ? 1 + kWarps : 1);
      mbar_init(b_empty + 8 * i, 1);
    }
    mbar_init(b_w, 1);
    mbar_init(b_pre, 1);
    for (int i = 0; i < stages; ++i) mbar_init(b_g + 8 * i, kWarps);
    mbar_init(b_dx, 1);
    mbar_init(b_free, 4 * q.drains);
    mbar_init(b_all, 1);
    mbar_fence_init();
  }
  for (int i = tid; i < kOnes / 4; i += kThreads) reinterpret_cast<uint32_t *>(ones)[i] = 0x3f803f80u;
  if (ACT) {
    const __nv_bfloat16 *const b = behind_wait(p.bias);
    for (int i = tid; i < 256; i += kThreads) bias[0][i] = b && i < p.outs ? __bfloat162float(b[i]) : 0.f, bias[1][i] = 0.f;
  }
  fence_async_smem();
  if (warp == 17) {
    tmem_alloc(smem_u32(&tmem_slot), q.t_cols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = (uint32_t)uniform((int)tmem_slot);
  const int mine = (p.tiles - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;  // tiles of this CTA
  const int nb = ACT ? q.nb : 1, steps = mine * nb;  // a step: a tile, or 128 columns of its outs
  const bool sums = p.part != nullptr || p.part_bias != nullptr;

  if (warp == 16) {
    // ---- loads: the weight, then x and dout tile by tile ----
    if (elect_one()) {
      mbar_expect_tx(b_w, q.w_bytes);
      for (int b = 0; b < q.xb; ++b) tma_load_2d(smem_u32(w_tile) + b * q.outs16 * kSlabRow, &tw, b_w, 64 * b, 0);
    }
    __syncwarp();
    bool go = true;
    for (int j = 0; j < steps; ++j) {
      const int at = j % stages, i = j / nb, n = j - i * nb, row0 = ((int)blockIdx.x + i * (int)gridDim.x) * kRows;
      const int blocks = min(q.gw, q.gb - n * q.gw);
      if (j >= stages) go = mbar_wait(b_empty + 8 * at, (j / stages - 1) & 1, &abort_flag, 401) && go;
      const uint32_t to = smem_u32(ring) + at * stage_bytes, bar = b_full + 8 * at;
      const int later = (j + stages) / nb, n2 = j + stages - later * nb, row2 = ((int)blockIdx.x + later * (int)gridDim.x) * kRows;
      if (elect_one() && go) {
        mbar_expect_tx(bar, ((p.load_x ? q.xb : 0) + blocks) * kBlock);
        for (int b = 0; b < blocks; ++b) tma_load_2d(to + (q.xb + b) * kBlock, &tg, bar, 64 * (n * q.gw + b), row0);
        if (p.load_x)
          for (int b = 0; b < q.xb; ++b) tma_load_2d(to + b * kBlock, &tx, bar, 64 * b, row0);
        if (ACT && later < mine) {
          for (int b = 0; b < min(q.gw, q.gb - n2 * q.gw); ++b) tma_prefetch_2d(&tg, 64 * (n2 * q.gw + b), row2);
          if (p.load_x && n2 == 0)
            for (int b = 0; b < q.xb; ++b) tma_prefetch_2d(&tx, 64 * b, row2);
        }
      }
      __syncwarp();
    }
  } else if (warp == 17) {
    // ---- products ----
    constexpr uint64_t kDown = (16 * kSlabRow) >> 4, kAlong = 2;  // a step of 16 of k, down the rows and along them
    constexpr uint32_t kAtom = 8 * kSlabRow;
    const uint64_t dones = smem_desc(smem_u32(ones), 16, kAtom, 2);
    const uint32_t i_dx = instr_desc(kRows, q.cols16, 0, 1), i_db = instr_desc(kRows, 16, 1, 0);
    const uint32_t w_block = q.outs16 * kSlabRow;
    auto width = [&](int n) { return min(64 * q.gw, q.outs16 - 64 * q.gw * n); };
    auto pre = [&](int j) {
      const int n = j % nb;
      const uint32_t x = smem_u32(ring) + j % stages * stage_bytes, w = smem_u32(w_tile) + 64 * q.gw * n * kSlabRow;
      const uint32_t idesc = instr_desc(kRows, width(n), 0, 0);
      uint64_t dx = smem_desc(x, 16, kAtom, 2), dw = smem_desc(w, 16, kAtom, 2);
      for (int c = 0; c < q.cols16; c += 64, dx += kBlock >> 4, dw += w_block >> 4) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (c + 16 * k < q.cols16) umma_bf16(tmem + q.t_pre, dx + k * kAlong, dw + k * kAlong, idesc, (c | k) != 0);
      }
      umma_commit(b_pre);
    };
    mbar_wait(b_w, 0, &abort_flag, 402);
    if (ACT) {
      mbar_wait(b_full, 0, &abort_flag, 403);
      tc_fence_after();
      if (elect_one()) pre(0);
      __syncwarp();
    }
    for (int j = 0; j < steps; ++j) {
      const int at = j % stages, i = j / nb, n = j - i * nb;
      const uint32_t x = smem_u32(ring) + at * stage_bytes, g0 = x + q.xb * kBlock;
      bool ahead = !ACT || j + 1 == steps;  // the next pre is on its way
      auto look = [&](bool wait) {
        if (ahead) return;
        const uint32_t bar = b_full + 8 * ((j + 1) % stages), parity = (j + 1) / stages & 1;
        if (wait) mbar_wait(bar, parity, &abort_flag, 405);
        else if (!mbar_done(bar, parity)) return;
        ahead = true;
        tc_fence_after();
        if (elect_one()) pre(j + 1);
        __syncwarp();
      };
      if (ACT) mbar_wait(b_g + 8 * at, j / stages & 1, &abort_flag, 404);
      else mbar_wait(b_full + 8 * at, j / stages & 1, &abort_flag, 406);
      look(false);
      const int wide = width(n);
      if (p.dx && n == 0 && i > 0) mbar_wait(b_free, (i - 1) & 1, &abort_flag, 407);
      tc_fence_after();
      for (int part = 0; part < q.parts; ++part) {
        const uint32_t g = g0 + part * q.gw * kBlock;
        if (p.dx && elect_one()) {
          uint64_t dg = smem_desc(g, 16, kAtom, 2), dw = smem_desc(smem_u32(w_tile) + 64 * q.gw * n * kSlabRow, w_block, kAtom, 2);
          for (int c = 0; c < wide; c += 64, dg += kBlock >> 4, dw += 4 * kDown) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (c + 16 * k < wide) umma_bf16(tmem + q.t_dx, dg + k * kAlong, dw + k * kDown, i_dx, (n | part | c | k) != 0);
          }
          if (n + 1 == nb && part + 1 == q.parts) umma_commit(b_dx);
        }
        __syncwarp();
        look(false);
        if (elect_one()) {
          if (p.part || (p.part_bias && q.ones_in_lanes)) {
            // the lanes: outs, of which a step has 128 with an activation and all without; or cols, all of them
            const uint64_t dn = smem_desc(q.wide_outs ? x : g, kBlock, kAtom, 2);
            const uint32_t idesc = instr_desc(kRows, q.wide_outs ? q.cols16 : wide, 1, 1);
            const int blocks = ACT && q.wide_outs ? 1 : q.mb;
            for (int m = 0; m < blocks; ++m) {
              const uint32_t from = (q.wide_outs ? g : x) + 2 * m * kBlock;
              // the second block of 64 lanes: the next one, or the ones, the same for every step down the rows
              const bool to_ones = q.ones_in_lanes && m + 1 == q.mb;
              const uint64_t dm = smem_desc(from, to_ones ? smem_u32(ones) - from : kBlock, kAtom, 2);
              const uint64_t down = to_ones ? kDown - (kDown << 16) : kDown;
              const uint32_t d = tmem + q.t_dw + (ACT && q.wide_outs ? n : m) * q.narrow32 + (q.wide_outs ? 0 : 64 * q.gw * n);
#pragma unroll
              for (int k = 0; k < kRows / 16; ++k) umma_bf16(d, dm + k * down, dn + k * kDown, idesc, (i | part | k) != 0);
            }
          }
          if (p.part_bias && !q.ones_in_lanes) {
            for (int m = 0; m < (ACT ? 1 : q.gmb); ++m) {
              const uint64_t dm = smem_desc(g + 2 * m * kBlock, kBlock, kAtom, 2);
#pragma unroll
              for (int k = 0; k < kRows / 16; ++k)
                umma_bf16(tmem + q.t_db + (ACT ? n : m) * 16, dm + k * kDown, dones, i_db, (i | part | k) != 0);
            }
          }
          if (part + 1 == q.parts) {
            umma_commit(b_empty + 8 * at);
            if (j + 1 == steps) umma_commit(b_all);
          }
        }
        __syncwarp();
        look(false);
      }
      look(true);
    }
  } else if (warp < kWarps) {
    // ---- per tile: G, or x from its 8 bits; then dx of the tile before ----
    const int quarter = warp & 3, turn = warp >> 2, r = 32 * quarter + lane;
    uint8_t *const staging = staging0 + warp * kStaging;
    // codes of a tile: 16 of a row a thread at a time, asked for a tile ahead
    const int pieces = packed ? p.cols / 16 : 1, slots = 32 * kWarps / pieces, slot = tid / pieces, column = tid - slot * pieces;
    const int8_t *const codes = behind_wait(p.codes) + 16 * column;
    const uint8_t *const scales = behind_wait(p.scales) + column / 2;
    uint4 next[kPieces];
    uint32_t exps[kPieces];
    auto ask = [&](int i) {
      const int row0 = ((int)blockIdx.x + i * (int)gridDim.x) * kRows;
#pragma unroll
      for (int u = 0; u < kPieces; ++u) {
        const int rr = slot + u * slots;
        const bool there = slot < slots && rr < kRows && row0 + rr < p.rows;
        next[u] = make_uint4(0, 0, 0, 0), exps[u] = 0;
        if (there) {
          next[u] = *reinterpret_cast<const uint4 *>(codes + (int64_t)(row0 + rr) * p.cols);
          exps[u] = scales[(int64_t)(row0 + rr) * (p.cols / 32)];
        }
      }
    };
    if (!ACT && packed) ask(0);
    auto drain = [&](int i) {  // dx of a tile: 32 rows, 32 columns at a time
      if (!p.dx || turn >= q.drains) return;
      const int row0 = ((int)blockIdx.x + i * (int)gridDim.x) * kRows + 32 * quarter, rows = p.rows - row0;
      mbar_wait(b_dx, i & 1, &abort_flag, 411);
      tc_fence_after();
#pragma unroll 1
      for (int c = 32 * turn; c < p.cols; c += 32 * q.drains) {
        if (rows <= 0) break;
        float v[32];
        tmem_ld32(tmem + q.t_dx + c + ((uint32_t)(32 * quarter) << 16), v);
        tmem_wait_ld();
#pragma unroll
        for (int k = 0; k < 4; ++k)
          *piece(staging, lane, k) = make_uint4(pack_bf16(v[8 * k], v[8 * k + 1]), pack_bf16(v[8 * k + 2], v[8 * k + 3]),
                                                pack_bf16(v[8 * k + 4], v[8 * k + 5]), pack_bf16(v[8 * k + 6], v[8 * k + 7]));
        __syncwarp();
        __nv_bfloat16 *const to = p.dx + (int64_t)row0 * p.ld_dx + c;
        if (rows >= 32 && p.cols - c >= 32 && p.wo == 8) write_whole(staging, to + (int64_t)(lane >> 2) * p.ld_dx + 8 * (lane & 3), 8 * p.ld_dx);
        else write_ragged(staging, to, p.ld_dx, rows, p.cols - c, p.wo);
        __syncwarp();
      }
      tc_fence_before();
      warp_arrive(b_free, lane);
    };
    with_slope<ACT>(p.act, [&](auto act) {
      const Curve<decltype(act)::value, true> curve;
      for (int j = 0; j < steps; ++j) {
        const int at = j % stages, i = j / nb, n = j - i * nb;
        if (ACT) {  // G in place of dout: a row a thread, every fourth 16 columns
          const int first = 64 * q.gw * n, wide = min(64 * q.gw, q.outs16 - first);
          const float *const own_bias = bias[((int)blockIdx.x + i * (int)gridDim.x) * kRows + r < p.rows ? 0 : 1] + first;
          uint8_t *const g = ring + at * stage_bytes + q.xb * kBlock + r * kSlabRow;
          mbar_wait(b_full + 8 * at, j / stages & 1, &abort_flag, 408);
          mbar_wait(b_pre, j & 1, &abort_flag, 409);
          tc_fence_after();
          float v[16];
          const uint32_t from = tmem + q.t_pre + ((uint32_t)(32 * quarter) << 16);
          if (16 * turn < wide) tmem_ld16(from + 16 * turn, v);
#pragma unroll 1
          for (int c = 16 * turn; c < wide; c += 64) {
            wait_for(v);
            float y[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) y[k] = v[k];
            if (c + 64 < wide) tmem_ld16(from + c + 64, v);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint4 *const to = reinterpret_cast<uint4 *>(g + c / 64 * kBlock + (((c % 64 / 8 + h) ^ (r & 7)) << 4));
              uint4 low;
              *to = finish8_parts(curve, &y[8 * h], own_bias + c + 8 * h, *to, low);
              to[q.gw * kBlock / 16] = low;
            }
          }
          tc_fence_before();
          fence_async_smem();
          warp_arrive(b_g + 8 * at, lane);
        } else if (packed) {
          if (j >= stages) mbar_wait(b_empty + 8 * at, (j / stages - 1) & 1, &abort_flag, 410);
          uint8_t *const x = ring + at * stage_bytes + column / 4 * kBlock;
#pragma unroll
          for (int u = 0; u < kPieces; ++u) {
            const int rr = slot + u * slots;
            if (slot >= slots || rr >= kRows) break;
            const float f = rows::value_per_code(exps[u]);
            const uint32_t w[4] = {next[u].x, next[u].y, next[u].z, next[u].w};
            uint32_t o[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const uint32_t two = w[k / 2] >> (16 * (k & 1));
              o[k] = pack_bf16((float)(int8_t)two * f, (float)(int8_t)(two >> 8) * f);
            }
            uint8_t *const to = x + rr * kSlabRow;
            *reinterpret_cast<uint4 *>(to + (((column % 4 * 2) ^ (rr & 7)) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
            *reinterpret_cast<uint4 *>(to + (((column % 4 * 2 + 1) ^ (rr & 7)) << 4)) = make_uint4(o[4], o[5], o[6], o[7]);
          }
          fence_async_smem();
          warp_arrive(b_full + 8 * at, lane);
          if (j + 1 < steps) ask(j + 1);
        }
        if (n == 0 && i > 0) drain(i - 1);
      }
      drain(mine - 1);
    });
  }
  // ---- the sums ----
  if (warp < kWarps && sums) {
    mbar_wait(b_all, 0, &abort_flag, 412);
    tc_fence_after();
    const int quarter = warp & 3, turn = warp >> 2, wide = q.wide_outs ? p.outs : p.cols, narrow = q.wide_outs ? p.cols : p.outs;
    float *const t = reinterpret_cast<float *>(ring + warp * kSums);  // (every copy and product has ended)
    const uint32_t lanes = (uint32_t)(32 * quarter) << 16;
    if (p.part) {
      const int per = q.narrow16 / 16;
      for (int u = turn; u < q.mb * per; u += 4) {
        const int m = u / per, c = u % per * 16, r0 = m * 128 + 32 * quarter;
        float v[16];
        tmem_ld16(tmem + q.t_dw + m * q.narrow32 + c + lanes, v);
        tmem_wait_ld();
        write_sums(v, t, p.part + ((int64_t)blockIdx.x * wide + r0) * narrow + c, narrow, wide - r0, narrow - c);
      }
    }
    if (p.part_bias && q.ones_in_lanes) {
      if (quarter == 2)  // the ones' first lane
        for (int c = 16 * turn; c < p.outs; c += 64) {
          float v[16];
          tmem_ld16(tmem + q.t_dw + (q.mb - 1) * q.narrow32 + c + lanes, v);
          tmem_wait_ld();
          if (lane == 0) {
#pragma unroll
            for (int k = 0; k < 16; ++k)
              if (c + k < p.outs) p.part_bias[(int64_t)blockIdx.x * p.outs + c + k] = v[k];
          }
        }
    } else if (p.part_bias && turn < q.gmb) {
      float v[16];
      tmem_ld16(tmem + q.t_db + turn * 16 + lanes, v);
      tmem_wait_ld();
      const int o = turn * 128 + 32 * quarter + lane;
      if (o < p.outs) p.part_bias[(int64_t)blockIdx.x * p.outs + o] = v[0];
    }
  }
  finish(warp == 17 ? 0 : 1, tmem, q.t_cols, &abort_flag, p.status);
}

}  // namespace

int narrow_splits(int rows) {
  const int tiles = parts_of(rows, kRows);
  return tiles < kSMs ? tiles : kSMs;
}

bool narrow_takes(const NarrowBackward &n) {
  Plan p;
  if (!make_plan(n.cols, n.outs, n.act != 0, &p)) return false;
  if (n.codes ? n.act || n.cols % 32 || reinterpret_cast<uintptr_t>(n.codes) % 16 : n.x && !tma_takes(n.x, n.ld_x)) return false;
  return tma_takes(n.dout, n.ld_dout) && tma_takes(n.weight, n.ld_weight);
}

bool narrow_turned(const NarrowBackward &n) {
  Plan p;
  return make_plan(n.cols, n.outs, n.act != 0, &p) && !p.wide_outs;
}

int launch_narrow(const NarrowBackward &n, cudaStream_t st) {
  Params p = {};
  if (!make_plan(n.cols, n.outs, n.act != 0, &p.plan)) return BLOSSOM_ERR_UNSUPPORTED;
  p.rows = n.rows, p.cols = n.cols, p.outs = n.outs, p.tiles = parts_of(n.rows, kRows), p.act = n.act;
  p.bias = static_cast<const __nv_bfloat16 *>(n.bias), p.dx = static_cast<__nv_bfloat16 *>(n.dx), p.ld_dx = n.ld_dx;
  p.codes = n.codes, p.scales = n.scales, p.part = n.part, p.part_bias = n.part_bias, p.status = n.status, p.clear = !n.later;
  rows::Alignment al;
  al.rows_at(n.dx, n.ld_dx, 2);
  p.wo = al.elements(n.cols, 2);
  CUtensorMap tx = {}, tg = {}, tw = {};
  p.load_x = !n.codes && n.x;
  if (p.load_x && !make_map(&tx, n.x, n.rows, n.cols, n.ld_x, kRows)) return BLOSSOM_ERR_CUDA;
  if (!make_map(&tg, n.dout, n.rows, n.outs, n.ld_dout, kRows) || !make_map(&tw, n.weight, n.outs, n.cols, n.ld_weight, p.plan.outs16))
    return BLOSSOM_ERR_CUDA;
  const auto kern = n.act ? narrow_bwd_kernel<true> : narrow_bwd_kernel<false>;
  // (one value for all of a kernel's launches: host threads share it)
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - 3 * 1024) != cudaSuccess) return BLOSSOM_ERR_CUDA;
  {
    LaunchScope ls(K_LINEAR_NARROW, st);
    launch_chained(kern, dim3((unsigned)narrow_splits(n.rows)), dim3(kThreads), (size_t)p.plan.smem, st, tx, tg, tw, p);
  }
  return cudaGetLastError() == cudaSuccess ? BLOSSOM_OK : BLOSSOM_ERR_CUDA;
}

}  // namespace linear
}  // namespace blossom
