// Products of bf16 matrices on the tensor cores (tcgen05, fp32 accumulators in tensor memory), with what follows them.
//
// A CTA an SM walks tiles of 128 x BN elements, the columns' tiles of a row tile one after another, so that the CTAs that run at
// once share their operands in L2.  Slabs of 64 steps of k come into a ring in shared memory (128-byte swizzle), either by TMA,
// where rows are 16 bytes apart, or by eight warps with plain loads, which take any alignment; one warp issues the products;
// eight warps empty an accumulator; two groups of them take the tiles in turn, of two to four accumulators, so that a tile's epilogue
// runs beside the next tile's and the products of those after.
// An operand whose k runs down the rows of memory is taken as it lies there (MN-major).
//
// Epilogue: a warp has 32 rows and 32 columns at a time.  A row is a thread's (its lane of tensor memory); memory is touched by
// whole rows of the 32 columns, four lanes a row, and shared memory turns one into the other.
//
// Bound: 131072 x 64 -> 256 with GELU 27 us, the epilogue's instructions (84 MB, 3.1 TB/s; with a shorter polynomial 24, then two
// accumulators 26, one and half the warps 31);
// 32768 x 1024 -> 4096 209 us forward, 223 dx, 272 dW and 29 the join of its two splits, the power (1.3 PFLOP/s, 94 % of what a
// library product sustains).  Rows that TMA does not take cost more the narrower the access: 32768 x 1023 -> 4096 2011 us forward,
// 2351 dx, 3266 dW, 96 loads of two bytes a thread and slab; 60000 x 490 -> 470 127, 121, 111 where 496 -> 472 takes 43, 45, 41.
#include "linear_tc.cuh"

namespace blossom {
namespace linear {
namespace {

using namespace tc;

constexpr int kM = 128, kK = 64, kGroupWarps = 8, kLoaderWarps = 8;  // kGroupWarps: of an accumulator
constexpr size_t kMostSmem = 227 * 1024 - 3 * 1024;     // (what the kernels' own arrays take besides)

// Rounded to whole atoms: what a stage, the staging of a warp, and the ones take.
template <int BN, bool PARTIAL, bool PLAIN>
struct Shape_ {
  static constexpr int kA = kM * kSlabRow, kB = BN * kSlabRow, kStage = kA + kB;
  // (the plain loads' registers leave room for one group of epilogue warps)
  static constexpr int kGroups = PARTIAL || PLAIN ? 1 : 2, kEpilogueWarps = kGroups * kGroupWarps;
  static constexpr int kThreads = 32 * (kEpilogueWarps + 4 + (PLAIN ? kLoaderWarps : 0));
  static constexpr int kStaging = PARTIAL ? 32 * 17 * 4 : 32 * 64;  // of a warp
  static constexpr int kOnes = PARTIAL ? 16 * kSlabRow : 0;
  static constexpr int kRest = 1024 + kOnes + kEpilogueWarps * kStaging;
  static constexpr int kFit = ((int)kMostSmem - kRest) / kStage, kStages = kFit < 8 ? kFit : 8;
  static constexpr int kSmem = kRest + kStages * kStage;
  static constexpr int kAccs = PARTIAL ? 1 : BN <= 128 ? 4 : 2;
  static constexpr int kCols = BN * kAccs + (PARTIAL ? 32 : 0), kTmem = kCols <= 128 ? 128 : kCols <= 256 ? 256 : 512;
};

struct Params {
  int m, n, k, mt, nt, items;   // items: tiles (of every split)
  int a_along, b_along;
  int slabs, slabs_per_split;
  int parts;                    // of A: 2 with a low one, whose slabs follow the first part's
  // plain loads
  const __nv_bfloat16 *a, *a_low, *b;
  int64_t lda, ldb;
  int w;                        // elements a load
  int nb;                       // columns of B that are there
  // epilogue
  int slope, act, wo;           // wo: elements a store, and a load of what the epilogue reads
  const __nv_bfloat16 *bias, *extra;
  int64_t ld_extra, ld_out;
  __nv_bfloat16 *out, *out_low;
  float *part, *part_bias;
  int32_t *status;
  int clear;                    // the status words first
};

template <int BN, bool PARTIAL, bool PLAIN>
__global__ void __launch_bounds__(Shape_<BN, PARTIAL, PLAIN>::kThreads, 1)
    product_tc_kernel(const __grid_constant__ CUtensorMap ta, const __grid_constant__ CUtensorMap ta_low,
                      const __grid_constant__ CUtensorMap tb, const __grid_constant__ Params p) {
  using S = Shape_<BN, PARTIAL, PLAIN>;
  constexpr int STAGES = S::kStages, ACCS = S::kAccs, GROUPS = S::kGroups, WARPS = S::kEpilogueWarps;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * STAGES + 2 * ACCS];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  __shared__ __align__(16) float bias_row[WARPS][32];
  grid_chain_enter();
  const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
  const uint32_t raw = smem_u32(smem_raw);
  uint8_t *const ring = smem_raw + (((raw + 1023u) & ~1023u) - raw);
  uint8_t *const ones = ring + STAGES * S::kStage, *const staging0 = ones + S::kOnes;
  const uint32_t b_full = smem_u32(&bars[0]), b_empty = smem_u32(&bars[STAGES]), b_acc = smem_u32(&bars[2 * STAGES]),
                 b_free = smem_u32(&bars[2 * STAGES + ACCS]);
  if (tid == 0) {
    abort_flag = 0;
    if (p.clear && blockIdx.x == 0)
      for (int i = 0; i < 8; ++i) p.status[i] = 0;  // (a wait that runs out does so long after this)
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(b_full + 8 * i, PLAIN ? kLoaderWarps : 1);
      mbar_init(b_empty + 8 * i, 1);
    }
    for (int i = 0; i < ACCS; ++i) {
      mbar_init(b_acc + 8 * i, 1);
      mbar_init(b_free + 8 * i, kGroupWarps);
    }
    mbar_fence_init();
  }
  if (PARTIAL)
    for (int i = tid; i < S::kOnes / 4; i += blockDim.x) reinterpret_cast<uint32_t *>(ones)[i] = 0x3f803f80u;
  if (PARTIAL) fence_async_smem();
  if (warp == WARPS + 1) {
    tmem_alloc(smem_u32(&tmem_slot), S::kTmem);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = (uint32_t)uniform((int)tmem_slot);
  const int tiles = p.mt * p.nt;
  // the slabs of an item
  auto slabs_of = [&](int item, int &first) {
    first = PARTIAL ? item / tiles * p.slabs_per_split : 0;
    return PARTIAL ? min(p.slabs_per_split, p.slabs - first) : p.slabs;
  };

  if (!PLAIN && warp == WARPS) {
    // ---- loads by TMA ----
    bool go = true;
    uint32_t j = 0;
    for (int item = blockIdx.x; item < p.items; item += gridDim.x) {
      const int tile = item % tiles, m0 = tile / p.nt * kM, n0 = tile % p.nt * BN;
      int first;
      const int count = slabs_of(item, first);
      for (int s = 0; s < count * p.parts; ++s, ++j) {
        const uint32_t at = j % STAGES, bar = b_full + 8 * at, to = smem_u32(ring + at * S::kStage);
        if (j >= STAGES) go = mbar_wait(b_empty + 8 * at, (j / STAGES - 1) & 1, &abort_flag, 301) && go;
        const int k0 = (first + (s < count ? s : s - count)) * kK;
        if (elect_one() && go) {
          const CUtensorMap *const from = s < count ? &ta : &ta_low;
          mbar_expect_tx(bar, S::kStage);
          if (p.a_along) {
            tma_load_2d(to, from, bar, k0, m0);
          } else {
            for (int i = 0; i < kM; i += 64) tma_load_2d(to + i * kSlabRow, from, bar, m0 + i, k0);
          }
          if (p.b_along) {
            tma_load_2d(to + S::kA, &tb, bar, k0, n0);
          } else {
            for (int i = 0; i < BN; i += 64) tma_load_2d(to + S::kA + i * kSlabRow, &tb, bar, n0 + i, k0);
          }
        }
        __syncwarp();
      }
    }
  } else if (PLAIN && warp >= WARPS + 4) {
    // ---- plain loads ----
    const __nv_bfloat16 *const a = behind_wait(p.a), *const a_low = behind_wait(p.a_low), *const b = behind_wait(p.b);
    const int t = tid - 32 * (WARPS + 4);
    auto go = [&](auto w) {
      constexpr int W = decltype(w)::value;
      Pieces<__nv_bfloat16, kM, kLoaderWarps, W> pa;
      Pieces<__nv_bfloat16, BN, kLoaderWarps, W> pb;
      int item = blockIdx.x, s = 0, first = 0, m0 = 0, n0 = 0, count = 0;
      auto on = [&]() {  // to the item
        const int tile = item % tiles;
        m0 = tile / p.nt * kM, n0 = tile % p.nt * BN, count = slabs_of(item, first);
      };
      auto deep = [&]() { return (first + (s < count ? s : s - count)) * kK; };
      on();
      pa.ask(t, a, p.lda, p.a_along, m0, p.m, deep(), p.k);
      for (uint32_t j = 0; item < p.items; ++j) {
        const uint32_t at = j % STAGES;
        uint8_t *const to = ring + at * S::kStage;
        auto put = [&](int at, const uint32_t (&x)[4]) { *reinterpret_cast<uint4 *>(to + at) = make_uint4(x[0], x[1], x[2], x[3]); };
        auto put_b = [&](int at, const uint32_t (&x)[4]) { put(S::kA + at, x); };
        pb.ask(t, b, p.ldb, p.b_along, n0, p.nb, deep(), p.k);
        if (j >= STAGES) mbar_wait(b_empty + 8 * at, (j / STAGES - 1) & 1, &abort_flag, 302);
        pa.put(t, put);
        if (++s == count * p.parts) {
          s = 0, item += gridDim.x;
          if (item < p.items) on();
        }
        if (item < p.items) pa.ask(t, s < count ? a : a_low, p.lda, p.a_along, m0, p.m, deep(), p.k);
        pb.put(t, put_b);
        fence_async_smem();
        warp_arrive(b_full + 8 * at, lane);
      }
    };
    with_width(p.w, go);
  } else if (warp == WARPS + 1) {
    // ---- products ----
    const uint32_t idesc = instr_desc(kM, BN, !p.a_along, !p.b_along), idesc_ones = instr_desc(kM, 16, !p.a_along, 0);
    const uint32_t step_a = p.a_along ? 2 : (16 * kSlabRow) >> 4, step_b = p.b_along ? 2 : (16 * kSlabRow) >> 4;
    const uint32_t lead_a = p.a_along ? 16 : kK * kSlabRow, lead_b = p.b_along ? 16 : kK * kSlabRow;
    const uint64_t dones = smem_desc(smem_u32(ones), 16, 8 * kSlabRow, 2);
    uint32_t j = 0, turn = 0;
    for (int item = blockIdx.x; item < p.items; item += gridDim.x, ++turn) {
      const uint32_t acc = turn % ACCS, d = tmem + acc * BN;
      int first;
      const int count = slabs_of(item, first);
      const int share = PARTIAL ? item % tiles % p.nt : 0;  // the tiles of a row of them share out the sums over k alone
      if (turn >= ACCS) mbar_wait(b_free + 8 * acc, (turn / ACCS - 1) & 1, &abort_flag, 303);
      for (int s = 0; s < count * p.parts; ++s, ++j) {
        const uint32_t at = j % STAGES;
        mbar_wait(b_full + 8 * at, (j / STAGES) & 1, &abort_flag, 304);
        tc_fence_after();
        const uint32_t from = smem_u32(ring + at * S::kStage);
        const uint64_t da = smem_desc(from, lead_a, 8 * kSlabRow, 2), db = smem_desc(from + S::kA, lead_b, 8 * kSlabRow, 2);
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < kK / 16; ++k) umma_bf16(d, da + k * step_a, db + k * step_b, idesc, (s | k) != 0);
          if (PARTIAL && p.part_bias && (s < count ? s : s - count) % p.nt == share) {
#pragma unroll
            for (int k = 0; k < kK / 16; ++k) umma_bf16(d + BN, da + k * step_a, dones, idesc_ones, (s != share) | (k != 0));
          }
          umma_commit(b_empty + 8 * at);
          if (s + 1 == count * p.parts) umma_commit(b_acc + 8 * acc);
        }
        __syncwarp();
      }
    }
  } else if (warp < WARPS) {
    // ---- epilogue: lanes 32 * (warp % 4) on, of the columns the first or second half ----
    constexpr int HALF = BN / 2;
    const int quarter = warp & 3, half = warp >> 2 & 1, group = warp / kGroupWarps;
    const uint32_t lanes = (uint32_t)(32 * quarter) << 16;
    uint8_t *const staging = staging0 + warp * S::kStaging;
    if constexpr (PARTIAL) {
      float *const t = reinterpret_cast<float *>(staging);
      uint32_t turn = 0;
      for (int item = blockIdx.x; item < p.items; item += gridDim.x, ++turn) {
        const int tile = item % tiles, m0 = tile / p.nt * kM + 32 * quarter, n0 = tile % p.nt * BN + half * HALF, rows = p.m - m0;
        mbar_wait(b_acc, turn & 1, &abort_flag, 305);
        tc_fence_after();
        const int last = rows > 0 && (p.part || p.out) ? min(p.n - n0, HALF) : 0;
        if (p.out) {  // one split: the results themselves
          __nv_bfloat16 *const out = p.out + (int64_t)m0 * p.ld_out + n0;
#pragma unroll 1
          for (int c = 0; c < last; c += 32) {
            float v[2][16];
            tmem_ld16(tmem + half * HALF + c + lanes, v[0]);
            tmem_ld16(tmem + half * HALF + c + 16 + lanes, v[1]);
            wait_for(v[0]);
            wait_for(v[1]);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const float *const y = &v[q / 2][8 * (q % 2)];
              *piece(staging, lane, q) = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
            }
            __syncwarp();
            if (rows >= 32 && p.wo == 8 && p.n - n0 - c >= 32)
              write_whole(staging, out + (int64_t)(lane >> 2) * p.ld_out + 8 * (lane & 3) + c, 8 * p.ld_out);
            else
              write_ragged(staging, out + c, p.ld_out, rows, p.n - n0 - c, p.wo);
            __syncwarp();
          }
        } else {
          float *const to = p.part + ((int64_t)(item / tiles) * p.m + m0) * p.n + n0;
#pragma unroll 1
          for (int c = 0; c < last; c += 16) {
            float v[16];
            tmem_ld16(tmem + half * HALF + c + lanes, v);
            wait_for(v);
            write_sums(v, t, to + c, p.n, rows, p.n - n0 - c);
          }
        }
        if (half == 0 && rows > 0 && p.part_bias) {  // the sums over k alone: any of the 16 columns
          float v[16];
          tmem_ld16(tmem + BN + lanes, v);
          wait_for(v);
          int first;
          const int share = tile % p.nt;
          const bool any = share < slabs_of(item, first);  // (fewer slabs than tiles: nothing was added up)
          if (lane < rows) p.part_bias[((int64_t)(item / tiles) * p.nt + share) * p.m + m0 + lane] = any ? v[0] : 0.f;
        }
        tc_fence_before();
        warp_arrive(b_free, lane);
      }
    } else {
      const __nv_bfloat16 *const extra = behind_wait(p.extra), *const bias = behind_wait(p.bias);
      with_curve(p.act, p.slope, extra != nullptr, [&](auto act, auto slope, auto read) {
        constexpr bool SLOPE = decltype(slope)::value, READ = decltype(read)::value;
        const Curve<decltype(act)::value, SLOPE> curve;
        const int64_t out_step = 8 * p.ld_out, extra_step = 8 * p.ld_extra;
        uint32_t turn = group;
        for (int tile = blockIdx.x + group * gridDim.x; tile < p.items; tile += GROUPS * gridDim.x, turn += GROUPS) {
          const uint32_t acc = turn % ACCS;
          const int mt = p.nt == 1 ? tile : tile / p.nt, m0 = mt * kM + 32 * quarter, n0 = (tile - mt * p.nt) * BN + half * HALF;
          const int rows = p.m - m0, cols = p.n - n0;
          const uint32_t from = tmem + acc * BN + half * HALF + lanes;
          const bool some = rows > 0 && cols > 0, whole = rows >= 32 && p.wo == 8;  // (the same for the warp)
          __nv_bfloat16 *const out0 = p.out + (int64_t)m0 * p.ld_out + n0, *const out = out0 + (int64_t)(lane >> 2) * p.ld_out + 8 * (lane & 3);
          const __nv_bfloat16 *const extra0 = extra + (int64_t)m0 * p.ld_extra + n0,
                              *const own_extra = extra0 + (int64_t)(lane >> 2) * p.ld_extra + 8 * (lane & 3);
          // what memory has to give is asked for before the wait: the biases, and a block of 32 columns ahead what the epilogue reads
          float b[HALF / 32];
#pragma unroll
          for (int i = 0; i < HALF / 32; ++i) b[i] = bias && 32 * i + lane < cols ? __bfloat162float(bias[n0 + 32 * i + lane]) : 0.f;
          uint4 x[4];
          auto ask = [&](int c) {
            if (whole && cols - c >= 32) {
#pragma unroll
              for (int j = 0; j < 4; ++j) x[j] = *reinterpret_cast<const uint4 *>(own_extra + j * extra_step + c);
            }
          };
          if (READ) ask(0);
          mbar_wait(b_acc + 8 * acc, (turn / ACCS) & 1, &abort_flag, 305);
          tc_fence_after();
          if (some) {
            float v[2][16];
            uint4 low[4];
            tmem_ld16(from, v[0]);
#pragma unroll 1
            for (int c = 0; c < HALF && c < cols; c += 32) {
              const bool full = whole && cols - c >= 32;
              float own = b[0];
#pragma unroll
              for (int i = 1; i < HALF / 32; ++i) own = c == 32 * i ? b[i] : own;
              bias_row[warp][lane] = own;
              if (READ) {
                if (full) {
#pragma unroll
                  for (int j = 0; j < 4; ++j) *piece(staging, (lane >> 2) + 8 * j, lane & 3) = x[j];
                } else {
                  read_ragged(staging, extra0 + c, p.ld_extra, rows, cols - c, p.wo);
                }
                if (c + 32 < HALF) ask(c + 32);
              }
              __syncwarp();
#pragma unroll
              for (int h = 0; h < 2; ++h) {  // 16 columns, the next 16 under way
                wait_for(v[h]);
                if (h == 0) tmem_ld16(from + c + 16, v[1]);
                else if (c + 32 < HALF) tmem_ld16(from + c + 32, v[0]);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                  uint4 *const at = piece(staging, lane, 2 * h + q);
                  uint4 e = make_uint4(0, 0, 0, 0);
                  if (READ) e = *at;
                  if constexpr (SLOPE) *at = finish8_parts(curve, &v[h][8 * q], &bias_row[warp][16 * h + 8 * q], e, low[2 * h + q]);
                  else *at = finish8<READ>(curve, &v[h][8 * q], &bias_row[warp][16 * h + 8 * q], e);
                }
              }
              __syncwarp();
              if (full) write_whole(staging, out + c, out_step);
              else write_ragged(staging, out0 + c, p.ld_out, rows, cols - c, p.wo);
              __syncwarp();
              if (SLOPE && p.out_low) {
#pragma unroll
                for (int q = 0; q < 4; ++q) *piece(staging, lane, q) = low[q];
                __syncwarp();
                if (full) write_whole(staging, out + c + (p.out_low - p.out), out_step);
                else write_ragged(staging, out0 + c + (p.out_low - p.out), p.ld_out, rows, cols - c, p.wo);
                __syncwarp();
              }
            }
            wait_for(v[0]);  // (a load that nobody uses may be under way)
          }
          tc_fence_before();
          warp_arrive(b_free + 8 * acc, lane);
        }
      });
    }
  }
  finish(warp == WARPS + 1 ? 0 : 1, tmem, S::kTmem, &abort_flag, p.status);
}

template <int BN, bool PARTIAL, bool PLAIN>
int launch_one(int kernel_id, const CUtensorMap &ta, const CUtensorMap &ta_low, const CUtensorMap &tb, const Params &p, cudaStream_t st) {
  using S = Shape_<BN, PARTIAL, PLAIN>;
  const auto kern = product_tc_kernel<BN, PARTIAL, PLAIN>;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem) != cudaSuccess) return BLOSSOM_ERR_CUDA;
  {
    LaunchScope ls(kernel_id, st);
    launch_chained(kern, dim3((unsigned)(p.items < kSMs ? p.items : kSMs)), dim3(S::kThreads), S::kSmem, st, ta, ta_low, tb, p);
  }
  return cudaGetLastError() == cudaSuccess ? BLOSSOM_OK : BLOSSOM_ERR_CUDA;
}

int width_of(const void *p, int64_t ld, int cols) {
  rows::Alignment al;
  al.rows_at(p, ld, 2);
  return al.elements(cols, 2);
}

}  // namespace

bool make_map(CUtensorMap *map, const void *base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
  return encode_map(map, base, 2, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

// Columns of a tile.  What a tile costs beside its columns (its rows' operand, hand-offs) weighs as 64 of them, as 24 where the
// epilogue bounds (ends: few slabs, by TMA) and four accumulators hide the hand-offs: the width with the least work of the busiest SM.
// Forward, us with 64, 128, 192, 256 columns: 131072 x 64 -> 192 15.3, 18.4, 14.3, 15.4; 131072 x 64 -> 256 with GELU 29.9, 27.4, 36.8,
// 29.7; x 256 -> 64 10.4, 15.3, 20.1, 26.9; 32768 x 1024 -> 4096 with GELU 398, 264, 243, 232.
int tile_columns(int m, int n, int splits, bool ends) {
  const int64_t mt = ((int64_t)m + kM - 1) / kM * splits;
  int best = 64;
  int64_t least = INT64_MAX;
  for (int bn : {64, 128, 192, 256}) {
    const int64_t cost = (mt * ((n + bn - 1) / bn) + kSMs - 1) / kSMs * (bn + (ends && bn <= 128 ? 24 : 64));
    if (cost <= least) least = cost, best = bn;
  }
  return best;
}

int tc_splits(int m, int n, int k, int parts) {
  // In clocks: a slab of a tile 1.6 a column and 100, an item's hand-offs and epilogue 4000, a partial sum's way to memory and
  // back 8 bytes at 3500 a clock.  Forward and backward, us with 1, 4, 9, 16, 37 splits: 5000 x 512 -> 512 45, 32, 31, 31, 45 (the rule:
  // 32); 2000 x 1024 -> 1024 with GELU 60, 81, 100, 155, 214 (60).
  // No accumulator adds up more than kMostSlabs, those of both parts of A: it cuts its sums, which loses 2e-6 of sums of one sign
  // over 1024 steps of k.  (32768 x 1024 -> 4096 with GELU: dweight is 3e-5 too small with 256 slabs, 5e-5 with 512 and 1e-4 with
  // 1024, where plain single precision loses 5e-6 and the rounding to bf16 is off by 1.7e-3; the step takes 1767, 1744, 1746 us.)
  const int64_t slabs = parts_of(k, kK), mt = parts_of(m, kM), fewest = parts_of((int)slabs, kMostSlabs / parts);
  int best = 1;
  double least = 1e30;
  for (int bn : {64, 128, 192, 256}) {
    const int64_t tiles = mt * ((n + bn - 1) / bn);
    for (int waves = 0; waves <= 4; ++waves) {
      int64_t s = waves ? kSMs * waves / tiles : 1;
      s = s < fewest ? fewest : s > slabs ? slabs : s;
      const int64_t per = (slabs + s - 1) / s;
      s = (slabs + per - 1) / per;  // (none empty)
      if (s > 1024 && s > fewest) continue;
      const double cost = (double)((tiles * s + kSMs - 1) / kSMs) * (per * (1.6 * bn + 100) + 4000) + (double)s * m * n * 8 / 3500;
      if (cost < least) least = cost, best = (int)s;
    }
  }
  return best;
}

int tc_bias_parts(int m, int n, int k, int parts) {
  const int splits = tc_splits(m, n, k, parts), bn = tile_columns(m, n, splits, false);
  return splits * ((n + bn - 1) / bn);
}

int launch_tc(int kernel_id, Mode mode, const Operand &a, const Operand &b, int m, int n, int k, const Epilogue &e, int32_t *status,
              cudaStream_t st) {
  const bool partial = mode == kPartial;
  const bool plain = !tma_takes(a.p, a.ld) || !tma_takes(b.p, b.ld);
  const int bn = tile_columns(m, n, partial ? e.splits : 1, !partial && !plain && k <= 4 * kK);
  Params p = {};
  p.m = m, p.n = n, p.k = k, p.mt = parts_of(m, kM), p.nt = (n + bn - 1) / bn;
  p.items = p.mt * p.nt * (partial ? e.splits : 1);
  p.a_along = a.along, p.b_along = b.along;
  p.slabs = parts_of(k, kK);
  p.slabs_per_split = parts_of(p.slabs, e.splits);
  p.parts = a.low ? 2 : 1, p.a_low = static_cast<const __nv_bfloat16 *>(a.low);
  p.a = static_cast<const __nv_bfloat16 *>(a.p), p.b = static_cast<const __nv_bfloat16 *>(b.p), p.lda = a.ld, p.ldb = b.ld;
  p.nb = b.there ? b.there : n;
  const int wa = width_of(a.p, a.ld, a.along ? k : m), wb = width_of(b.p, b.ld, b.along ? k : p.nb);
  p.w = wa < wb ? wa : wb;
  p.slope = mode == kSlope, p.act = e.act;
  p.bias = static_cast<const __nv_bfloat16 *>(e.bias), p.extra = static_cast<const __nv_bfloat16 *>(e.extra);
  p.ld_extra = e.ld_extra, p.ld_out = e.ld_out, p.out = static_cast<__nv_bfloat16 *>(e.out), p.out_low = static_cast<__nv_bfloat16 *>(e.out_low);
  p.part = e.part, p.part_bias = e.part_bias, p.status = status, p.clear = e.first;
  rows::Alignment al;
  al.rows_at(e.extra, e.ld_extra, 2);
  al.rows_at(e.out, e.ld_out, 2);
  p.wo = al.elements(n, 2);
  CUtensorMap ta = {}, ta_low = {}, tb = {};
  if (!plain) {
    if (!make_map(&ta, a.p, a.along ? m : k, a.along ? k : m, a.ld, a.along ? kM : kK)) return BLOSSOM_ERR_CUDA;
    if (a.low && !make_map(&ta_low, a.low, a.along ? m : k, a.along ? k : m, a.ld, a.along ? kM : kK)) return BLOSSOM_ERR_CUDA;
    if (!make_map(&tb, b.p, b.along ? p.nb : k, b.along ? k : p.nb, b.ld, b.along ? bn : kK)) return BLOSSOM_ERR_CUDA;
  }
  auto go = [&](auto width) {
    constexpr int BN = decltype(width)::value;
    if (partial) return plain ? launch_one<BN, true, true>(kernel_id, ta, ta_low, tb, p, st) : launch_one<BN, true, false>(kernel_id, ta, ta_low, tb, p, st);
    return plain ? launch_one<BN, false, true>(kernel_id, ta, ta_low, tb, p, st) : launch_one<BN, false, false>(kernel_id, ta, ta_low, tb, p, st);
  };
  using std::integral_constant;
  return bn == 64 ? go(integral_constant<int, 64>()) : bn == 128 ? go(integral_constant<int, 128>())
         : bn == 192 ? go(integral_constant<int, 192>()) : go(integral_constant<int, 256>());
}

}  // namespace linear
}  // namespace blossom
