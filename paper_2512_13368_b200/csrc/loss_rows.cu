// Sampled softmax loss, the part over positions: logits of a position's candidates, their log-sum-exp, the loss, and with
// it the gradient of the position's hidden row, sum_j p_j table[c_j] - table[c_target]; nothing is stored per candidate.
//
// A warp takes a position.  Groups of LPC lanes hold one candidate's row each; a group keeps a running maximum, sum and
// weighted sum of rows, and the groups are joined at the end.  Every candidate's row is read once.
// Bound: 131072 positions of 128 candidates of 64 bf16 columns take 2.1 GB from L2 and 0.17 GB from HBM (26 us) in 250 us, 8.6
// TB/s; L2 is at 41 % of its rate, the issue slots are 64 % busy: unpacking, weighing (two FMAs an instruction) and the
// ids.  32768 x 128 x 128: 117 us, 9.2 TB/s.  fp32, 12795 x 100 x 50: 45 us.  64 x 101, no gradient: 4 us of a block's latency.
#include <float.h>

#include "loss.cuh"

namespace blossom {
namespace loss {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ void write_mean(double2 s, float *loss, float *count) {
  *loss = s.y > 0.0 ? (float)(s.x / s.y) : 0.f;
  *count = (float)s.y;
}
// A CTA's sum from its warps': to scratch for a second kernel, or, if it is the only one, the mean.  (A cluster that adds its
// CTAs' sums in place of the second kernel lost: 64 rows of 101 candidates 8.4 -> 10.6 us on 8 CTAs.)
template <int THREADS>
__device__ __forceinline__ void close_sums(double2 mine, double2 *sums, float *loss, float *count) {
  __shared__ double2 warp_sums[THREADS / 32];
  if (threadIdx.x % 32 == 0) warp_sums[threadIdx.x / 32] = mine;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < THREADS / 32; ++i) mine.x += warp_sums[i].x, mine.y += warp_sums[i].y;
    if (gridDim.x == 1) write_mean(mine, loss, count);
    else sums[blockIdx.x] = mine;
  }
}

// Few positions with many candidates: a block takes a position, its warps every NW-th 32 candidates, joined in shared memory.
// (Against a warp a position: 592 x 101 8.6 us to 10.7, 1184 x 501 15 to 23; in fp32 1184 x 101 13 to 15, but 2368 x 101 21 to
// 15; 33 candidates alike.)
template <int NW>
struct Shares {  // of a block's warps
  float high[NW], total[NW];
  // the common reference point, and the sum in its units
  __device__ __forceinline__ void join(float &top, float &sum) const {
    top = high[0];
#pragma unroll
    for (int i = 1; i < NW; ++i) top = fmaxf(top, high[i]);
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) sum += total[i] * exp2f(high[i] - top);  // (0 from a warp that met no candidate)
  }
};

template <typename T, int W, typename P, bool GRAD>
__global__ void __launch_bounds__(kThreads, P::V == 1 ? 4 : P::V == 2 ? 2 : 1)
    loss_rows_kernel(Args a, int split, const T *__restrict__ hidden, const T *__restrict__ table, float *__restrict__ lse,
                     float *__restrict__ dh, double2 *__restrict__ sums, float *__restrict__ loss) {
  using S = Strip<T, W, P>;
  constexpr int LPC = P::LPC, V = P::V, CPW = 32 / LPC, U = V == 1 ? 2 : 1, NW = kThreads / 32;
  __shared__ Shares<NW> shares;
  __shared__ float shared_sums[GRAD ? NW : 1][V * 8][LPC];
  grid_chain_enter();
  const int lane = (int)threadIdx.x % 32, warp = (int)threadIdx.x / 32, col = lane % LPC, sub = lane / LPC;
  double2 mine = make_double2(0.0, 0.0);
  const int64_t step = split ? gridDim.x : (int64_t)gridDim.x * NW;
  const int c_first = split ? 32 * warp : 0, c_step = split ? 32 * NW : 32;
  for (int64_t r = split ? blockIdx.x : (int64_t)blockIdx.x * NW + warp; r < a.rows; r += step) {
    const int row = (int)r, target = row_target(a, row);
    // of the candidates c0 .. c0 + 31, one a lane; -1: none
    int id = c_first + lane <= a.n ? candidate(a, row, target, c_first + lane) : -1;
    Group acc[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[v].p[i] = both(0.f);
    float row_lse = 0.f;
    if (target >= 0) {
      Group h[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        h[v] = S::load(hidden + row * a.sh, col, v, a.cols);
#pragma unroll
        for (int i = 0; i < 4; ++i) h[v].p[i] = mul2(h[v].p[i], both(kLog2e));  // logits in units of log 2
      }
      float top = -FLT_MAX, total = 0.f, own = 0.f;
      for (int c0 = c_first; c0 <= a.n; c0 += c_step) {
        int64_t next = -1;  // (not looked at before it is wanted: whoever looks waits)
        if (c0 + c_step + lane <= a.n) next = load_negative(a, row, c0 + c_step + lane);
        const int steps = (min(32, a.n + 1 - c0) + CPW - 1) / CPW;
        for (int k = 0; k < steps; k += U) {
          Group w[U][V];
          float l[U];
          int at[U];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            at[u] = __shfl_sync(0xffffffffu, id, (k + u) * CPW + sub);
#pragma unroll
            for (int v = 0; v < V; ++v) w[u][v] = S::load(table + at[u] * a.st, col, v, a.cols, at[u] >= 0);
          }
          float high = top;
          bool any = false;
#pragma unroll
          for (int u = 0; u < U; ++u) {
            any |= at[u] >= 0;
            l[u] = dot<V>(h, w[u]);
#pragma unroll
            for (int o = 1; o < LPC; o <<= 1) l[u] += __shfl_xor_sync(0xffffffffu, l[u], o);
            if (at[u] < 0) l[u] = -INFINITY;
            high = fmaxf(high, l[u]);
          }
          if (c0 == 0 && k == 0) own = __shfl_sync(0xffffffffu, l[0], 0);
          if (any) {  // (logits that are no numbers go in as well and make the row's sum one)
            const float shrink = exp2f(top - high);
            total *= shrink;
            if (GRAD) {
#pragma unroll
              for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[v].p[i] = mul2(acc[v].p[i], both(shrink));
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
              const float p = exp2f(l[u] - high);
              total += p;
              if (GRAD) {
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                  for (int i = 0; i < 4; ++i) acc[v].p[i] = fma2(both(p), w[u][v].p[i], acc[v].p[i]);
              }
            }
            top = high;
          }
        }
        id = valid_negative(a, target, next);
      }
      // the groups of lanes, joined (one that has met no candidate weighs nothing)
      float high = top;
#pragma unroll
      for (int o = LPC; o < 32; o <<= 1) high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, o));
      const float weight = exp2f(top - high);
      total *= weight;
#pragma unroll
      for (int o = LPC; o < 32; o <<= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
      if (GRAD) {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            float &x = acc[v].at(i);
            x *= weight;
#pragma unroll
            for (int o = LPC; o < 32; o <<= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
          }
      }
      if (split) {
        if (lane == 0) shares.high[warp] = high, shares.total[warp] = total;
        if (GRAD && sub == 0) {
#pragma unroll
          for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) shared_sums[warp][8 * v + i][col] = acc[v].at(i);
        }
        __syncthreads();
        if (warp == 0) {
          shares.join(high, total);
          if (GRAD) {
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                float x = 0.f;
#pragma unroll
                for (int w = 0; w < NW; ++w) x += shared_sums[w][8 * v + i][col] * exp2f(shares.high[w] - high);
                acc[v].at(i) = x;
              }
          }
        }
        __syncthreads();  // (the next row's shares may come)
      }
      const float lse2 = high + log2f(total);
      row_lse = lse2 * kLn2;
      if (!split || warp == 0) {
        mine.x += (double)((lse2 - own) * kLn2);
        mine.y += 1.0;
      }
      if (GRAD) {
        const float inv = 1.f / total;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const Group w = S::load(table + target * a.st, col, v, a.cols);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            acc[v].p[i] = fma2(acc[v].p[i], both(inv), make_float2(-w.p[i].x, -w.p[i].y));
        }
      }
    }
    if (split && warp > 0) continue;
    if (lane == 0) lse[row] = row_lse;
    if (GRAD && sub == 0) {
#pragma unroll
      for (int v = 0; v < V; ++v) store_sums<W, P>(dh + (int64_t)row * a.cols, col, v, a.cols, acc[v]);
    }
  }
  close_sums<kThreads>(mine, sums, loss, lse + a.rows);
}

// The same on the matrix units: a warp scores 16 candidates at a time.  What is no candidate is read as the target's row and
// weighs nothing.  Other warps work while a warp's 16 rows are under way: two buffers of rows a warp in 80 registers were slower
// (324 us against 305, 131072 x 128 candidates x 64).  4 lanes a row of 64 columns need neither shuffles nor each exponential
// eight times (252 us against 270 with 8; 51200 x 32 candidates 41 against 39); for 128 columns they take too many registers.
// The weighted sum stays on the CUDA cores: as a second product, its operand transposed in registers, it took 377 us.
// Blocks an SM: 8 and 5 (7 259 us, 9 283; with 128 columns 4 127 us, 6 125, 5 117); the grid is two rounds of them.
constexpr int row_blocks(int lines) { return lines == 1 ? 8 : 5; }  // an SM
template <int NL, bool FULL, bool GRAD>
__global__ void __launch_bounds__(kMmaThreads, row_blocks(NL))
    loss_rows_mma_kernel(Args a, int split, const __nv_bfloat16 *__restrict__ hidden, const __nv_bfloat16 *__restrict__ table,
                         float *__restrict__ lse, float *__restrict__ dh, double2 *__restrict__ sums,
                         float *__restrict__ loss) {
  constexpr int L = 4 * NL;  // lanes a row
  using R = Rows16<NL, L>;
  constexpr int NW = kMmaThreads / 32;
  __shared__ Shares<NW> shares;
  __shared__ float2 shared_sums[NW][NL][32];
  grid_chain_enter();
  const int lane = (int)threadIdx.x % 32, warp = (int)threadIdx.x / 32, group = lane / R::kLanes;
  const Lanes16<NL, L, FULL> from_hidden(hidden, a.sh, a.cols), from_table(table, a.st, a.cols);
  double2 mine = make_double2(0.0, 0.0);
  const int64_t step = split ? gridDim.x : (int64_t)gridDim.x * NW;
  const int c_first = split ? 32 * warp : 0, c_step = split ? 32 * NW : 32;
  for (int64_t r = split ? blockIdx.x : (int64_t)blockIdx.x * NW + warp; r < a.rows; r += step) {
    const int row = (int)r, target = row_target(a, row);
    // of the candidates c0 .. c0 + 31, one a lane; -1: none
    int id = c_first + lane <= a.n ? candidate(a, row, target, c_first + lane) : -1;
    float row_lse = 0.f;
    float2 grad[NL];
#pragma unroll
    for (int c = 0; c < NL; ++c) grad[c] = make_float2(0.f, 0.f);
    if (target >= 0) {
      uint2 h[R::kParts];
      from_hidden.vector((uint32_t)row, a.cols, h);
      float2 acc[R::kParts][4];
#pragma unroll
      for (int e = 0; e < R::kParts; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[e][i] = make_float2(0.f, 0.f);
      auto rows_of = [&](int id, uint32_t &there) {  // there: a bit for each candidate
        there = __ballot_sync(0xffffffffu, id >= 0);
        return (uint32_t)(id >= 0 ? id : target);
      };
      // of a group of lanes: its rows of every 16; logits as they come (top: half the lowest number, so that log2(e) times
      // it is one)
      float top = -0.5f * FLT_MAX, total = 0.f, own = 0.f;
      auto score = [&](const R &w, uint32_t there) {
        float l[R::kRows];
        dots16<NL, L>(w, h, l);
        const float first = l[0];
        if (~there & 0xffffu) {  // (the same for the warp)
          there >>= group;
#pragma unroll
          for (int j = 0; j < R::kRows; ++j)
            if (!(there >> (R::kStep * j) & 1)) l[j] = -INFINITY;
        }
        // The reference point only moves if it has to, by more than 2^10 in the exponentials: the sums stay far from the type's
        // limits, and their relative rounding does not depend on it.
        float high = l[0];
#pragma unroll
        for (int j = 1; j < R::kRows; ++j) high = fmaxf(high, l[j]);
        if (high > top + 7.f) {
          const float shrink = exp2f((top - high) * kLog2e);
          total *= shrink;
          if (GRAD) {
#pragma unroll
            for (int e = 0; e < R::kParts; ++e)
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[e][i].x *= shrink, acc[e][i].y *= shrink;
          }
          top = high;
        }
        const float shift = -top * kLog2e;
#pragma unroll
        for (int j = 0; j < R::kRows; ++j) l[j] = exp2f(fmaf(l[j], kLog2e, shift));
#pragma unroll
        for (int j = 0; j < R::kRows; ++j) total += l[j];
        if (GRAD) weigh16<NL, L>(w, l, acc);
        return first;
      };
      R w;
      for (int c0 = c_first; c0 <= a.n; c0 += c_step) {
        uint32_t there;
        const uint32_t ids = rows_of(id, there);
        from_table.load16(ids, 0, w);
        int64_t raw = -1;  // (the next 32 are not looked at before they are wanted: whoever looks waits)
        if (c0 + c_step + lane <= a.n) raw = load_negative(a, row, c0 + c_step + lane);
        const float l0 = score(w, there);
        if (c0 == 0) own = __shfl_sync(0xffffffffu, l0, 0) * kLog2e;
        if (c0 + 16 <= a.n) {
          from_table.load16(ids, 16, w);
          score(w, there >> 16);
        }
        id = valid_negative(a, target, raw);
      }
      top *= kLog2e;  // in units of log 2 from here on
      float high = top;
#pragma unroll
      for (int o = R::kLanes; o < 32; o <<= 1) high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, o));
      const float weight = exp2f(top - high);  // (0 for a group that met no candidate)
      total *= weight;
#pragma unroll
      for (int o = R::kLanes; o < 32; o <<= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
      if (GRAD) {
#pragma unroll
        for (int e = 0; e < R::kParts; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[e][i] = mul2(acc[e][i], both(weight));
        scatter16<NL, L>(acc, grad);
      }
      if (split) {
        if (lane == 0) shares.high[warp] = high, shares.total[warp] = total;
        if (GRAD) {
#pragma unroll
          for (int c = 0; c < NL; ++c) shared_sums[warp][c][lane] = grad[c];
        }
        __syncthreads();
        if (warp == 0) {
          shares.join(high, total);
          if (GRAD) {
#pragma unroll
            for (int c = 0; c < NL; ++c) {
              grad[c] = both(0.f);
#pragma unroll
              for (int w = 0; w < NW; ++w) grad[c] = fma2(shared_sums[w][c][lane], both(exp2f(shares.high[w] - high)), grad[c]);
            }
          }
        }
        __syncthreads();  // (the next row's shares may come)
      }
      const float lse2 = high + log2f(total);
      row_lse = lse2 * kLn2;
      if (!split || warp == 0) {
        mine.x += (double)((lse2 - own) * kLn2);
        mine.y += 1.0;
      }
      if (GRAD) {
        const float inv = 1.f / total;
#pragma unroll
        for (int c = 0; c < NL; ++c) {
          const int col = scattered_column<L>(c);
          if (FULL || col < a.cols) {
            const float2 w = rows::halves(*reinterpret_cast<const uint32_t *>(table + target * a.st + col));
            grad[c] = fma2(grad[c], both(inv), make_float2(-w.x, -w.y));
          }
        }
      }
    }
    if (split && warp > 0) continue;
    if (lane == 0) lse[row] = row_lse;
    if (GRAD) {
#pragma unroll
      for (int c = 0; c < NL; ++c) {
        const int col = scattered_column<L>(c);
        if (FULL || col < a.cols) *reinterpret_cast<float2 *>(dh + (int64_t)row * a.cols + col) = grad[c];
      }
    }
  }
  close_sums<kMmaThreads>(mine, sums, loss, lse + a.rows);
}

// The mean, from the CTAs' sums in a fixed order.  Bound: one block's latency (2 us).
__global__ void __launch_bounds__(kThreads) loss_mean_kernel(int ctas, const double2 *__restrict__ sums, float *__restrict__ loss,
                                                             float *__restrict__ count) {
  __shared__ double2 warp_sums[kThreads / 32];
  grid_chain_enter();
  double2 s = make_double2(0.0, 0.0);
  for (int i = (int)threadIdx.x; i < ctas; i += kThreads) s.x += sums[i].x, s.y += sums[i].y;
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    s.x += __shfl_xor_sync(0xffffffffu, s.x, o);
    s.y += __shfl_xor_sync(0xffffffffu, s.y, o);
  }
  if (threadIdx.x % 32 == 0) warp_sums[threadIdx.x / 32] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < kThreads / 32; ++i) s.x += warp_sums[i].x, s.y += warp_sums[i].y;
    write_mean(s, loss, count);
  }
}

int check(const blossom_loss_params *p, Args *a) {
  if (!p || p->rows < 0 || p->cols < 1 || p->items < 1 || p->negatives < 0) return BLOSSOM_ERR_INVALID_ARG;
  if (p->dtype != BLOSSOM_DTYPE_FP32 && p->dtype != BLOSSOM_DTYPE_BF16) return BLOSSOM_ERR_INVALID_ARG;
  if ((p->index_bytes != 4 && p->index_bytes != 8) || p->mask_hits < 0 || p->mask_hits > 1) return BLOSSOM_ERR_INVALID_ARG;
  int64_t st[4] = {p->hidden_stride, p->table_stride, p->dhidden_stride, p->dtable_stride};
  for (int64_t &s : st) {
    if (s == 0) s = p->cols;
    if (s < p->cols) return BLOSSOM_ERR_INVALID_ARG;
  }
  if (p->negatives_stride < 0) return BLOSSOM_ERR_INVALID_ARG;
  const int64_t most = 0x7fffffffLL;
  if (p->cols > kMaxCols || p->items >= 1 << 30 || p->negatives_stride > most || p->rows > most || p->negatives > kMaxNegatives ||
      (p->rows > 0 && p->rows > most / ((int64_t)p->negatives + 1)))
    return BLOSSOM_ERR_UNSUPPORTED;
  a->rows = (int)p->rows, a->cols = p->cols, a->groups = (p->cols + 7) / 8, a->items = p->items, a->n = p->negatives;
  a->ignore = p->ignore_index, a->sh = st[0], a->st = st[1], a->sn = (uint32_t)p->negatives_stride, a->sdh = st[2], a->sdt = st[3];
  a->idx8 = p->index_bytes == 8, a->hits = p->mask_hits;
  a->targets = a->negatives = nullptr;
  return BLOSSOM_OK;
}
// the inputs of either call
int check_inputs(Args *a, int dtype, int index_bytes, const void *hidden, const void *table, const void *targets,
                 const void *negatives) {
  if (!table || (a->rows && (!hidden || !targets || (a->n && !negatives)))) return BLOSSOM_ERR_INVALID_ARG;
  const size_t esz = dtype == BLOSSOM_DTYPE_FP32 ? 4 : 2;
  if ((reinterpret_cast<uintptr_t>(hidden) | reinterpret_cast<uintptr_t>(table)) % esz) return BLOSSOM_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(targets) | reinterpret_cast<uintptr_t>(negatives)) % (size_t)index_bytes)
    return BLOSSOM_ERR_INVALID_ARG;
  a->targets = targets;
  a->negatives = negatives;
  return BLOSSOM_OK;
}

}  // namespace
}  // namespace loss
}  // namespace blossom

extern "C" size_t blossom_sampled_loss_workspace_bytes(const blossom_loss_params *params) {
  using namespace blossom;
  loss::Args a;
  return loss::check(params, &a) ? 0 : loss::carve(a, nullptr).bytes;
}

extern "C" int blossom_sampled_loss_fwd(const blossom_loss_params *params, const void *hidden, const void *table,
                                        const void *targets, const void *negatives, float *loss_out, float *lse,
                                        float *grad_hidden, void *workspace, size_t workspace_bytes, blossom_stream_t stream) {
  using namespace blossom;
  prof_break();
  loss::Args a;
  if (int rc = loss::check(params, &a)) return rc;
  if (int rc = loss::check_inputs(&a, params->dtype, params->index_bytes, hidden, table, targets, negatives)) return rc;
  if (!loss_out || !lse || (reinterpret_cast<uintptr_t>(loss_out) | reinterpret_cast<uintptr_t>(lse)) % 4 ||
      reinterpret_cast<uintptr_t>(grad_hidden) % 16)
    return BLOSSOM_ERR_INVALID_ARG;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 || workspace_bytes < loss::kForwardBytes)
    return BLOSSOM_ERR_WORKSPACE;
  const cudaStream_t st = (cudaStream_t)stream;
  const size_t esz = params->dtype == BLOSSOM_DTYPE_FP32 ? 4 : 2;
  double2 *sums = static_cast<double2 *>(workspace);
  rows::Alignment al;
  al.rows_at(hidden, a.sh, esz);
  al.rows_at(table, a.st, esz);
  const int width = al.elements(a.cols, esz), lines = loss::mma_lines(a, params->dtype, width);
  const int warps = (lines ? loss::kMmaThreads : loss::kThreads) / 32;  // a row each
  const int64_t want = ((int64_t)a.rows + warps - 1) / warps, most = loss::kSMs * (lines ? 2 * loss::row_blocks(lines) : 64 / warps);
  // (a block a row while the rows alone do not give an SM 8 warps; measured at Shares)
  const int split = a.n >= 32 && a.rows <= loss::kSMs * 8;
  const int ctas = split ? a.rows : (int)(want < most ? want : most);
  auto launch = [&](auto kern, int threads, auto... args) {
    LaunchScope ls(K_LOSS_ROWS, st);
    launch_chained(kern, dim3((unsigned)ctas), dim3((unsigned)threads), 0, st, a, split, args..., loss_out);
  };
  if (ctas && lines) {
    loss::with_lines(lines, a.cols, [&](auto n, auto all) {
      constexpr int NL = decltype(n)::value;
      constexpr bool FULL = decltype(all)::value;
      launch(grad_hidden ? loss::loss_rows_mma_kernel<NL, FULL, true> : loss::loss_rows_mma_kernel<NL, FULL, false>,
             loss::kMmaThreads, static_cast<const __nv_bfloat16 *>(hidden), static_cast<const __nv_bfloat16 *>(table), lse,
             grad_hidden, sums);
    });
  } else if (ctas) {
    loss::with_plan(a.groups, [&](auto plan) {
      using P = decltype(plan);
      rows::with_type(params->dtype, width, [&](auto t, auto w) {
        using T = decltype(t);
        constexpr int W = decltype(w)::value;
        launch(grad_hidden ? loss::loss_rows_kernel<T, W, P, true> : loss::loss_rows_kernel<T, W, P, false>, loss::kThreads,
               static_cast<const T *>(hidden), static_cast<const T *>(table), lse, grad_hidden, sums);
      });
    });
  }
  if (ctas != 1) {
    LaunchScope ls(K_LOSS_MEAN, st);
    launch_chained(loss::loss_mean_kernel, dim3(1), dim3(loss::kThreads), 0, st, ctas, (const double2 *)sums, loss_out,
                   lse + a.rows);
  }
  return cudaGetLastError() == cudaSuccess ? BLOSSOM_OK : BLOSSOM_ERR_CUDA;
}

extern "C" int blossom_sampled_loss_bwd(const blossom_loss_params *params, const void *hidden, const void *table,
                                        const void *targets, const void *negatives, const float *lse,
                                        const float *grad_hidden, const float *grad_loss, void *dhidden, void *dtable,
                                        void *workspace, size_t workspace_bytes, blossom_stream_t stream) {
  using namespace blossom;
  prof_break();
  loss::Args a;
  if (int rc = loss::check(params, &a)) return rc;
  if (int rc = loss::check_inputs(&a, params->dtype, params->index_bytes, hidden, table, targets, negatives)) return rc;
  const size_t esz = params->dtype == BLOSSOM_DTYPE_FP32 ? 4 : 2;
  if (!lse || (reinterpret_cast<uintptr_t>(lse) | reinterpret_cast<uintptr_t>(grad_loss)) % 4 || !(dhidden || dtable) ||
      (reinterpret_cast<uintptr_t>(dhidden) | reinterpret_cast<uintptr_t>(dtable)) % esz ||
      (dhidden && a.rows && !grad_hidden) || reinterpret_cast<uintptr_t>(grad_hidden) % 16)
    return BLOSSOM_ERR_INVALID_ARG;
  const loss::Scratch s = loss::carve(a, workspace);
  if (dtable && (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 || workspace_bytes < s.bytes))
    return BLOSSOM_ERR_WORKSPACE;
  rows::Alignment al;
  al.rows_at(hidden, a.sh, esz);
  al.rows_at(table, a.st, esz);
  al.rows_at(dtable, a.sdt, esz);
  al.rows_at(dhidden, a.sdh, esz);
  return loss::launch_items(a, params->dtype, hidden, table, lse, grad_hidden, grad_loss, a.rows ? dhidden : nullptr, dtable,
                            al.elements(a.cols, esz), s, (cudaStream_t)stream);
}
