// A linear layer with bias, activation and residual, forward and backward: checks, workspace and the choice of kernels.
#include "linear.cuh"

namespace blossom {
namespace linear {
namespace {

constexpr int kMaxPackedCols = 8192;

struct Args {
  int rows, cols, outs, dtype, act, packed;
  size_t esz;
  int64_t sx, sw, sr, so, sdx, sdw;
};

int check(const blossom_linear_params *p, Args *a) {
  if (!p || p->rows < 0 || p->cols < 1 || p->outs < 1) return BLOSSOM_ERR_INVALID_ARG;
  if (p->dtype != BLOSSOM_DTYPE_FP32 && p->dtype != BLOSSOM_DTYPE_BF16) return BLOSSOM_ERR_INVALID_ARG;
  if (p->activation < BLOSSOM_ACT_NONE || p->activation > BLOSSOM_ACT_SILU || p->packed < 0 || p->packed > 1)
    return BLOSSOM_ERR_INVALID_ARG;
  auto stride = [](int64_t s, int width) { return s == 0 ? (int64_t)width : s; };
  a->sx = stride(p->x_stride, p->cols), a->sw = stride(p->weight_stride, p->cols), a->sr = stride(p->residual_stride, p->outs);
  a->so = stride(p->out_stride, p->outs), a->sdx = stride(p->dx_stride, p->cols), a->sdw = stride(p->dweight_stride, p->cols);
  for (int64_t s : {a->sx, a->sw, a->sdx, a->sdw})
    if (s < p->cols) return BLOSSOM_ERR_INVALID_ARG;
  for (int64_t s : {a->sr, a->so})
    if (s < p->outs) return BLOSSOM_ERR_INVALID_ARG;
  if (p->packed && a->sx != p->cols) return BLOSSOM_ERR_INVALID_ARG;
  if (p->rows > 0x7fffffffLL || p->cols > kMaxWidth || p->outs > kMaxWidth || (p->packed && p->cols > kMaxPackedCols))
    return BLOSSOM_ERR_UNSUPPORTED;
  a->rows = (int)p->rows, a->cols = p->cols, a->outs = p->outs, a->dtype = p->dtype, a->act = p->activation, a->packed = p->packed;
  a->esz = p->dtype == BLOSSOM_DTYPE_FP32 ? 4 : 2;
  return BLOSSOM_OK;
}

// Device scratch of a backward; the forward uses the status words alone.
struct Scratch {
  int32_t *status;
  void *g, *g_low;  // [rows][ld_g] the upstream gradient times the activation's slope, and what its rounding to bf16 leaves
  void *x;  // [rows][ld_x] x from its 8 bits
  int64_t ld_g, ld_x;
  float *part, *part_bias;  // [splits][outs][cols], [bias_parts][outs]
  int splits, bias_parts;
  int narrow;  // splits of the kernel for narrow layers
  int dx_splits;
  size_t bytes;
};
// Between the products G is bf16.  Rounded to one its error is as large as the results' own rounding (together 1.4 times that), so
// what the rounding leaves goes through the products as a second part of G, which makes that of dx and dweight twice the work:
// forward and backward of 32768 x 1024 -> 4096 1145 us without, 1721 with it, of 8192 x 1024 -> 1024 128 and 165.
int parts(const Args &a) { return a.act && a.esz == 2 ? 2 : 1; }
// Few rows go to kernels of their own rather than to tiles of 128 rows that are mostly empty.  Forward, us against tiles: single
// precision 1, 16 rows of 1024 -> 4096 4.8, 19.4 against 23; bf16 1, 4, 8, 16 rows 4.1, 4.9, 8.8, 14.5 against 8.  Forward and
// backward with GELU, 16 rows: 1024 -> 4096 single 62 against 98, bf16 53 against 61; 64 -> 256 single 23 against 31, but bf16 24
// against 21 (4 rows 15), where the narrow layers' kernel is.
bool few_forward(const Args &a) { return a.rows <= (a.esz == 4 ? kFewRows : 4); }
bool few_backward(const Args &a) { return a.rows <= 4 || (a.rows <= kFewRows && (a.esz == 4 || a.cols > 256 || a.outs > 256)); }
// Rows that the kernel for narrow layers takes at a time, as many as its accumulators may add up; those from `row` on.
int64_t narrow_rows(const Args &a) { return (int64_t)kSMs * kMostSlabs * 64 / parts(a); }
int narrow_rows(const Args &a, int64_t row) { return (int)(a.rows - row < narrow_rows(a) ? a.rows - row : narrow_rows(a)); }
NarrowBackward from_row(const Args &a, const NarrowBackward &n, int64_t row) {
  NarrowBackward m = n;
  m.rows = narrow_rows(a, row);
  auto on = [&](const void *p, int64_t bytes) { return p ? static_cast<const char *>(p) + row * bytes : nullptr; };
  m.x = on(n.x, n.ld_x * 2), m.dout = on(n.dout, n.ld_dout * 2);
  m.dx = const_cast<char *>(on(n.dx, n.ld_dx * 2));
  m.codes = reinterpret_cast<const int8_t *>(on(n.codes, n.cols));
  m.scales = reinterpret_cast<const uint8_t *>(on(n.scales, (n.cols + 31) / 32));
  return m;
}
int64_t align8(int64_t n) { return (n + 7) / 8 * 8; }

// What becomes of a backward whose tensors lie where these do: one kernel, for narrow layers, and from x as it is or its codes.
struct Way {
  bool one_kernel, x_as_it_is;
};
NarrowBackward narrow_of(const Args &a, const void *x, const uint8_t *scales, const void *weight, const void *dout) {
  NarrowBackward n = {};
  n.rows = a.rows, n.cols = a.cols, n.outs = a.outs, n.act = a.act;
  n.weight = weight, n.ld_weight = a.sw, n.dout = dout, n.ld_dout = a.so, n.ld_dx = a.sdx;
  if (a.packed) n.codes = static_cast<const int8_t *>(x), n.scales = scales;
  else n.x = x, n.ld_x = a.sx;
  return n;
}
Way way_of(const Args &a, const void *x, const void *weight, const void *dout) {
  Way w = {};
  if (few_backward(a) || a.esz != 2 || a.rows == 0) return w;
  w.x_as_it_is = narrow_takes(narrow_of(a, x, nullptr, weight, dout));
  // (codes can be turned into rows first)
  w.one_kernel = w.x_as_it_is || (a.packed && narrow_takes(narrow_of(a, nullptr, nullptr, weight, dout)));
  return w;
}

Scratch carve(const Args &a, const Way &way, void *base) {
  Scratch s;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char *r = base ? static_cast<char *>(base) + off : nullptr;
    off += (bytes + 255) / 256 * 256;
    return r;
  };
  s.status = reinterpret_cast<int32_t *>(take(BLOSSOM_LINEAR_FORWARD_BYTES));
  s.ld_g = align8(a.outs), s.ld_x = align8(a.cols);
  if (few_backward(a)) {
    s.g = take(a.act ? (size_t)a.rows * s.ld_g * sizeof(float) : 0);
    s.g_low = nullptr;
    s.x = take(a.packed ? (size_t)a.rows * s.ld_x * a.esz : 0);
    s.splits = s.bias_parts = s.narrow = s.dx_splits = 0;
    s.part = reinterpret_cast<float *>(take((size_t)few_shares(a.cols, a.outs) * a.rows * a.cols * sizeof(float)));
    s.part_bias = nullptr;
    s.bytes = off;
    return s;
  }
  s.x = take(a.packed && !way.x_as_it_is ? (size_t)a.rows * s.ld_x * a.esz : 0);
  s.g = s.g_low = nullptr, s.splits = s.bias_parts = s.narrow = 0, s.dx_splits = 1;
  if (way.one_kernel) {
    for (int64_t r = 0; r < a.rows; r += narrow_rows(a)) s.narrow += narrow_splits(narrow_rows(a, r));
    s.part = reinterpret_cast<float *>(take((size_t)s.narrow * a.outs * a.cols * sizeof(float)));
    s.part_bias = reinterpret_cast<float *>(take((size_t)s.narrow * a.outs * sizeof(float)));
    s.bytes = off;
    return s;
  }
  s.g = take(a.act ? (size_t)a.rows * s.ld_g * a.esz : 0);
  s.g_low = parts(a) == 2 ? take((size_t)a.rows * s.ld_g * a.esz) : nullptr;
  if (a.esz == 2) {
    s.splits = tc_splits(a.outs, a.cols, a.rows ? a.rows : 1, parts(a));
    s.bias_parts = tc_bias_parts(a.outs, a.cols, a.rows ? a.rows : 1, parts(a));
  } else {
    s.splits = s.bias_parts = f32_splits(a.outs, a.cols, a.rows ? a.rows : 1);
  }
  // dx of few tiles (all of a row's columns in one) over many outs leaves SMs idle: its sums are split as well (forward and backward in
  // single precision, us with splits and with a cluster a tile: 64 x 64 -> 1000 17.8, 23.0, 600 x 64 -> 1000 24.6, 31.5, but
  // 200 x 1000 -> 1000 37.8, 33.9).  So is dx over more than the forward's most
  // steps in one accumulator.
  const bool few_tiles = (int64_t)parts_of(a.rows, 128) * parts_of(a.cols, 128) < kSMs && a.outs >= 256,
             long_sums = a.esz == 2 && a.outs * parts(a) > kMaxWidth;
  if ((few_tiles || long_sums) && a.rows)
    s.dx_splits = a.esz == 2 ? tc_splits(a.rows, a.cols, a.outs, parts(a)) : f32_splits(a.rows, a.cols, a.outs);
  // (one split's sums go where they belong)
  const size_t weight = s.splits > 1 ? (size_t)s.splits * a.outs * a.cols : 0, dx = s.dx_splits > 1 ? (size_t)s.dx_splits * a.rows * a.cols : 0;
  s.part = reinterpret_cast<float *>(take((weight > dx ? weight : dx) * sizeof(float)));
  s.part_bias = reinterpret_cast<float *>(take((size_t)s.bias_parts * a.outs * sizeof(float)));
  s.bytes = off;
  return s;
}

int launch_product(int kernel_id, Mode mode, const Args &a, const Operand &x, const Operand &y, int m, int n, int k,
                   const Epilogue &e, int32_t *status, cudaStream_t st) {
  if (a.esz == 2) return launch_tc(kernel_id, mode, x, y, m, n, k, e, status, st);
  return launch_f32(kernel_id, mode, x, y, m, n, k, e, status, st);
}

bool misaligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }
int check_workspace(const void *p, size_t bytes, size_t need) {
  return !p || misaligned(p, 256) || bytes < need ? BLOSSOM_ERR_WORKSPACE : BLOSSOM_OK;
}

}  // namespace
}  // namespace linear
}  // namespace blossom

extern "C" size_t blossom_linear_workspace_bytes(const blossom_linear_params *params) {
  using namespace blossom;
  linear::Args a;
  if (linear::check(params, &a)) return 0;
  // one kernel's partial sums may be more than what products after one another need
  const linear::Way one = linear::way_of(a, nullptr, nullptr, nullptr);
  const size_t any = linear::carve(a, {}, nullptr).bytes, single = one.one_kernel ? linear::carve(a, {true, false}, nullptr).bytes : 0;
  return any > single ? any : single;
}

extern "C" size_t blossom_linear_bwd_workspace_bytes(const blossom_linear_params *params, const void *x, const void *weight,
                                                     const void *dout) {
  using namespace blossom;
  linear::Args a;
  return linear::check(params, &a) ? 0 : linear::carve(a, linear::way_of(a, x, weight, dout), nullptr).bytes;
}

extern "C" int blossom_linear_fwd(const blossom_linear_params *params, const void *x, const void *weight, const void *bias,
                                  const void *residual, void *out, void *workspace, size_t workspace_bytes,
                                  blossom_stream_t stream) {
  using namespace blossom;
  prof_break();
  linear::Args a;
  if (int rc = linear::check(params, &a)) return rc;
  if (!weight || (a.rows && (!x || !out))) return BLOSSOM_ERR_INVALID_ARG;
  for (const void *p : {x, weight, bias, residual, (const void *)out})
    if (linear::misaligned(p, a.esz)) return BLOSSOM_ERR_INVALID_ARG;
  if (int rc = linear::check_workspace(workspace, workspace_bytes, BLOSSOM_LINEAR_FORWARD_BYTES)) return rc;
  const cudaStream_t st = (cudaStream_t)stream;
  // (the kernel clears the words itself)
  if (a.rows == 0 && cudaMemsetAsync(workspace, 0, 32, st) != cudaSuccess) return BLOSSOM_ERR_CUDA;
  if (a.rows == 0) return BLOSSOM_OK;
  if (linear::few_forward(a))
    return linear::launch_few_forward({a.dtype, a.rows, a.cols, a.outs, a.act, x, weight, bias, a.sx, a.sw}, false, residual, a.sr, out,
                                      a.so, static_cast<int32_t *>(workspace), st);
  linear::Epilogue e;
  e.act = a.act, e.bias = bias, e.extra = residual, e.ld_extra = a.sr, e.out = out, e.ld_out = a.so;
  return linear::launch_product(K_LINEAR_FWD, linear::kForward, a, {x, a.sx, true}, {weight, a.sw, true}, a.rows, a.outs, a.cols, e,
                                static_cast<int32_t *>(workspace), st);
}

extern "C" int blossom_linear_bwd(const blossom_linear_params *params, const void *x, const uint8_t *x_scales, const void *weight,
                                  const void *bias, const void *dout, void *dx, void *dweight, void *dbias, void *workspace,
                                  size_t workspace_bytes, blossom_stream_t stream) {
  using namespace blossom;
  prof_break();
  linear::Args a;
  if (int rc = linear::check(params, &a)) return rc;
  const bool reads_x = a.act || dweight;
  if (!weight || !(dx || dweight || dbias) || (a.rows && (!dout || (reads_x && (!x || (a.packed && !x_scales))))))
    return BLOSSOM_ERR_INVALID_ARG;
  for (const void *p : {weight, bias, dout, (const void *)dx, (const void *)dweight, (const void *)dbias})
    if (linear::misaligned(p, a.esz)) return BLOSSOM_ERR_INVALID_ARG;
  if (!a.packed && linear::misaligned(x, a.esz)) return BLOSSOM_ERR_INVALID_ARG;
  const linear::Way way = linear::way_of(a, reads_x ? x : nullptr, weight, dout);
  const linear::Scratch s = linear::carve(a, way, workspace);
  if (int rc = linear::check_workspace(workspace, workspace_bytes, s.bytes)) return rc;
  const cudaStream_t st = (cudaStream_t)stream;
  if (a.rows == 0) {  // sums over no rows
    if (cudaMemsetAsync(workspace, 0, 32, st) != cudaSuccess) return BLOSSOM_ERR_CUDA;
    return dweight || dbias ? linear::launch_join(a.dtype, s.part, s.part_bias, 0, 0, a.outs, a.cols, dweight, a.sdw, dbias, st) : BLOSSOM_OK;
  }
  linear::Operand xo = {x, a.sx, true}, g = {dout, a.so, true};
  if (a.packed && reads_x && !way.x_as_it_is) {
    blossom_rows_params p = {};
    p.rows = a.rows, p.cols = a.cols, p.dtype = p.weight_dtype = a.dtype, p.out_stride = s.ld_x;
    if (int rc = blossom_unpack_rows(&p, static_cast<const int8_t *>(x), x_scales, s.x, stream)) return rc;
    xo = {s.x, s.ld_x, true};
  }
  // (the first kernel clears the status words: a call for that alone would stand between two kernels that follow closely)
  if (linear::few_backward(a)) {
    const linear::FewRows f = {a.dtype, a.rows, a.cols, a.outs, a.act, xo.p, weight, bias, xo.ld, a.sw};
    if (a.act)
      if (int rc = linear::launch_few_forward(f, true, dout, a.so, s.g, s.ld_g, s.status, st)) return rc;
    return linear::launch_few_backward(f, a.act ? s.g : dout, a.act ? s.ld_g : a.so, a.act != 0, s.part, dx, a.sdx, dweight, a.sdw, dbias,
                                       a.act ? nullptr : s.status, st);
  }
  if (way.one_kernel) {
    linear::NarrowBackward n = linear::narrow_of(a, reads_x ? x : nullptr, x_scales, weight, dout);
    if (!way.x_as_it_is) n.codes = nullptr, n.scales = nullptr, n.x = xo.p, n.ld_x = xo.ld;
    n.bias = bias, n.dx = dx, n.part = dweight ? s.part : nullptr, n.part_bias = dbias ? s.part_bias : nullptr, n.status = s.status;
    for (int64_t r = 0; r < a.rows; r += linear::narrow_rows(a)) {
      linear::NarrowBackward m = linear::from_row(a, n, r);
      if (int rc = linear::launch_narrow(m, st)) return rc;
      const int64_t splits = linear::narrow_splits(m.rows);
      if (n.part) n.part += splits * a.outs * a.cols;
      if (n.part_bias) n.part_bias += splits * a.outs;
      n.later = true;
    }
    if (!dweight && !dbias) return BLOSSOM_OK;
    return linear::launch_join(a.dtype, s.part, s.part_bias, s.narrow, s.narrow, a.outs, a.cols, dweight, a.sdw, dbias, st, linear::narrow_turned(n));
  }
  if (a.act) {
    linear::Epilogue e;
    e.act = a.act, e.bias = bias, e.extra = dout, e.ld_extra = a.so, e.out = s.g, e.out_low = s.g_low, e.ld_out = s.ld_g;
    if (int rc = linear::launch_product(K_LINEAR_SLOPE, linear::kSlope, a, xo, {weight, a.sw, true}, a.rows, a.outs, a.cols, e, s.status, st))
      return rc;
    g = {s.g, s.ld_g, true, 0, s.g_low};
  }
  if (dx) {
    linear::Epilogue e;
    e.first = !a.act;
    if (s.dx_splits > 1) {
      e.part = s.part, e.splits = s.dx_splits;
      if (int rc = linear::launch_product(K_LINEAR_DX, linear::kPartial, a, g, {weight, a.sw, false}, a.rows, a.cols, a.outs, e, s.status, st))
        return rc;
      if (int rc = linear::launch_join(a.dtype, s.part, nullptr, s.dx_splits, 0, a.rows, a.cols, dx, a.sdx, nullptr, st)) return rc;
    } else {
      e.out = dx, e.ld_out = a.sdx;
      if (int rc = linear::launch_product(K_LINEAR_DX, linear::kPlain, a, g, {weight, a.sw, false}, a.rows, a.cols, a.outs, e, s.status, st))
        return rc;
    }
  }
  if (dweight || dbias) {
    linear::Epilogue e;
    e.first = !a.act && !dx;
    e.part = dweight ? s.part : nullptr, e.part_bias = dbias ? s.part_bias : nullptr, e.splits = s.splits;
    // one split's sums are the results (32768 x 1024 -> 4096 with GELU as one: 1106 us; by way of single precision 1132)
    const bool direct = s.splits == 1 && dweight;
    if (direct) e.out = dweight, e.ld_out = a.sdw;
    const bool direct_bias = s.bias_parts == 1 && dbias && a.esz == 4;
    if (direct_bias) e.part_bias = static_cast<float *>(dbias);
    // dbias alone: x is not read; a product of the same shape is formed with G in the place of x
    linear::Operand right = {xo.p, xo.ld, false};
    if (!dweight) right = {g.p, g.ld, false, a.outs < a.cols ? a.outs : a.cols};
    if (int rc = linear::launch_product(K_LINEAR_DWEIGHT, linear::kPartial, a, {g.p, g.ld, false, 0, g.low}, right, a.outs, a.cols,
                                        a.rows, e, s.status, st))
      return rc;
    if (direct) dweight = nullptr;
    if (direct_bias) dbias = nullptr;
    if (!dweight && !dbias) return BLOSSOM_OK;
    return linear::launch_join(a.dtype, s.part, s.part_bias, s.splits, s.bias_parts, a.outs, a.cols, dweight, a.sdw, dbias, st);
  }
  return BLOSSOM_OK;
}
