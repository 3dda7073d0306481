// Native half of autograd.py: one Python call per forward, one autograd node per backward.
//
// A call on a short batch is host time: as a Python autograd.Function around ctypes the forward
// cost 75-90 us of interpreter, marshalling and allocator time and a training step 210-240 us, on
// kernels that need a fraction of that.  Here the arguments are read with the C API of Python, the
// buffers come from PyTorch's caching allocator without the dispatcher, what only the library and the
// backward read (saved branch outputs, log-sum-exps, workspace) is one allocation, and the backward is a C++
// node of the autograd graph.  Without a gradient to compute nothing is saved at all.
//
// Plumbing only, as in autograd.py: every step of the method runs behind the C ABI (blossom.h).
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/autograd/saved_variable.h>
#include <torch/csrc/autograd/variable.h>

#include <algorithm>
#include <stdexcept>
#include <string>

#include "../../include/blossom.h"

namespace {

using at::Tensor;
using torch::autograd::Node;
using torch::autograd::SavedVariable;
using torch::autograd::variable_list;

// the tensor's elements tile its storage span without gaps or overlap, so that a buffer of numel elements laid
// out with the same strides holds every one
bool dense(const Tensor &t) {
  int64_t span = 1;
  for (int64_t i = 0; i < t.dim(); ++i) {
    if (t.stride(i) <= 0) return false;
    span += (t.size(i) - 1) * t.stride(i);
  }
  return t.numel() > 0 && span == t.numel();
}

// an uninitialised tensor with exactly t's shape and strides (empty_like does not keep those of a view that is
// not dense, and the library writes every q-shaped buffer with the strides it is given)
Tensor like(const Tensor &t) {
  if (!t.is_cuda()) return at::empty_strided(t.sizes(), t.strides(), t.options());
  return at::detail::empty_strided_cuda(t.sizes(), t.strides(), t.scalar_type(), t.device());
}
Tensor fresh(at::IntArrayRef sizes, at::ScalarType type, const at::Device &dev) {
  return at::detail::empty_cuda(sizes, type, dev, std::nullopt);
}

// src's values in `dst` (same sizes, another layout) by the library's copy of rows in 16-byte pieces.  False, and
// nothing done, for every other form: types, strides of the last dimension, views that have to be resolved, tensors
// without memory of their own, empty ones.
bool copy_rows(const Tensor &src, const Tensor &dst) {
  if (!src.is_cuda() || !src.has_storage() || src.unsafeGetTensorImpl()->is_python_dispatch() || src.dim() != 4 ||
      src.scalar_type() != dst.scalar_type() || src.device() != dst.device() || src.sizes() != dst.sizes() ||
      src.numel() == 0 || src.stride(3) != 1 || dst.stride(3) != 1 || src.is_neg() || src._is_zerotensor() ||
      src.size(0) > INT32_MAX || src.size(1) > INT32_MAX || src.size(2) > INT32_MAX || src.size(3) > 1024)
    return false;
  const int64_t e = src.element_size();
  const int64_t ss[3] = {src.stride(0) * e, src.stride(1) * e, src.stride(2) * e},
                ds[3] = {dst.stride(0) * e, dst.stride(1) * e, dst.stride(2) * e};
  return blossom_copy_rows((int32_t)src.size(0), (int32_t)src.size(1), (int32_t)src.size(2), (int32_t)(src.size(3) * e),
                           src.data_ptr(), ss, dst.data_ptr(), ds,
                           (blossom_stream_t)c10::cuda::getCurrentCUDAStream(dst.device().index()).stream()) == BLOSSOM_OK;
}
Tensor copied(const Tensor &src, const Tensor &dst) { return copy_rows(src, dst) ? dst : dst.copy_(src); }
Tensor packed(const Tensor &t) {
  if (t.is_contiguous() || !t.is_cuda() || !t.has_storage() || t.unsafeGetTensorImpl()->is_python_dispatch())
    return t.contiguous();
  const Tensor dst = at::empty(t.sizes(), t.options());
  return copy_rows(t, dst) ? dst : t.contiguous();
}

// Makes `t`, whose layout is already the one wanted, plain memory: the library reads addresses, which know nothing of a view
// that negates (wrong signs) and of a zero tensor (no memory).
void make_plain(Tensor &t) {
  if (t.defined() && (t.is_neg() || t._is_zerotensor())) t = like(t).copy_(t);
}

std::string failure(const char *where, int rc) {
  return std::string(where) + ": " + blossom_status_string(rc) + " (status " + std::to_string(rc) + ")";
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

// What the backward needs beside q, k, v, the gate and the indices: one allocation
// [out_lt | out_st | lse | workspace].
struct Scratch {
  size_t span, lse_bytes, ws_bytes;
  size_t bytes() const { return 2 * span + lse_bytes + ws_bytes; }
  void *out_lt(char *base) const { return base; }
  void *out_st(char *base) const { return base + span; }
  float *lse(char *base) const { return reinterpret_cast<float *>(base + 2 * span); }
  void *workspace(char *base) const { return base + 2 * span + lse_bytes; }
};

struct BlossomAttentionBackward : public Node {
  // (the scratch buffer, the largest of them, goes through the saved-tensor hooks like the rest: offloading and
  // checkpointing free it between the passes)
  SavedVariable q_, k_, v_, gate_, idx_, buf_;
  Tensor lens_, phi_;  // (the params hold phi's address)
  Scratch scratch_;
  blossom_params params_;
  at::ScalarType gate_type_;

  std::string name() const override { return "BlossomAttentionBackward"; }
  void release_variables() override {
    q_.reset_data();
    k_.reset_data();
    v_.reset_data();
    gate_.reset_data();
    idx_.reset_data();
    buf_.reset_data();
  }
  variable_list apply(variable_list &&grads) override {
    at::NoGradGuard no_grad;
    variable_list res(4);
    if (!grads[0].defined()) return res;
    const Tensor q = q_.unpack(), k = k_.unpack(), v = v_.unpack(), gate = gate_.unpack(), idx = idx_.unpack(),
                 buf = buf_.unpack();
    if (buf.device() != q.device() || (size_t)buf.nbytes() != scratch_.bytes() || !buf.is_contiguous())
      throw std::runtime_error("blossom_attention: a saved-tensor hook returned another tensor than it was given");
    char *const base = static_cast<char *>(buf.data_ptr());
    c10::cuda::CUDAGuard guard(q.device());
    Tensor dout = grads[0];
    if (dout.strides() != q.strides() || dout.scalar_type() != q.scalar_type())  // the library wants q's layout
      dout = copied(dout, like(q));
    make_plain(dout);
    Tensor dq = like(q), dk = like(k), dv = like(k);
    Tensor dgate = fresh(gate.sizes(), at::kFloat, q.device());
    // The workspace is this call's own and its last user was the training forward (or an earlier
    // backward, which leaves the lists alone): the tile lists of that call are still in it.
    blossom_params p = params_;
    p.reuse_tile_lists = 1;
    const int rc = blossom_attn_bwd(
        &p, q.data_ptr(), k.data_ptr(), v.data_ptr(), gate.data_ptr<float>(),
        lens_.defined() ? lens_.data_ptr<int32_t>() : nullptr, idx.data_ptr<int32_t>(), scratch_.out_lt(base),
        scratch_.out_st(base), scratch_.lse(base), dout.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
        dgate.data_ptr<float>(), scratch_.workspace(base), scratch_.ws_bytes,
        (blossom_stream_t)c10::cuda::getCurrentCUDAStream(q.device().index()).stream());
    if (rc) throw std::runtime_error(failure("blossom_attn_bwd", rc));
    res[0] = dq;
    res[1] = dk;
    res[2] = dv;
    res[3] = gate_type_ == at::kFloat ? dgate : dgate.to(gate_type_);
    return res;
  }
};

bool read_int(PyObject *o, int32_t *out) {
  long x;
  if (PyLong_Check(o)) {
    x = PyLong_AsLong(o);
  } else {  // bool, numpy integers, floats: what int() takes
    PyObject *n = PyNumber_Long(o);
    if (!n) return false;
    x = PyLong_AsLong(n);
    Py_DECREF(n);
  }
  if (x == -1 && PyErr_Occurred()) return false;
  if (x != static_cast<int32_t>(x)) {
    PyErr_Format(PyExc_OverflowError, "%ld does not fit 32 bits", x);
    return false;
  }
  *out = static_cast<int32_t>(x);
  return true;
}
bool read_float(PyObject *o, float *out) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) return false;
  *out = static_cast<float>(x);
  return true;
}

// Raises binding.BlossomError(status, where).
PyObject *raise_blossom(int rc, const char *where) {
  PyObject *mod = PyImport_ImportModule("paper_2512_13368_b200.binding");
  PyObject *cls = mod ? PyObject_GetAttrString(mod, "BlossomError") : nullptr;
  PyObject *exc = cls ? PyObject_CallFunction(cls, "is", rc, where) : nullptr;
  if (exc) PyErr_SetObject(cls, exc);
  Py_XDECREF(exc);
  Py_XDECREF(cls);
  Py_XDECREF(mod);
  return nullptr;
}

// attention(q, k, v, gate, seq_lens, phi, block, topk, window, sm_scale, stis_mode, stis_block,
//           cmp_block, cmp_stride, per_query, gate_mode, causal, rope_theta) -> (out, idx)
// None: the arguments are not what the library can be handed (autograd.check_arguments says why).
PyObject *attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 18) {
    PyErr_SetString(PyExc_TypeError, "attention() takes 18 arguments");
    return nullptr;
  }
  for (int i = 0; i < 4; ++i)
    if (!THPVariable_Check(a[i])) Py_RETURN_NONE;
  blossom_params p = {};
  if (!read_int(a[6], &p.block_size) || !read_int(a[7], &p.top_k) || !read_int(a[8], &p.window) ||
      !read_float(a[9], &p.sm_scale) || !read_int(a[10], &p.stis_mode) || !read_int(a[11], &p.stis_block) ||
      !read_int(a[12], &p.cmp_block) || !read_int(a[13], &p.cmp_stride) || !read_int(a[14], &p.select_mode) ||
      !read_int(a[15], &p.gate_mode) || !read_int(a[16], &p.causal) || !read_float(a[17], &p.rope_theta))
    return nullptr;
  try {
    const Tensor &q0 = THPVariable_Unpack(a[0]), &k0 = THPVariable_Unpack(a[1]), &v0 = THPVariable_Unpack(a[2]),
                 &gate0 = THPVariable_Unpack(a[3]);
    const at::ScalarType dt = q0.scalar_type();
    if (dt != at::kFloat && dt != at::kBFloat16) Py_RETURN_NONE;
    if (!q0.is_cuda() || q0.dim() != 4 || k0.dim() != 4 || k0.sizes() != v0.sizes() || k0.scalar_type() != dt ||
        v0.scalar_type() != dt || k0.device() != q0.device() || v0.device() != q0.device())
      Py_RETURN_NONE;
    const int64_t B = q0.size(0), H = q0.size(1), L = q0.size(2), D = q0.size(3), Hkv = k0.size(1);
    if (k0.size(0) != B || k0.size(2) != L || k0.size(3) != D || Hkv < 1 || H % Hkv) Py_RETURN_NONE;
    if (gate0.dim() != 2 || gate0.size(0) != H || gate0.size(1) != (p.gate_mode ? 2 * D + 1 : 2) ||
        gate0.device() != q0.device() || !at::isFloatingType(gate0.scalar_type()))
      Py_RETURN_NONE;
    Tensor lens;
    if (a[4] != Py_None) {
      if (!THPVariable_Check(a[4])) Py_RETURN_NONE;
      lens = THPVariable_Unpack(a[4]);
      if (lens.dim() != 1 || lens.size(0) != B || lens.device() != q0.device() ||
          (lens.scalar_type() != at::kInt && lens.scalar_type() != at::kLong))
        Py_RETURN_NONE;
      if (lens.scalar_type() != at::kInt || !lens.is_contiguous()) lens = lens.to(at::kInt).contiguous();
    }
    Tensor phi;
    if (a[5] != Py_None) phi = THPVariable_Unpack(a[5]);  // (checked by the caller)

    // (the tangents would be dropped without a word)
    for (const Tensor *t : {&q0, &k0, &v0, &gate0})
      if (t->_fw_grad(/*level=*/0).defined()) {
        PyErr_SetString(PyExc_NotImplementedError, "blossom_attention has no forward-mode derivative");
        return nullptr;
      }

    c10::cuda::CUDAGuard guard(q0.device());
    Tensor q = q0, k = k0, v = v0, gate = gate0;
    {
      at::NoGradGuard no_grad;
      // The library addresses every q-shaped buffer with q's strides and every k-shaped one with k's:
      // views that are not dense (a slice of a packed projection) are copied first.
      if (!(dense(q) && q.stride(3) == 1)) q = packed(q);
      if (!(dense(k) && k.stride(3) == 1 && k.strides() == v.strides())) {
        k = packed(k);
        v = packed(v);
      }
      if (Hkv == H && k.strides() != q.strides()) {
        k = copied(k, like(q));
        v = copied(v, like(q));
      }
      if (gate.scalar_type() != at::kFloat || !gate.is_contiguous()) gate = gate.to(at::kFloat).contiguous();
      for (Tensor *t : {&q, &k, &v, &gate, &lens, &phi}) make_plain(*t);
    }
    p.batch = (int32_t)B;
    p.heads = (int32_t)H;
    p.kv_heads = (int32_t)Hkv;
    p.seq_len = (int32_t)L;
    p.head_dim = (int32_t)D;
    p.dtype = dt == at::kFloat ? BLOSSOM_DTYPE_FP32 : BLOSSOM_DTYPE_BF16;
    p.stride_b = q.stride(0);
    p.stride_h = q.stride(1);
    p.stride_l = q.stride(2);
    p.kv_stride_b = k.stride(0);
    p.kv_stride_h = k.stride(1);
    p.kv_stride_l = k.stride(2);
    p.phi_logits = phi.defined() ? phi.data_ptr<float>() : nullptr;
    const size_t ws_bytes = blossom_workspace_bytes(&p);
    if (ws_bytes == 0) return raise_blossom(BLOSSOM_ERR_UNSUPPORTED, "blossom_workspace_bytes");

    const bool grad = torch::autograd::compute_requires_grad(q0, k0, v0, gate0);
    const at::Device dev = q.device();
    Scratch s;
    s.span = grad ? align256((size_t)q.numel() * q.element_size()) : 0;
    s.lse_bytes = grad ? align256((size_t)2 * B * H * L * sizeof(float)) : 0;
    s.ws_bytes = ws_bytes;
    const Tensor buf = fresh({(int64_t)s.bytes()}, at::kByte, dev);
    char *const base = static_cast<char *>(buf.data_ptr());
    const int64_t rows = p.select_mode ? L : (L + p.block_size - 1) / p.block_size;
    Tensor out = like(q), idx = fresh({B, Hkv, rows, p.top_k}, at::kInt, dev);
    const blossom_stream_t st = (blossom_stream_t)c10::cuda::getCurrentCUDAStream(dev.index()).stream();
    // Every address is taken before the interpreter is let go: a tensor without memory of its own (a batched
    // one inside vmap) throws here, and an exception must not leave the block below.
    const void *qp = q.data_ptr(), *kp = k.data_ptr(), *vp = v.data_ptr();
    const float *gp = gate.data_ptr<float>();
    const int32_t *np = lens.defined() ? lens.data_ptr<int32_t>() : nullptr;
    int32_t *ip = idx.data_ptr<int32_t>();
    void *op = out.data_ptr(), *lp = grad ? s.out_lt(base) : nullptr, *sp = grad ? s.out_st(base) : nullptr,
         *wp = s.workspace(base);
    float *ep = grad ? s.lse(base) : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = blossom_attn_fwd(&p, qp, kp, vp, gp, np, ip, 0, op, lp, sp, ep, wp, ws_bytes, st);
    Py_END_ALLOW_THREADS;
    if (rc) return raise_blossom(rc, "blossom_attn_fwd");
    if (grad) {
      auto node = std::shared_ptr<BlossomAttentionBackward>(new BlossomAttentionBackward(), torch::autograd::deleteNode);
      node->set_next_edges(torch::autograd::collect_next_edges(q0, k0, v0, gate0));
      node->q_ = SavedVariable(q, false);
      node->k_ = SavedVariable(k, false);
      node->v_ = SavedVariable(v, false);
      node->gate_ = SavedVariable(gate.is_same(gate0) ? gate : gate.detach(), false);
      node->idx_ = SavedVariable(idx, false);
      node->buf_ = SavedVariable(buf, false);
      node->lens_ = lens;
      node->phi_ = phi;
      node->scratch_ = s;
      node->params_ = p;
      node->gate_type_ = gate0.scalar_type();
      torch::autograd::set_history(out, node);
    }
    PyObject *res = PyTuple_New(2);
    if (!res) return nullptr;
    PyTuple_SET_ITEM(res, 0, THPVariable_Wrap(std::move(out)));
    PyTuple_SET_ITEM(res, 1, THPVariable_Wrap(std::move(idx)));
    return res;
  } catch (const std::exception &e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// ---- rows around the attention: dropout, residual + layer norm ------------------------------------
// A tensor as rows of its last dimension with one stride between them.
struct RowView {
  int64_t rows = 0, cols = 0, stride = 0;
};
bool row_view(const Tensor &t, RowView *v) {
  const int64_t d = t.dim();
  v->cols = t.size(d - 1);
  v->rows = 1;
  v->stride = v->cols;
  if (t.stride(d - 1) != 1 && v->cols > 1) return false;
  for (int64_t i = d - 2; i >= 0; --i) {
    if (t.size(i) == 1) continue;
    if (v->rows == 1) v->stride = t.stride(i);
    else if (t.stride(i) != v->stride * v->rows) return false;
    v->rows *= t.size(i);
  }
  return v->stride >= v->cols;
}
// t, or a copy of it that is plain rows
Tensor as_rows(const Tensor &t, RowView *v) {
  if (!t.defined()) return t;
  Tensor r = t;
  if (!row_view(r, v)) {
    r = r.contiguous();
    row_view(r, v);
  }
  make_plain(r);
  return r;
}
const void *address(const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }
blossom_stream_t stream_of(const Tensor &t) {
  return (blossom_stream_t)c10::cuda::getCurrentCUDAStream(t.device().index()).stream();
}

// What a node saved, as the saved-tensor hooks return it: the same numbers, in any layout (offloading to the host gives a slice
// of a wider buffer back without the gaps), so that strides are those of what came back.
void expect_saved(bool same, const char *what) {
  if (!same) throw std::runtime_error(std::string(what) + ": a saved-tensor hook returned another tensor than it was given");
}
Tensor saved_rows(const SavedVariable &saved, int64_t rows, int64_t cols, at::ScalarType type, at::Device dev, const char *what,
                  RowView *v) {
  const Tensor t = saved.unpack();
  expect_saved(t.defined() && t.device() == dev && t.scalar_type() == type && t.dim() > 0, what);
  const Tensor r = as_rows(t, v);
  expect_saved(v->rows == rows && v->cols == cols, what);
  return r;
}
Tensor saved_plain(const SavedVariable &saved, int64_t numel, at::ScalarType type, at::Device dev, const char *what) {
  const Tensor t = saved.unpack();
  expect_saved(t.defined() && t.device() == dev && t.scalar_type() == type && t.numel() == numel, what);
  Tensor r = t.contiguous();
  make_plain(r);
  return r;
}

// The gradients are not differentiable again: asked for a graph of them, whoever uses it is told so.
void once_differentiable(variable_list &res, const char *what) {
  if (!at::GradMode::is_enabled()) return;
  for (Tensor &t : res)
    if (t.defined()) {
      t = t.detach();
      auto node = std::shared_ptr<Node>(
          new torch::autograd::Error(std::string(what) + " has no second derivative"), torch::autograd::deleteNode);
      torch::autograd::set_history(t, node);
    }
}

struct BlossomDropoutBackward : public Node {
  SavedVariable rng_;
  blossom_rows_params params_;

  std::string name() const override { return "BlossomDropoutBackward"; }
  void release_variables() override { rng_.reset_data(); }
  variable_list apply(variable_list &&grads) override {
    variable_list res(1);
    if (!grads[0].defined()) return res;
    {
      at::NoGradGuard no_grad;
      c10::cuda::CUDAGuard guard(grads[0].device());
      const Tensor rng = saved_plain(rng_, 2, at::kLong, grads[0].device(), "blossom_dropout");
      RowView v;
      const Tensor dout = as_rows(grads[0], &v);
      const Tensor dx = fresh(dout.sizes(), dout.scalar_type(), dout.device());
      blossom_rows_params p = params_;
      p.x_stride = v.stride;
      p.out_stride = 0;
      const int rc = blossom_dropout(&p, dout.data_ptr(), rng.data_ptr<int64_t>(), dx.data_ptr(), stream_of(dout));
      if (rc) throw std::runtime_error(failure("blossom_dropout", rc));
      res[0] = dx;
    }
    once_differentiable(res, "blossom_dropout");
    return res;
  }
};

struct BlossomAddNormBackward : public Node {
  SavedVariable x_, res_, weight_, rng_, stats_;
  blossom_rows_params params_;
  bool has_res_, has_weight_, has_bias_;

  std::string name() const override { return "BlossomAddNormBackward"; }
  void release_variables() override {
    for (SavedVariable *v : {&x_, &res_, &weight_, &rng_, &stats_}) v->reset_data();
  }
  variable_list apply(variable_list &&grads) override {
    variable_list out(4);  // x, residual, weight, bias
    if (!grads[0].defined()) return out;
    {
      at::NoGradGuard no_grad;
      const char *const what = "blossom_add_norm";
      blossom_rows_params p = params_;
      const at::Device dev = grads[0].device();
      const auto type = p.dtype == BLOSSOM_DTYPE_FP32 ? at::kFloat : at::kBFloat16,
                 wtype = p.weight_dtype == BLOSSOM_DTYPE_FP32 ? at::kFloat : at::kBFloat16;
      c10::cuda::CUDAGuard guard(dev);
      RowView xv, rv, v;
      Tensor res, weight, rng;
      const Tensor x = saved_rows(x_, p.rows, p.cols, type, dev, what, &xv);
      if (has_res_) res = saved_rows(res_, p.rows, p.cols, type, dev, what, &rv);
      if (has_weight_) weight = saved_plain(weight_, p.cols, wtype, dev, what);
      if (p.dropout > 0.0) rng = saved_plain(rng_, 2, at::kLong, dev, what);
      const Tensor stats = saved_plain(stats_, 2 * p.rows, at::kFloat, dev, what);
      const Tensor dout = as_rows(grads[0], &v);
      p.x_stride = xv.stride;
      p.residual_stride = rv.stride;
      p.out_stride = v.stride;
      const bool want_x = task_should_compute_output(0), want_res = res.defined() && task_should_compute_output(1);
      // without dropout the two gradients are one
      if (want_x || (want_res && p.dropout == 0.0)) out[0] = fresh(dout.sizes(), type, dev);
      if (want_res && p.dropout > 0.0) out[1] = fresh(dout.sizes(), type, dev);
      if (weight.defined() && task_should_compute_output(2)) out[2] = fresh({p.cols}, wtype, dev);
      if (has_bias_ && task_should_compute_output(3)) out[3] = fresh({p.cols}, wtype, dev);
      const size_t bytes = out[2].defined() || out[3].defined() ? blossom_add_norm_workspace_bytes(&p) : 0;
      Tensor ws;
      if (bytes) ws = fresh({(int64_t)bytes}, at::kByte, dev);
      auto at = [](const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; };
      const int rc = blossom_add_norm_bwd(&p, x.data_ptr(), at(res), at(weight), static_cast<const int64_t *>(at(rng)),
                                          stats.data_ptr<float>(), dout.data_ptr(), at(out[0]), at(out[1]), at(out[2]),
                                          at(out[3]), at(ws), bytes, stream_of(x));
      if (rc) throw std::runtime_error(failure("blossom_add_norm_bwd", rc));
      if (want_res && p.dropout == 0.0) {
        out[1] = out[0];
        if (!want_x) out[0] = Tensor();
      }
    }
    once_differentiable(out, "blossom_add_norm");
    return out;
  }
};

bool row_type(const Tensor &t) { return t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16; }
int32_t type_code(const Tensor &t) { return t.scalar_type() == at::kFloat ? BLOSSOM_DTYPE_FP32 : BLOSSOM_DTYPE_BF16; }
// an argument that may be None
bool optional(PyObject *o, Tensor *t) {
  if (o == Py_None) return true;
  if (!THPVariable_Check(o)) return false;
  *t = THPVariable_Unpack(o);
  return true;
}
bool rng_ok(const Tensor &rng, const Tensor &x) {
  return rng.defined() && rng.scalar_type() == at::kLong && rng.dim() == 1 && rng.size(0) == 2 && rng.device() == x.device();
}
PyObject *no_tangents(const char *what) {
  return PyErr_Format(PyExc_NotImplementedError, "%s has no forward-mode derivative", what);
}
bool has_tangent(const Tensor &t) { return t.defined() && t._fw_grad(/*level=*/0).defined(); }

// dropout(x, p, rng, site) -> out; None: not what the library can be handed (autograd.check_rows says why)
PyObject *dropout(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 4) return PyErr_Format(PyExc_TypeError, "dropout() takes 4 arguments");
  blossom_rows_params p = {};
  p.dropout = PyFloat_AsDouble(a[1]);
  if ((p.dropout == -1.0 && PyErr_Occurred()) || !read_int(a[3], &p.site)) return nullptr;
  try {
    Tensor rng;
    if (!THPVariable_Check(a[0]) || !optional(a[2], &rng)) Py_RETURN_NONE;
    const Tensor &x0 = THPVariable_Unpack(a[0]);
    if (!x0.is_cuda() || !row_type(x0) || x0.dim() < 1 || x0.size(x0.dim() - 1) < 1 || !rng_ok(rng, x0)) Py_RETURN_NONE;
    if (has_tangent(x0)) return no_tangents("blossom_dropout");
    c10::cuda::CUDAGuard guard(x0.device());
    Tensor x, state;
    RowView v;
    {
      at::NoGradGuard no_grad;
      x = as_rows(x0, &v);
      state = rng.contiguous();
      make_plain(state);
    }
    p.rows = v.rows;
    p.cols = (int32_t)std::min<int64_t>(v.cols, INT32_MAX);
    p.dtype = p.weight_dtype = type_code(x);
    p.x_stride = v.stride;
    Tensor out = fresh(x.sizes(), x.scalar_type(), x.device());
    const void *xp = address(x);
    const int64_t *rp = state.data_ptr<int64_t>();
    void *op = out.data_ptr();
    const blossom_stream_t st = stream_of(x);
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = blossom_dropout(&p, xp, rp, op, st);
    Py_END_ALLOW_THREADS;
    if (rc) return raise_blossom(rc, "blossom_dropout");
    if (torch::autograd::compute_requires_grad(x0)) {
      auto node = std::shared_ptr<BlossomDropoutBackward>(new BlossomDropoutBackward(), torch::autograd::deleteNode);
      node->set_next_edges(torch::autograd::collect_next_edges(x0));
      node->rng_ = SavedVariable(state, false);
      node->params_ = p;
      torch::autograd::set_history(out, node);
    }
    return THPVariable_Wrap(std::move(out));
  } catch (const std::exception &e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// add_norm(x, residual, weight, bias, p, rng, site, eps) -> out; None: as above
PyObject *add_norm(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 8) return PyErr_Format(PyExc_TypeError, "add_norm() takes 8 arguments");
  blossom_rows_params p = {};
  p.dropout = PyFloat_AsDouble(a[4]);
  if ((p.dropout == -1.0 && PyErr_Occurred()) || !read_int(a[6], &p.site)) return nullptr;
  p.eps = PyFloat_AsDouble(a[7]);
  if (p.eps == -1.0 && PyErr_Occurred()) return nullptr;
  try {
    Tensor res0, weight0, bias0, rng;
    if (!THPVariable_Check(a[0]) || !optional(a[1], &res0) || !optional(a[2], &weight0) || !optional(a[3], &bias0) ||
        !optional(a[5], &rng))
      Py_RETURN_NONE;
    const Tensor &x0 = THPVariable_Unpack(a[0]);
    if (!x0.is_cuda() || !row_type(x0) || x0.dim() < 1 || x0.size(x0.dim() - 1) < 1) Py_RETURN_NONE;
    if (res0.defined() && (res0.sizes() != x0.sizes() || res0.scalar_type() != x0.scalar_type() || res0.device() != x0.device()))
      Py_RETURN_NONE;
    for (const Tensor *t : {&weight0, &bias0})
      if (t->defined() && (t->dim() != 1 || t->size(0) != x0.size(x0.dim() - 1) || !row_type(*t) || t->device() != x0.device()))
        Py_RETURN_NONE;
    if (weight0.defined() && bias0.defined() && weight0.scalar_type() != bias0.scalar_type()) Py_RETURN_NONE;
    if (p.dropout != 0.0 && !rng_ok(rng, x0)) Py_RETURN_NONE;
    for (const Tensor *t : {&x0, (const Tensor *)&res0, (const Tensor *)&weight0, (const Tensor *)&bias0})
      if (has_tangent(*t)) return no_tangents("blossom_add_norm");
    c10::cuda::CUDAGuard guard(x0.device());
    Tensor x, res, weight = weight0, bias = bias0, state;
    RowView v, rv;
    {
      at::NoGradGuard no_grad;
      x = as_rows(x0, &v);
      res = as_rows(res0, &rv);
      for (Tensor *t : {&weight, &bias})
        if (t->defined()) {
          *t = t->contiguous();
          make_plain(*t);
        }
      if (p.dropout != 0.0) {
        state = rng.contiguous();
        make_plain(state);
      }
    }
    p.rows = v.rows;
    p.cols = (int32_t)std::min<int64_t>(v.cols, INT32_MAX);
    p.dtype = type_code(x);
    p.weight_dtype = weight.defined() ? type_code(weight) : bias.defined() ? type_code(bias) : p.dtype;
    p.x_stride = v.stride;
    p.residual_stride = rv.stride;
    const bool grad = torch::autograd::compute_requires_grad(x0, res0, weight0, bias0);
    Tensor out = fresh(x.sizes(), x.scalar_type(), x.device()), stats;
    if (grad) stats = fresh({v.rows, 2}, at::kFloat, x.device());
    const void *xp = address(x), *ep = address(res), *wp = address(weight), *bp = address(bias);
    const int64_t *rp = state.defined() ? state.data_ptr<int64_t>() : nullptr;
    void *op = out.data_ptr();
    float *sp = grad ? stats.data_ptr<float>() : nullptr;
    const blossom_stream_t st = stream_of(x);
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = blossom_add_norm_fwd(&p, xp, ep, wp, bp, rp, op, sp, st);
    Py_END_ALLOW_THREADS;
    if (rc) return raise_blossom(rc, "blossom_add_norm_fwd");
    if (grad) {
      auto node = std::shared_ptr<BlossomAddNormBackward>(new BlossomAddNormBackward(), torch::autograd::deleteNode);
      node->set_next_edges(torch::autograd::collect_next_edges(x0, res0, weight0, bias0));
      node->x_ = SavedVariable(x, false);
      node->res_ = SavedVariable(res, false);
      node->weight_ = SavedVariable(weight, false);
      node->rng_ = SavedVariable(state, false);
      node->stats_ = SavedVariable(stats, false);
      node->params_ = p;
      node->has_res_ = res.defined();
      node->has_weight_ = weight.defined();
      node->has_bias_ = bias.defined();
      torch::autograd::set_history(out, node);
    }
    return THPVariable_Wrap(std::move(out));
  } catch (const std::exception &e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// ---- sampled softmax loss ------------------------------------------------------------------------
struct BlossomSampledLossBackward : public Node {
  SavedVariable hidden_, table_, targets_, negatives_, lse_, grad_;
  blossom_loss_params params_;
  bool has_grad_;

  std::string name() const override { return "BlossomSampledLossBackward"; }
  void release_variables() override {
    for (SavedVariable *v : {&hidden_, &table_, &targets_, &negatives_, &lse_, &grad_}) v->reset_data();
  }
  variable_list apply(variable_list &&grads) override {
    variable_list out(2);  // hidden, table
    if (!grads[0].defined()) return out;
    {
      at::NoGradGuard no_grad;
      const char *const what = "blossom_sampled_loss";
      blossom_loss_params p = params_;
      const at::Device dev = grads[0].device();
      const auto type = p.dtype == BLOSSOM_DTYPE_FP32 ? at::kFloat : at::kBFloat16,
                 ids = p.index_bytes == 8 ? at::kLong : at::kInt;
      c10::cuda::CUDAGuard guard(dev);
      RowView hv, tv, nv;
      Tensor negatives, grad;
      const Tensor hidden = saved_rows(hidden_, p.rows, p.cols, type, dev, what, &hv);
      const Tensor table = saved_rows(table_, p.items, p.cols, type, dev, what, &tv);
      const Tensor targets = saved_plain(targets_, p.rows, ids, dev, what);
      if (p.negatives && p.negatives_stride) {
        negatives = saved_rows(negatives_, p.rows, p.negatives, ids, dev, what, &nv);
        p.negatives_stride = nv.stride;
      } else if (p.negatives) {
        negatives = saved_plain(negatives_, p.negatives, ids, dev, what);
      }
      const Tensor lse = saved_plain(lse_, p.rows + 1, at::kFloat, dev, what);
      if (has_grad_) grad = saved_plain(grad_, p.rows * p.cols, at::kFloat, dev, what);
      p.hidden_stride = hv.stride;
      p.table_stride = tv.stride;
      Tensor g = grads[0];
      make_plain(g);
      if (grad.defined() && task_should_compute_output(0)) out[0] = fresh(hidden.sizes(), hidden.scalar_type(), dev);
      Tensor ws;
      if (task_should_compute_output(1)) {
        out[1] = fresh(table.sizes(), table.scalar_type(), dev);
        ws = fresh({(int64_t)blossom_sampled_loss_workspace_bytes(&p)}, at::kByte, dev);
      }
      auto at = [](const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; };
      if (out[0].defined() || out[1].defined()) {
        const int rc = blossom_sampled_loss_bwd(
            &p, hidden.data_ptr(), table.data_ptr(), targets.data_ptr(), at(negatives), lse.data_ptr<float>(),
            static_cast<const float *>(at(grad)), g.data_ptr<float>(), at(out[0]), at(out[1]), at(ws),
            ws.defined() ? (size_t)ws.nbytes() : 0, stream_of(hidden));
        if (rc) throw std::runtime_error(failure("blossom_sampled_loss_bwd", rc));
      }
    }
    once_differentiable(out, "blossom_sampled_loss");
    return out;
  }
};

// sampled_loss(hidden, table, targets, negatives, ignore_index, mask_hits) -> loss; None: not what the library can be
// handed (autograd.check_loss says why)
PyObject *sampled_loss(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 6) return PyErr_Format(PyExc_TypeError, "sampled_loss() takes 6 arguments");
  blossom_loss_params p = {};
  p.ignore_index = PyLong_AsLongLong(a[4]);
  if ((p.ignore_index == -1 && PyErr_Occurred()) || !read_int(a[5], &p.mask_hits)) return nullptr;
  try {
    for (int i = 0; i < 4; ++i)
      if (!THPVariable_Check(a[i])) Py_RETURN_NONE;
    const Tensor &hidden0 = THPVariable_Unpack(a[0]), &table0 = THPVariable_Unpack(a[1]),
                 &targets0 = THPVariable_Unpack(a[2]), &negatives0 = THPVariable_Unpack(a[3]);
    const int64_t d = hidden0.dim();
    if (!hidden0.is_cuda() || !row_type(hidden0) || d < 1 || hidden0.size(d - 1) < 1 || table0.dim() != 2 ||
        table0.size(1) != hidden0.size(d - 1) || table0.size(0) < 1 || table0.scalar_type() != hidden0.scalar_type())
      Py_RETURN_NONE;
    for (const Tensor *t : {&table0, &targets0, &negatives0})
      if (t->device() != hidden0.device()) Py_RETURN_NONE;
    const at::ScalarType ids = targets0.scalar_type();
    if ((ids != at::kLong && ids != at::kInt) || negatives0.scalar_type() != ids) Py_RETURN_NONE;
    const at::IntArrayRef lead = hidden0.sizes().slice(0, d - 1);
    if (targets0.sizes() != lead || negatives0.dim() < 1) Py_RETURN_NONE;
    const bool shared = negatives0.dim() == 1;
    if (!shared && (negatives0.dim() != d || negatives0.sizes().slice(0, d - 1) != lead)) Py_RETURN_NONE;
    for (const Tensor *t : {&hidden0, &table0})
      if (has_tangent(*t)) return no_tangents("blossom_sampled_loss");
    c10::cuda::CUDAGuard guard(hidden0.device());
    Tensor hidden, table, targets, negatives = negatives0;
    RowView hv, tv, nv;
    {
      at::NoGradGuard no_grad;
      hidden = as_rows(hidden0, &hv);
      table = as_rows(table0, &tv);
      targets = targets0.contiguous();
      bool one = true;  // the same ids for every position: a vector, or one that is expanded
      for (int64_t i = 0; i + 1 < negatives.dim(); ++i) one = one && (negatives.stride(i) == 0 || negatives.size(i) == 1);
      if (one && negatives.numel()) {
        while (negatives.dim() > 1) negatives = negatives.select(0, 0);
        negatives = negatives.contiguous();
        nv.stride = 0;
      } else {
        negatives = as_rows(negatives, &nv);
      }
      for (Tensor *t : {&targets, &negatives}) make_plain(*t);
    }
    const int64_t n_neg = negatives0.size(negatives0.dim() - 1);
    if (n_neg >= INT32_MAX || table.size(0) > INT32_MAX || hv.cols > INT32_MAX)
      return raise_blossom(BLOSSOM_ERR_UNSUPPORTED, "blossom_sampled_loss_fwd");
    p.rows = hv.rows;
    p.cols = (int32_t)hv.cols;
    p.items = (int32_t)table.size(0);
    p.negatives = (int32_t)n_neg;
    p.dtype = type_code(hidden);
    p.index_bytes = ids == at::kLong ? 8 : 4;
    p.hidden_stride = hv.stride;
    p.table_stride = tv.stride;
    p.negatives_stride = n_neg ? nv.stride : 0;
    const at::Device dev = hidden.device();
    const bool grad = torch::autograd::compute_requires_grad(hidden0, table0);
    const bool grad_hidden = grad && hidden0.requires_grad();
    Tensor loss = fresh({}, at::kFloat, dev), lse = fresh({hv.rows + 1}, at::kFloat, dev), gh;
    if (grad_hidden) gh = fresh({hv.rows, hv.cols}, at::kFloat, dev);
    const Tensor ws = fresh({BLOSSOM_LOSS_FORWARD_BYTES}, at::kByte, dev);
    const void *hp = address(hidden), *tp = address(table), *gp = address(targets), *np = n_neg ? address(negatives) : nullptr;
    float *lp = loss.data_ptr<float>(), *sp = lse.data_ptr<float>(), *dp = gh.defined() ? gh.data_ptr<float>() : nullptr;
    void *wp = ws.data_ptr();
    const blossom_stream_t st = stream_of(hidden);
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = blossom_sampled_loss_fwd(&p, hp, tp, gp, np, lp, sp, dp, wp, BLOSSOM_LOSS_FORWARD_BYTES, st);
    Py_END_ALLOW_THREADS;
    if (rc) return raise_blossom(rc, "blossom_sampled_loss_fwd");
    if (grad) {
      auto node = std::shared_ptr<BlossomSampledLossBackward>(new BlossomSampledLossBackward(), torch::autograd::deleteNode);
      node->set_next_edges(torch::autograd::collect_next_edges(hidden0, table0));
      node->hidden_ = SavedVariable(hidden, false);
      node->table_ = SavedVariable(table, false);
      node->targets_ = SavedVariable(targets, false);
      node->negatives_ = SavedVariable(n_neg ? negatives : Tensor(), false);
      node->lse_ = SavedVariable(lse, false);
      node->grad_ = SavedVariable(gh, false);
      node->has_grad_ = gh.defined();
      node->params_ = p;
      torch::autograd::set_history(loss, node);
    }
    return THPVariable_Wrap(std::move(loss));
  } catch (const std::exception &e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// dense(tensor) -> bool, like(tensor) -> tensor: the two rules above, for the host-side tests
PyObject *py_dense(PyObject *, PyObject *t) {
  if (!THPVariable_Check(t)) return PyErr_Format(PyExc_TypeError, "dense() takes a tensor");
  return PyBool_FromLong(dense(THPVariable_Unpack(t)));
}
PyObject *py_like(PyObject *, PyObject *t) {
  if (!THPVariable_Check(t)) return PyErr_Format(PyExc_TypeError, "like() takes a tensor");
  try {
    return THPVariable_Wrap(like(THPVariable_Unpack(t)));
  } catch (const std::exception &e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

PyMethodDef methods[] = {
    {"dense", py_dense, METH_O, nullptr},
    {"like", py_like, METH_O, nullptr},
    {"attention", (PyCFunction)(void (*)(void))attention, METH_FASTCALL, nullptr},
    {"dropout", (PyCFunction)(void (*)(void))dropout, METH_FASTCALL, nullptr},
    {"add_norm", (PyCFunction)(void (*)(void))add_norm, METH_FASTCALL, nullptr},
    {"sampled_loss", (PyCFunction)(void (*)(void))sampled_loss, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_front", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__front(void) { return PyModule_Create(&module); }
