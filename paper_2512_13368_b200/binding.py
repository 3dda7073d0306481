"""ctypes binding of ``libblossom.so`` (the C ABI declared in ``include/blossom.h``).

Argument marshalling only: every step of the path runs in the CUDA library.  Functions keep
the C names.  Tensor arguments may be ``torch.Tensor`` (their ``data_ptr()`` is passed), an
``int`` address, or ``None`` (NULL).  A non-zero status raises ``BlossomError``.  There is no
fallback: if the shared library is missing the first call raises.
"""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libblossom.so")

BLOSSOM_OK = 0
BLOSSOM_ERR_INVALID_ARG = 1
BLOSSOM_ERR_UNSUPPORTED = 2
BLOSSOM_ERR_WORKSPACE = 3
BLOSSOM_ERR_CUDA = 4
BLOSSOM_ERR_TIMEOUT = 5
BLOSSOM_ERR_TOO_LARGE = 6
DTYPE_FP32 = 0
DTYPE_BF16 = 1

EXPORTS = (
    "blossom_workspace_bytes", "blossom_select_blocks", "blossom_select_blocks_static",
    "blossom_attn_fwd", "blossom_attn_bwd",
    "blossom_device_status", "blossom_status_string", "blossom_version", "blossom_launch_count",
    "blossom_profile_start", "blossom_profile_every", "blossom_profile_stop", "blossom_kernel_name",
    "blossom_debug_switch",
    "blossom_selftest_wait_timeout", "blossom_copy_rows", "blossom_launch_plan",
    "blossom_dropout", "blossom_add_norm_fwd", "blossom_add_norm_bwd", "blossom_add_norm_workspace_bytes",
    "blossom_sampled_loss_fwd", "blossom_sampled_loss_bwd", "blossom_sampled_loss_workspace_bytes",
    "blossom_embedding_fwd", "blossom_embedding_bwd", "blossom_embedding_workspace_bytes",
    "blossom_pack_rows", "blossom_unpack_rows",
    "blossom_linear_fwd", "blossom_linear_bwd", "blossom_linear_workspace_bytes", "blossom_linear_bwd_workspace_bytes",
)
LOSS_FORWARD_BYTES = 65536  # what blossom_sampled_loss_fwd uses of its workspace
LINEAR_FORWARD_BYTES = 256  # the same of blossom_linear_fwd
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}


class blossom_params(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
        ("seq_len", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("block_size", ctypes.c_int32),
        ("top_k", ctypes.c_int32), ("window", ctypes.c_int32), ("causal", ctypes.c_int32),
        ("select_mode", ctypes.c_int32), ("dtype", ctypes.c_int32), ("sm_scale", ctypes.c_float),
        ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_l", ctypes.c_int64),
        ("stis_mode", ctypes.c_int32), ("stis_block", ctypes.c_int32),
        ("cmp_block", ctypes.c_int32), ("cmp_stride", ctypes.c_int32),
        ("kv_stride_b", ctypes.c_int64), ("kv_stride_h", ctypes.c_int64), ("kv_stride_l", ctypes.c_int64),
        ("phi_logits", ctypes.c_void_p), ("gate_mode", ctypes.c_int32),
        ("rope_theta", ctypes.c_float),
        ("reuse_tile_lists", ctypes.c_int32),
    ]


class blossom_rows_params(ctypes.Structure):
    _fields_ = [
        ("rows", ctypes.c_int64), ("cols", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("weight_dtype", ctypes.c_int32), ("site", ctypes.c_int32),
        ("dropout", ctypes.c_double), ("eps", ctypes.c_double),
        ("x_stride", ctypes.c_int64), ("residual_stride", ctypes.c_int64), ("out_stride", ctypes.c_int64),
        ("dx_stride", ctypes.c_int64), ("dresidual_stride", ctypes.c_int64),
    ]


class blossom_loss_params(ctypes.Structure):
    _fields_ = [
        ("rows", ctypes.c_int64), ("cols", ctypes.c_int32), ("items", ctypes.c_int32),
        ("negatives", ctypes.c_int32), ("dtype", ctypes.c_int32), ("index_bytes", ctypes.c_int32),
        ("mask_hits", ctypes.c_int32), ("ignore_index", ctypes.c_int64),
        ("hidden_stride", ctypes.c_int64), ("table_stride", ctypes.c_int64), ("dhidden_stride", ctypes.c_int64),
        ("dtable_stride", ctypes.c_int64), ("negatives_stride", ctypes.c_int64),
    ]


class blossom_embedding_params(ctypes.Structure):
    _fields_ = [
        ("rows", ctypes.c_int64), ("cols", ctypes.c_int32), ("items", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("index_bytes", ctypes.c_int32), ("padding", ctypes.c_int64),
        ("scale", ctypes.c_double), ("table_stride", ctypes.c_int64), ("out_stride", ctypes.c_int64),
        ("dtable_stride", ctypes.c_int64),
    ]


class blossom_linear_params(ctypes.Structure):
    _fields_ = [
        ("rows", ctypes.c_int64), ("cols", ctypes.c_int32), ("outs", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("activation", ctypes.c_int32), ("packed", ctypes.c_int32),
        ("x_stride", ctypes.c_int64), ("weight_stride", ctypes.c_int64), ("residual_stride", ctypes.c_int64),
        ("out_stride", ctypes.c_int64), ("dx_stride", ctypes.c_int64), ("dweight_stride", ctypes.c_int64),
    ]


class BlossomError(RuntimeError):
    def __init__(self, status, where):
        self.status = int(status)
        super().__init__(f"{where}: {blossom_status_string(status)} (status {int(status)})")


_lib = None


def load():
    """Load the shared library (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2512_13368_b200.build` "
            "(there is no CPU or PyTorch fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    pp = ctypes.POINTER(blossom_params)
    lib.blossom_workspace_bytes.restype = sz
    lib.blossom_workspace_bytes.argtypes = [pp]
    lib.blossom_select_blocks.restype = ctypes.c_int
    lib.blossom_select_blocks.argtypes = [pp, vp, vp, vp, vp, vp, sz, vp]
    lib.blossom_select_blocks_static.restype = ctypes.c_int
    lib.blossom_select_blocks_static.argtypes = [pp, vp, vp, vp, vp, vp]
    lib.blossom_attn_fwd.restype = ctypes.c_int
    lib.blossom_attn_fwd.argtypes = [pp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, sz, vp]
    lib.blossom_attn_bwd.restype = ctypes.c_int
    lib.blossom_attn_bwd.argtypes = [pp] + [vp] * 15 + [sz, vp]
    lib.blossom_device_status.restype = ctypes.c_int
    lib.blossom_device_status.argtypes = [vp, vp, ctypes.POINTER(i32)]
    lib.blossom_status_string.restype = ctypes.c_char_p
    lib.blossom_status_string.argtypes = [ctypes.c_int]
    lib.blossom_version.restype = ctypes.c_int
    lib.blossom_launch_count.restype = ctypes.c_uint64
    lib.blossom_profile_start.restype = ctypes.c_int
    lib.blossom_profile_start.argtypes = [ctypes.c_int]
    lib.blossom_profile_every.restype = ctypes.c_int
    lib.blossom_profile_every.argtypes = [ctypes.c_int]
    lib.blossom_profile_stop.restype = ctypes.c_int
    lib.blossom_profile_stop.argtypes = [ctypes.POINTER(i32), ctypes.POINTER(ctypes.c_float), ctypes.c_int]
    lib.blossom_kernel_name.restype = ctypes.c_char_p
    lib.blossom_kernel_name.argtypes = [ctypes.c_int]
    lib.blossom_selftest_wait_timeout.restype = ctypes.c_int
    lib.blossom_selftest_wait_timeout.argtypes = [vp, sz, vp]
    lib.blossom_launch_plan.restype = ctypes.c_int
    lib.blossom_launch_plan.argtypes = [pp, ctypes.c_int, ctypes.c_int]
    lib.blossom_debug_switch.restype = ctypes.c_int
    lib.blossom_debug_switch.argtypes = [ctypes.c_int, ctypes.c_int]
    rp = ctypes.POINTER(blossom_rows_params)
    lib.blossom_dropout.restype = ctypes.c_int
    lib.blossom_dropout.argtypes = [rp] + [vp] * 4
    lib.blossom_add_norm_fwd.restype = ctypes.c_int
    lib.blossom_add_norm_fwd.argtypes = [rp] + [vp] * 8
    lib.blossom_add_norm_bwd.restype = ctypes.c_int
    lib.blossom_add_norm_bwd.argtypes = [rp] + [vp] * 11 + [sz, vp]
    lib.blossom_add_norm_workspace_bytes.restype = sz
    lib.blossom_add_norm_workspace_bytes.argtypes = [rp]
    lp = ctypes.POINTER(blossom_loss_params)
    lib.blossom_sampled_loss_workspace_bytes.restype = sz
    lib.blossom_sampled_loss_workspace_bytes.argtypes = [lp]
    lib.blossom_sampled_loss_fwd.restype = ctypes.c_int
    lib.blossom_sampled_loss_fwd.argtypes = [lp] + [vp] * 8 + [sz, vp]
    lib.blossom_sampled_loss_bwd.restype = ctypes.c_int
    lib.blossom_sampled_loss_bwd.argtypes = [lp] + [vp] * 10 + [sz, vp]
    ep = ctypes.POINTER(blossom_embedding_params)
    lib.blossom_embedding_workspace_bytes.restype = sz
    lib.blossom_embedding_workspace_bytes.argtypes = [ep]
    lib.blossom_embedding_fwd.restype = ctypes.c_int
    lib.blossom_embedding_fwd.argtypes = [ep] + [vp] * 4
    lib.blossom_embedding_bwd.restype = ctypes.c_int
    lib.blossom_embedding_bwd.argtypes = [ep] + [vp] * 4 + [sz, vp]
    lib.blossom_pack_rows.restype = ctypes.c_int
    lib.blossom_pack_rows.argtypes = [rp] + [vp] * 4
    lib.blossom_unpack_rows.restype = ctypes.c_int
    lib.blossom_unpack_rows.argtypes = [rp] + [vp] * 4
    np_ = ctypes.POINTER(blossom_linear_params)
    lib.blossom_linear_workspace_bytes.restype = sz
    lib.blossom_linear_workspace_bytes.argtypes = [np_]
    lib.blossom_linear_bwd_workspace_bytes.restype = sz
    lib.blossom_linear_bwd_workspace_bytes.argtypes = [np_] + [vp] * 3
    lib.blossom_linear_fwd.restype = ctypes.c_int
    lib.blossom_linear_fwd.argtypes = [np_] + [vp] * 6 + [sz, vp]
    lib.blossom_linear_bwd.restype = ctypes.c_int
    lib.blossom_linear_bwd.argtypes = [np_] + [vp] * 9 + [sz, vp]
    _lib = lib
    return lib


def _ptr(x):
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _nbytes(x):
    if x is None:
        return 0
    if isinstance(x, int):
        return x
    return x.numel() * x.element_size()


def _current_stream():
    """The current stream's handle: torch's raw accessor where it has one (a Stream object costs a few microseconds)."""
    global _raw_stream
    import torch
    if _raw_stream is None:
        torch.cuda.init()
        get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        dev = getattr(torch._C, "_cuda_getDevice", None)
        _raw_stream = (lambda: get(dev())) if get and dev else (lambda: torch.cuda.current_stream().cuda_stream)
    return _raw_stream()


_raw_stream = None


def _stream(stream):
    if stream is None:
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def make_params(batch, heads, seq_len, head_dim, block_size, top_k, window, dtype, sm_scale=0.0,
                strides=None, kv_heads=None, causal=1, select_mode=0, stis_mode=0,
                stis_block=1, cmp_block=0, cmp_stride=0, kv_strides=None, phi_logits=None,
                gate_mode=0, rope_theta=0.0, reuse_tile_lists=0) -> blossom_params:
    """Fill a ``blossom_params``; ``strides`` = (stride_b, stride_h, stride_l) in elements,
    default contiguous [B, H, L, D].  ``phi_logits``: float32 device tensor (the caller keeps it
    alive) or None."""
    if strides is None:
        strides = (heads * seq_len * head_dim, seq_len * head_dim, head_dim)
    d = {"fp32": DTYPE_FP32, "bf16": DTYPE_BF16}.get(dtype, dtype)
    return blossom_params(batch, heads, heads if kv_heads is None else kv_heads, seq_len, head_dim,
                          block_size, top_k, window, causal, select_mode, d, float(sm_scale),
                          int(strides[0]), int(strides[1]), int(strides[2]), int(stis_mode),
                          int(stis_block), int(cmp_block), int(cmp_stride),
                          *((0, 0, 0) if kv_strides is None else [int(x) for x in kv_strides]),
                          _ptr(phi_logits), int(gate_mode), float(rope_theta), int(reuse_tile_lists))


def blossom_status_string(status) -> str:
    return load().blossom_status_string(int(status)).decode()


def blossom_version() -> int:
    return int(load().blossom_version())


def blossom_launch_count() -> int:
    return int(load().blossom_launch_count())


def blossom_workspace_bytes(params) -> int:
    return int(load().blossom_workspace_bytes(ctypes.byref(params)))


def blossom_select_blocks(params, q, k, seq_lens, block_idx, workspace, workspace_bytes=None,
                          stream=None, check=True) -> int:
    rc = load().blossom_select_blocks(ctypes.byref(params), _ptr(q), _ptr(k), _ptr(seq_lens),
                                      _ptr(block_idx), _ptr(workspace),
                                      _nbytes(workspace) if workspace_bytes is None else workspace_bytes,
                                      _stream(stream))
    if rc and check:
        raise BlossomError(rc, "blossom_select_blocks")
    return rc


def blossom_select_blocks_static(params, q, k, seq_lens, block_idx, stream=None, check=True) -> int:
    """Selection without a caller workspace: the scratch is a fixed array inside the library, so
    nothing on the path allocates.  For callers that are handed tensors but may not allocate
    device memory themselves.  Capacity-limited (see include/blossom.h); calls that could overlap
    on one device must be serialised by the caller."""
    rc = load().blossom_select_blocks_static(ctypes.byref(params), _ptr(q), _ptr(k), _ptr(seq_lens),
                                             _ptr(block_idx), _stream(stream))
    if rc and check:
        raise BlossomError(rc, "blossom_select_blocks_static")
    return rc


def blossom_attn_fwd(params, q, k, v, gate_logits, seq_lens, block_idx, idx_is_input, out, out_lt,
                     out_st, lse, workspace, workspace_bytes=None, stream=None, check=True) -> int:
    rc = load().blossom_attn_fwd(ctypes.byref(params), _ptr(q), _ptr(k), _ptr(v), _ptr(gate_logits),
                                 _ptr(seq_lens), _ptr(block_idx), int(idx_is_input), _ptr(out),
                                 _ptr(out_lt), _ptr(out_st), _ptr(lse), _ptr(workspace),
                                 _nbytes(workspace) if workspace_bytes is None else workspace_bytes,
                                 _stream(stream))
    if rc and check:
        raise BlossomError(rc, "blossom_attn_fwd")
    return rc


def blossom_attn_bwd(params, q, k, v, gate_logits, seq_lens, block_idx, out_lt, out_st, lse, dout,
                     dq, dk, dv, dgate, workspace, workspace_bytes=None, stream=None,
                     check=True) -> int:
    rc = load().blossom_attn_bwd(ctypes.byref(params), _ptr(q), _ptr(k), _ptr(v), _ptr(gate_logits),
                                 _ptr(seq_lens), _ptr(block_idx), _ptr(out_lt), _ptr(out_st),
                                 _ptr(lse), _ptr(dout), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dgate),
                                 _ptr(workspace),
                                 _nbytes(workspace) if workspace_bytes is None else workspace_bytes,
                                 _stream(stream))
    if rc and check:
        raise BlossomError(rc, "blossom_attn_bwd")
    return rc


def _dtype(dtype):
    return {"fp32": DTYPE_FP32, "bf16": DTYPE_BF16}.get(dtype, dtype)


def make_rows_params(rows, cols, dtype, dropout=0.0, site=0, eps=1e-5, weight_dtype=None, x_stride=0, residual_stride=0,
                     out_stride=0, dx_stride=0, dresidual_stride=0) -> blossom_rows_params:
    """Fill a ``blossom_rows_params``; strides in elements from row to row, 0 = ``cols``; the weights' type is ``dtype``
    unless given."""
    return blossom_rows_params(int(rows), int(cols), _dtype(dtype), _dtype(dtype if weight_dtype is None else weight_dtype),
                               int(site), float(dropout), float(eps), int(x_stride), int(residual_stride),
                               int(out_stride), int(dx_stride), int(dresidual_stride))


def blossom_dropout(params, x, rng, out, stream=None, check=True) -> int:
    rc = load().blossom_dropout(ctypes.byref(params), _ptr(x), _ptr(rng), _ptr(out), _stream(stream))
    if rc and check:
        raise BlossomError(rc, "blossom_dropout")
    return rc


def blossom_add_norm_workspace_bytes(params) -> int:
    return int(load().blossom_add_norm_workspace_bytes(ctypes.byref(params)))


def blossom_add_norm_fwd(params, x, residual, weight, bias, rng, out, stats, stream=None, check=True) -> int:
    rc = load().blossom_add_norm_fwd(ctypes.byref(params), _ptr(x), _ptr(residual), _ptr(weight), _ptr(bias), _ptr(rng),
                                     _ptr(out), _ptr(stats), _stream(stream))
    if rc and check:
        raise BlossomError(rc, "blossom_add_norm_fwd")
    return rc


def blossom_add_norm_bwd(params, x, residual, weight, rng, stats, dout, dx, dresidual, dweight, dbias, workspace,
                         workspace_bytes=None, stream=None, check=True) -> int:
    rc = load().blossom_add_norm_bwd(ctypes.byref(params), _ptr(x), _ptr(residual), _ptr(weight), _ptr(rng), _ptr(stats),
                                     _ptr(dout), _ptr(dx), _ptr(dresidual), _ptr(dweight), _ptr(dbias), _ptr(workspace),
                                     _nbytes(workspace) if workspace_bytes is None else workspace_bytes,
                                     _stream(stream))
    if rc and check:
        raise BlossomError(rc, "blossom_add_norm_bwd")
    return rc


def make_loss_params(rows, cols, items, negatives, dtype, index_bytes=8, mask_hits=0, ignore_index=-100, hidden_stride=0,
                     table_stride=0, dhidden_stride=0, dtable_stride=0, negatives_stride=None) -> blossom_loss_params:
    """Fill a ``blossom_loss_params``; strides in elements, 0 = ``cols``; ``negatives_stride``: None = a row of
    ``negatives`` ids per position, 0 = the same ids for all."""
    return blossom_loss_params(int(rows), int(cols), int(items), int(negatives), _dtype(dtype), int(index_bytes),
                               int(mask_hits), int(ignore_index), int(hidden_stride), int(table_stride),
                               int(dhidden_stride), int(dtable_stride),
                               int(negatives if negatives_stride is None else negatives_stride))


def blossom_sampled_loss_workspace_bytes(params) -> int:
    return int(load().blossom_sampled_loss_workspace_bytes(ctypes.byref(params)))


def blossom_sampled_loss_fwd(params, hidden, table, targets, negatives, loss, lse, grad_hidden, workspace,
                             workspace_bytes=None, stream=None, check=True) -> int:
    rc = load().blossom_sampled_loss_fwd(ctypes.byref(params), _ptr(hidden), _ptr(table), _ptr(targets), _ptr(negatives),
                                         _ptr(loss), _ptr(lse), _ptr(grad_hidden), _ptr(workspace),
                                         _nbytes(workspace) if workspace_bytes is None else workspace_bytes,
                                         _stream(stream))
    if rc and check:
        raise BlossomError(rc, "blossom_sampled_loss_fwd")
    return rc


def blossom_sampled_loss_bwd(params, hidden, table, targets, negatives, lse, grad_hidden, grad_loss, dhidden, dtable,
                             workspace, workspace_bytes=None, stream=None, check=True) -> int:
    rc = load().blossom_sampled_loss_bwd(ctypes.byref(params), _ptr(hidden), _ptr(table), _ptr(targets), _ptr(negatives),
                                         _ptr(lse), _ptr(grad_hidden), _ptr(grad_loss), _ptr(dhidden), _ptr(dtable),
                                         _ptr(workspace),
                                         _nbytes(workspace) if workspace_bytes is None else workspace_bytes,
                                         _stream(stream))
    if rc and check:
        raise BlossomError(rc, "blossom_sampled_loss_bwd")
    return rc


def make_embedding_params(rows, cols, items, dtype, scale=1.0, padding=-1, index_bytes=8, table_stride=0, out_stride=0,
                          dtable_stride=0) -> blossom_embedding_params:
    """Fill a ``blossom_embedding_params``; strides in elements, 0 = ``cols``; ``padding``: None or -1 = no such item."""
    return blossom_embedding_params(int(rows), int(cols), int(items), _dtype(dtype), int(index_bytes),
                                    -1 if padding is None else int(padding), float(scale), int(table_stride),
                                    int(out_stride), int(dtable_stride))


def blossom_embedding_workspace_bytes(params) -> int:
    return int(load().blossom_embedding_workspace_bytes(ctypes.byref(params)))


def blossom_embedding_fwd(params, table, ids, out, stream=None, check=True) -> int:
    rc = load().blossom_embedding_fwd(ctypes.byref(params), _ptr(table), _ptr(ids), _ptr(out), _stream(stream))
    if rc and check:
        raise BlossomError(rc, "blossom_embedding_fwd")
    return rc


def blossom_embedding_bwd(params, ids, dout, dtable, workspace, workspace_bytes=None, stream=None, check=True) -> int:
    rc = load().blossom_embedding_bwd(ctypes.byref(params), _ptr(ids), _ptr(dout), _ptr(dtable), _ptr(workspace),
                                      _nbytes(workspace) if workspace_bytes is None else workspace_bytes, _stream(stream))
    if rc and check:
        raise BlossomError(rc, "blossom_embedding_bwd")
    return rc


def blossom_pack_rows(params, x, codes, scales, stream=None, check=True) -> int:
    rc = load().blossom_pack_rows(ctypes.byref(params), _ptr(x), _ptr(codes), _ptr(scales), _stream(stream))
    if rc and check:
        raise BlossomError(rc, "blossom_pack_rows")
    return rc


def blossom_unpack_rows(params, codes, scales, out, stream=None, check=True) -> int:
    rc = load().blossom_unpack_rows(ctypes.byref(params), _ptr(codes), _ptr(scales), _ptr(out), _stream(stream))
    if rc and check:
        raise BlossomError(rc, "blossom_unpack_rows")
    return rc


def make_linear_params(rows, cols, outs, dtype, activation="none", packed=False, x_stride=0, weight_stride=0,
                       residual_stride=0, out_stride=0, dx_stride=0, dweight_stride=0) -> blossom_linear_params:
    """Fill a ``blossom_linear_params``; strides in elements from row to row, 0 = rows without gaps."""
    return blossom_linear_params(int(rows), int(cols), int(outs), _dtype(dtype),
                                 int(ACTIVATIONS.get(activation, activation)), int(packed), int(x_stride),
                                 int(weight_stride), int(residual_stride), int(out_stride), int(dx_stride),
                                 int(dweight_stride))


def blossom_linear_workspace_bytes(params) -> int:
    return int(load().blossom_linear_workspace_bytes(ctypes.byref(params)))


def blossom_linear_bwd_workspace_bytes(params, x, weight, dout) -> int:
    """What the backward needs for tensors that lie where these do."""
    return int(load().blossom_linear_bwd_workspace_bytes(ctypes.byref(params), _ptr(x), _ptr(weight), _ptr(dout)))


def blossom_linear_fwd(params, x, weight, bias, residual, out, workspace, workspace_bytes=None, stream=None,
                       check=True) -> int:
    rc = load().blossom_linear_fwd(ctypes.byref(params), _ptr(x), _ptr(weight), _ptr(bias), _ptr(residual), _ptr(out),
                                   _ptr(workspace), _nbytes(workspace) if workspace_bytes is None else workspace_bytes,
                                   _stream(stream))
    if rc and check:
        raise BlossomError(rc, "blossom_linear_fwd")
    return rc


def blossom_linear_bwd(params, x, x_scales, weight, bias, dout, dx, dweight, dbias, workspace, workspace_bytes=None,
                       stream=None, check=True) -> int:
    rc = load().blossom_linear_bwd(ctypes.byref(params), _ptr(x), _ptr(x_scales), _ptr(weight), _ptr(bias), _ptr(dout),
                                   _ptr(dx), _ptr(dweight), _ptr(dbias), _ptr(workspace),
                                   _nbytes(workspace) if workspace_bytes is None else workspace_bytes, _stream(stream))
    if rc and check:
        raise BlossomError(rc, "blossom_linear_bwd")
    return rc


def blossom_device_status(workspace, stream=None) -> int:
    out = ctypes.c_int32(-1)
    rc = load().blossom_device_status(_ptr(workspace), _stream(stream), ctypes.byref(out))
    if rc:
        raise BlossomError(rc, "blossom_device_status")
    return int(out.value)


def blossom_profile_start(max_launches: int) -> None:
    rc = load().blossom_profile_start(int(max_launches))
    if rc:
        raise BlossomError(rc, "blossom_profile_start")


def blossom_profile_every(n: int) -> None:
    rc = load().blossom_profile_every(int(n))
    if rc:
        raise BlossomError(rc, "blossom_profile_every")


def blossom_profile_stop(capacity: int):
    """Returns a list of (kernel name, milliseconds), one entry per recorded launch."""
    ids = (ctypes.c_int32 * capacity)()
    ms = (ctypes.c_float * capacity)()
    n = load().blossom_profile_stop(ids, ms, int(capacity))
    if n < 0:
        raise RuntimeError("blossom_profile_stop failed (no profile running or a CUDA error)")
    return [(blossom_kernel_name(ids[i]), float(ms[i])) for i in range(n)]


def blossom_kernel_name(kernel_id: int) -> str:
    return load().blossom_kernel_name(int(kernel_id)).decode()


SWITCH_FORCE_SIMT = 0
SWITCH_EXACT_SELECT = 1
SWITCH_SERIAL_LAUNCH = 2


def blossom_debug_switch(which: int, value: int) -> None:
    """Process-wide debugging switch: 1 on, 0 off, -1 back to the environment's default."""
    rc = load().blossom_debug_switch(int(which), int(value))
    if rc:
        raise BlossomError(rc, "blossom_debug_switch")


PLAN_SHORT_SPLIT = 0
PLAN_DKDV_SPLIT = 1
PLAN_GATE_ROWS = 2


def blossom_launch_plan(params, which: int, lengths: bool) -> int:
    """How the backward of these params is launched (a ``PLAN_`` constant says what of it); 0 where that kernel does not run."""
    n = int(load().blossom_launch_plan(ctypes.byref(params), int(which), int(bool(lengths))))
    if n < 0:
        raise BlossomError(BLOSSOM_ERR_INVALID_ARG, "blossom_launch_plan")
    return n


def blossom_selftest_wait_timeout(workspace, stream=None) -> None:
    """Launch the diagnostic kernel whose only wait cannot complete; read the outcome with
    ``blossom_device_status(workspace)`` (it must be BLOSSOM_ERR_TIMEOUT)."""
    rc = load().blossom_selftest_wait_timeout(_ptr(workspace), _nbytes(workspace), _stream(stream))
    if rc:
        raise BlossomError(rc, "blossom_selftest_wait_timeout")
