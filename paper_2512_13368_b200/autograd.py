"""``torch.autograd`` front end of the library: ``blossom_attention(q, k, v, gate_logits, ...)``.

Plumbing only, and native (``csrc/front.cpp``, built into ``_front.so``): it allocates the outputs
and the workspace with PyTorch, calls ``blossom_attn_fwd`` / ``blossom_attn_bwd`` through the C ABI
on the current stream and hands the gradients back to autograd.  Every step of the method runs in
the CUDA library; there is no PyTorch fallback.  The selection is not differentiated (top-k is piecewise constant).
"""
from __future__ import annotations

import torch

from . import binding

_DT = {torch.float32: "fp32", torch.bfloat16: "bf16"}


def _dense(t) -> bool:
    """The native front end's test of a layout (``dense`` in ``csrc/front.cpp``): True if the tensor's elements
    tile its storage span without gaps or overlap."""
    return _module().dense(t)


def _like(t):
    """The native front end's output allocation (``like`` in ``csrc/front.cpp``): an uninitialised tensor with
    exactly t's shape AND strides."""
    return _module().like(t)


def check_arguments(q, k, v, gate_logits, seq_lens, require_cuda=True, gate_mode=0):
    """Why the native front end, which makes the same tests, would not take the arguments: raises for what
    is wrong with them (the library receives raw addresses, so a host tensor, a tensor on another device, a
    wrong integer width or a wrong shape would become a device memory fault instead of a Python error).
    Returns seq_lens as the int32 tensor that the front end makes of it (or None).  ``require_cuda=False`` (host-side tests only) skips the test that
    the tensors are CUDA tensors and keeps every other check, the same-device one included."""
    if q.dtype not in _DT or k.dtype != q.dtype or v.dtype != q.dtype:
        raise TypeError("q, k, v must share one dtype, float32 or bfloat16")
    if not ((q.is_cuda or not require_cuda) and q.dim() == 4 and k.dim() == 4 and k.shape == v.shape):
        raise ValueError("q [B, H, L, D] and k, v [B, Hkv, L, D] must be CUDA tensors")
    if k.device != q.device or v.device != q.device:
        raise ValueError("q, k, v must live on one device")
    B, H, L, D = q.shape
    if k.shape[0] != B or k.shape[2] != L or k.shape[3] != D or k.shape[1] < 1 or H % k.shape[1]:
        raise ValueError("k, v must be [B, Hkv, L, D] with Hkv dividing the number of query heads")
    gshape = (H, 2 * D + 1) if gate_mode else (H, 2)
    if not isinstance(gate_logits, torch.Tensor) or tuple(gate_logits.shape) != gshape:
        raise ValueError(f"gate_logits must be a tensor of shape {list(gshape)}")
    if (require_cuda and not gate_logits.is_cuda) or gate_logits.device != q.device:
        raise ValueError("gate_logits must be a CUDA tensor on q's device")
    if not gate_logits.dtype.is_floating_point:
        raise TypeError("gate_logits must be a floating-point tensor")
    if seq_lens is not None:
        if not isinstance(seq_lens, torch.Tensor) or tuple(seq_lens.shape) != (B,):
            raise ValueError("seq_lens must be None or a tensor of shape [B]")
        if seq_lens.dtype not in (torch.int32, torch.int64):
            raise TypeError("seq_lens must be int32 (int64 is converted)")
        if (require_cuda and not seq_lens.is_cuda) or seq_lens.device != q.device:
            raise ValueError("seq_lens must be a CUDA tensor on q's device")
        seq_lens = seq_lens.to(torch.int32).contiguous()
    return seq_lens


_native = _mod = None


def _module():
    """``csrc/front.cpp`` as a module; the library it links is loaded first (the same instance, and its own
    message if it is missing)."""
    global _mod
    if _mod is None:
        binding.load()
        try:
            from . import _front as m
        except ImportError as e:
            raise RuntimeError("_front.so is missing or stale: build it with "
                               "`python -m paper_2512_13368_b200.build`") from e
        _mod = m
    return _mod


def _front():
    """The native front end, loaded on first use: it validates, allocates the outputs and one scratch buffer,
    calls ``blossom_attn_fwd`` and puts a C++ node into the autograd graph that calls ``blossom_attn_bwd``."""
    global _native
    if _native is None:
        _native = _module().attention
    return _native


def blossom_attention(q, k, v, gate_logits, block_size, top_k, window, seq_lens=None, sm_scale=0.0,
                      return_indices=False, short_term="window", mask_block=1, cmp_block=0,
                      cmp_stride=0, select_per_query=False, phi_logits=None, input_dependent_gate=False, causal=True, rope_theta=0.0):
    """Gated two-branch sparse attention of q [B, H, L, D] and k, v [B, Hkv, L, D] (float32 or
    bfloat16, CUDA; Hkv divides H: with Hkv < H the query heads of a group share key/value head
    and selection, and the returned indices are [B, Hkv, M, top_k]).

    gate_logits: [H, 2] (column 0 long-term, column 1 short-term branch); seq_lens: optional int32
    [B] valid lengths of left-padded sequences; sm_scale 0 means 1/sqrt(D).  Differentiable in
    q, k, v and gate_logits.  Returns the output, and the selected block indices if asked.
    A wait that runs out inside a kernel is reported through ``binding.blossom_device_status`` of
    the call's workspace (it synchronises, so this front end does not poll it).
    short_term: "window" (keys t - window < p <= t) or "power-law" (Eq. 15: the window, blocks of
    mask_block positions at power-of-two block distances, and the last mask_block positions).
    cmp_block / cmp_stride: length and stride of overlapping compression blocks for the selection
    (Eq. 8, 11); 0 = the selection blocks themselves.
    select_per_query: one selection per query position (Eq. 13 as printed; indices [B, Hkv, L,
    top_k]) instead of one per query block.
    input_dependent_gate: Eq. 18's gate with a one-layer F_o: gate_logits is [H, 2 D + 1] = (w_lt,
    w_st, b) per head and alpha = sigmoid(<w_lt, out_lt> + <w_st, out_st> + b) per query row
    (differentiable in those parameters).
    causal: False drops the causal mask (bidirectional encoders): a query block scores every other
    live block, a query sees all valid keys of its selected blocks, Eq. 15 is symmetric.
    rope_theta: > 0 applies rotary position embedding to q and k inside the library (interleaved
    pairs, angle t * rope_theta^(-2i / D)); the gradients returned are those of the unrotated q, k.
    phi_logits: optional float32 CUDA tensor [cmp_block or block_size]: Eq. 9's learnable block
    summary as a softmax pooling over a block's positions (None = the mean).  It only steers the
    selection, which is not differentiated, so it receives no gradient here.
    """
    if phi_logits is not None:
        n = int(cmp_block) or int(block_size)
        if not (isinstance(phi_logits, torch.Tensor) and phi_logits.is_cuda and phi_logits.device == q.device
                and phi_logits.dtype == torch.float32 and tuple(phi_logits.shape) == (n,)):
            raise ValueError(f"phi_logits must be a float32 CUDA tensor of shape [{n}] on q's device")
        phi_logits = phi_logits.detach().contiguous()
    if short_term not in ("window", "power-law"):
        raise ValueError("short_term must be 'window' or 'power-law'")
    res = (_native or _front())(
        q, k, v, gate_logits, seq_lens, phi_logits, block_size, top_k, window, sm_scale,
        1 if short_term == "power-law" else 0, mask_block, cmp_block, cmp_stride, 1 if select_per_query else 0,
        1 if input_dependent_gate else 0, 1 if causal else 0, rope_theta)
    if res is None:  # not what the library can be handed: say why
        check_arguments(q, k, v, gate_logits, seq_lens, gate_mode=int(bool(input_dependent_gate)))
        raise ValueError("blossom_attention: unusable arguments")
    return res if return_indices else res[0]


# ---- the rows around the attention ---------------------------------------------------------------
def check_rows(x, p, rng, others=(), weights=(), require_cuda=True):
    """Why the native front end would not take the arguments of ``blossom_dropout`` and ``blossom_add_norm``: raises for
    what is wrong with them.  ``others``: (name, tensor or None) that must look like x; ``weights``: (name, tensor or
    None) of x's last size."""
    if not isinstance(x, torch.Tensor) or (require_cuda and not x.is_cuda) or x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("x must be a CUDA tensor with at least one column")
    if x.dtype not in _DT:
        raise TypeError("x must be float32 or bfloat16")
    for name, t in others:
        if t is None:
            continue
        if not isinstance(t, torch.Tensor) or t.shape != x.shape or t.device != x.device:
            raise ValueError(f"{name} must be a tensor of x's shape on x's device")
        if t.dtype != x.dtype:
            raise TypeError(f"{name} must have x's dtype")
    kinds = set()
    for name, t in weights:
        if t is None:
            continue
        if not isinstance(t, torch.Tensor) or tuple(t.shape) != (x.shape[-1],) or t.device != x.device:
            raise ValueError(f"{name} must be a tensor of shape [{x.shape[-1]}] on x's device")
        kinds.add(t.dtype)
    if len(kinds) > 1 or any(k not in _DT for k in kinds):
        raise TypeError(" and ".join(n for n, _ in weights) + " must share one dtype, float32 or bfloat16")
    if p:
        if not (isinstance(rng, torch.Tensor) and rng.dtype == torch.int64 and tuple(rng.shape) == (2,)
                and rng.device == x.device):
            raise ValueError("rng must be an int64 tensor (seed, step) of shape [2] on x's device")


def blossom_dropout(x, p, rng, site=0):
    """Dropout of x [..., C] (float32 or bfloat16, CUDA) with probability p in [0, 1] (in steps of 1 / 65536: the kept
    elements are scaled by the inverse of the probability in use), from a counter-based generator: which elements are
    kept is a function of ``rng``, ``site`` and the element's place, evaluated again in the backward and never stored.

    rng: int64 CUDA tensor (seed, step).  The caller moves the step on between training steps (``rng[1] += 1``: after the
    backward, which reads it again; autograd notices a change in between); it is read on the device, so a captured
    graph draws anew on every replay.  site: 0 .. 65535, another one for every dropout of a step."""
    p = float(p)
    if p == 0.0:
        check_rows(x, p, rng)
        return x
    res = _module().dropout(x, p, rng, site)
    if res is None:
        check_rows(x, p, rng)
        raise ValueError("blossom_dropout: unusable arguments")
    return res


def blossom_add_norm(x, residual, weight, bias, p=0.0, rng=None, site=0, eps=1e-5):
    """LayerNorm(residual + dropout(x)) over the last dimension of x [..., C], C up to 8192 (float32 or bfloat16, CUDA): the
    end of a post-norm sub-layer (Eq. 20-22) in one pass.

    residual: like x, or None.  weight, bias: [C] float32 or bfloat16, either may be None.  p, rng, site: as for
    ``blossom_dropout`` (p = 0: no dropout, rng may be None).  Differentiable in x, residual, weight and bias."""
    res = _module().add_norm(x, residual, weight, bias, p, rng, site, eps)
    if res is None:
        check_rows(x, p, rng, (("residual", residual),), (("weight", weight), ("bias", bias)))
        raise ValueError("blossom_add_norm: unusable arguments")
    return res


# ---- the loss ------------------------------------------------------------------------------------
def check_loss(hidden, table, targets, negatives, require_cuda=True):
    """Why the native front end would not take the arguments of ``blossom_sampled_loss``: raises for what is wrong."""
    if not isinstance(hidden, torch.Tensor) or (require_cuda and not hidden.is_cuda) or hidden.dim() < 1 or hidden.shape[-1] < 1:
        raise ValueError("hidden must be a CUDA tensor [..., C]")
    if hidden.dtype not in _DT:
        raise TypeError("hidden must be float32 or bfloat16")
    if not isinstance(table, torch.Tensor) or table.dim() != 2 or table.shape[1] != hidden.shape[-1] or table.shape[0] < 1:
        raise ValueError(f"table must be [items, {hidden.shape[-1]}]")
    if table.dtype != hidden.dtype:
        raise TypeError("table must have hidden's dtype")
    if not isinstance(targets, torch.Tensor) or targets.shape != hidden.shape[:-1]:
        raise ValueError(f"targets must be a tensor of shape {list(hidden.shape[:-1])}")
    if not isinstance(negatives, torch.Tensor) or negatives.dim() < 1 or (
            negatives.dim() > 1 and negatives.shape[:-1] != hidden.shape[:-1]):
        raise ValueError(f"negatives must be a tensor of shape [n] or {list(hidden.shape[:-1])} + [n]")
    if targets.dtype not in (torch.int32, torch.int64) or negatives.dtype != targets.dtype:
        raise TypeError("targets and negatives must both be int64 or both int32")
    if any(t.device != hidden.device for t in (table, targets, negatives)):
        raise ValueError("hidden, table, targets and negatives must live on one device")


def blossom_sampled_loss(hidden, table, targets, negatives, ignore_index=-100, mask_hits=False):
    """Sampled softmax cross-entropy over an item table: the mean, over the positions that take part, of
    ``logsumexp(logits) - logits[target]`` with the logits ``<hidden, table[c]>`` of the target and the negatives.

    hidden [..., C] and table [items, C]: float32 or bfloat16 (CUDA), C up to 1024; targets [...]: int32 or int64, a position
    whose target is ``ignore_index`` or no item takes no part; negatives [..., n], or [n] for all positions alike (n < 2^24): ids
    that are no items are no candidates, and with ``mask_hits`` those equal to the position's target are none.
    Returns a float32 scalar (0 if no position takes part), differentiable in hidden and table."""
    res = _module().sampled_loss(hidden, table, targets, negatives, ignore_index, mask_hits)
    if res is None:
        check_loss(hidden, table, targets, negatives)
        raise ValueError("blossom_sampled_loss: unusable arguments")
    return res


# ---- embedding -------------------------------------------------------------------------------------
def check_embedding(ids, table, require_cuda=True):
    """Why the native front end would not take the arguments of ``blossom_embedding``: raises for what is wrong with them."""
    if not isinstance(table, torch.Tensor) or (require_cuda and not table.is_cuda) or table.dim() != 2 or min(table.shape) < 1:
        raise ValueError("table must be a CUDA tensor [items, C]")
    if table.dtype not in _DT:
        raise TypeError("table must be float32 or bfloat16")
    if not isinstance(ids, torch.Tensor) or ids.device != table.device:
        raise ValueError("ids must be a tensor on table's device")
    if ids.dtype not in (torch.int32, torch.int64):
        raise TypeError("ids must be int64 or int32")


def blossom_embedding(ids, table, scale=1.0, padding_idx=None):
    """``scale * table[ids]`` for ids [...] (int64 or int32) and table [items, C] (float32 or bfloat16, CUDA; C up to 8192):
    [..., C], differentiable in table (the gradient is dense, a sum per item in a fixed order).

    padding_idx: the item that gets no gradient (its row is looked up like any other); a negative number is no item.  An id that is no
    item gives zeros and no gradient."""
    res = _module().embedding(ids, table, scale, -1 if padding_idx is None else padding_idx)
    if res is None:
        check_embedding(ids, table)
        raise ValueError("blossom_embedding: unusable arguments")
    return res


# ---- linear layer ----------------------------------------------------------------------------------
def check_linear(x, weight, bias, residual, require_cuda=True):
    """Why the native front end would not take the arguments of ``blossom_linear``: raises for what is wrong with them."""
    if not isinstance(x, torch.Tensor) or (require_cuda and not x.is_cuda) or x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("x must be a CUDA tensor with at least one column")
    if x.dtype not in _DT:
        raise TypeError("x must be float32 or bfloat16")
    if not isinstance(weight, torch.Tensor) or weight.dim() != 2 or weight.shape[1] != x.shape[-1] or weight.shape[0] < 1:
        raise ValueError(f"weight must be [outs, {x.shape[-1]}]")
    outs = weight.shape[0]
    if bias is not None and (not isinstance(bias, torch.Tensor) or tuple(bias.shape) != (outs,)):
        raise ValueError(f"bias must be None or a tensor of shape [{outs}]")
    if residual is not None and (not isinstance(residual, torch.Tensor) or residual.shape != x.shape[:-1] + (outs,)):
        raise ValueError(f"residual must be None or a tensor of shape {list(x.shape[:-1]) + [outs]}")
    for name, t in (("weight", weight), ("bias", bias), ("residual", residual)):
        if t is not None and t.dtype != x.dtype:
            raise TypeError(f"{name} must have x's dtype")
        if t is not None and t.device != x.device:
            raise ValueError(f"{name} must live on x's device")


def blossom_linear(x, weight, bias=None, residual=None, activation="none", packed=False):
    """``act(x W^T + bias) + residual`` in one pass for x [..., K] and weight [N, K] as ``nn.Linear`` has it (float32 or
    bfloat16, CUDA, all of one type; K and N up to 65536): [..., N], differentiable in x, weight, bias and residual.

    bias: [N] or None.  residual: [..., N] or None.  activation: "none", "relu", "gelu" (x Phi(x), the one with the error
    function, to single precision, of bf16 results to 2^-10) or "silu"; its argument is not kept, the backward forms it again from x.
    packed: keep x for the backward in 8 bits, a power of two per 32 columns (33/32 bytes an element; K up to 8192): the
    weight's gradient and the activation's argument in the backward are those of the rounded x.  The output is not
    affected, nor is the gradient of x without an activation.
    A wait that runs out inside a kernel is reported through ``binding.blossom_device_status`` of the call's workspace,
    which this front end does not poll."""
    kind = binding.ACTIVATIONS.get(activation)
    if kind is None:
        raise ValueError(f"activation must be one of {', '.join(binding.ACTIVATIONS)}")
    res = _module().linear(x, weight, bias, residual, kind, 1 if packed else 0)
    if res is None:
        check_linear(x, weight, bias, residual)
        raise ValueError("blossom_linear: unusable arguments")
    return res
