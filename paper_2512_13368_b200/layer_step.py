"""The end-to-end layer case: a 2-layer SASRec-style causal encoder whose self-attention is the
library's gated sparse attention, trained one step on synthetic item sequences.

This module is a measurement harness around the op (PyTorch supplies embeddings, projections,
LayerNorm, the feed-forward block, the loss and autograd; the attention itself runs in the CUDA
library through ``autograd.blossom_attention``).  It exists to time the attention's share of a
full forward + backward step, not to train a recommender.  With ``native`` the rows around the attention
run in the library too: dropout of the embeddings, residual + dropout + LayerNorm (Eq. 20-22) and the loss
(``autograd.blossom_dropout``, ``blossom_add_norm``, ``blossom_sampled_loss``); with ``products`` the item embedding,
the projections and the feed-forward block as well (Eq. 6, 7; ``blossom_embedding``, ``blossom_linear`` with GELU behind the
first product), and with ``packed`` the feed-forward block keeps its inputs for the backward in 8 bits.

Shapes of the layer case: hidden 64, 2 heads (head dim 32), feed-forward 256 with GELU, post-LN,
dropout off (``dropout`` turns it on), item table 50,000 x 64 in bf16, batch 128 x sequence 1024 of item ids drawn from a
Zipf(1.1) law, next-item cross-entropy over 1 positive + 127 uniform negatives per position;
rotary position encoding on q and k; attention hyper-parameters of the mid-length case
(block 32, top-k 8, window 64) since the layer case names none.
"""
from __future__ import annotations

import numpy as np
import torch
import torch.nn as nn
import torch.nn.functional as F

from . import binding
from .autograd import (blossom_add_norm, blossom_attention, blossom_dropout, blossom_embedding, blossom_linear,
                       blossom_sampled_loss)


def zipf_ids(batch, seq_len, n_items, s=1.1, seed=1):
    """[batch, seq_len + 1] int64 item ids in [1, n_items], rank r drawn with weight r^-s."""
    rng = np.random.default_rng(seed)
    w = np.arange(1, n_items + 1, dtype=np.float64) ** (-s)
    return torch.from_numpy(rng.choice(n_items, size=(batch, seq_len + 1), p=w / w.sum()) + 1)


def rope(x):
    """Rotary position encoding of [B, H, L, D] (pairs (2i, 2i+1), base 10000)."""
    B, H, L, D = x.shape
    pos = torch.arange(L, device=x.device, dtype=torch.float32)
    inv = 10000.0 ** (-torch.arange(0, D, 2, device=x.device, dtype=torch.float32) / D)
    ang = pos[:, None] * inv[None, :]
    cos, sin = ang.cos().to(x.dtype), ang.sin().to(x.dtype)
    x0, x1 = x[..., 0::2], x[..., 1::2]
    return torch.stack((x0 * cos - x1 * sin, x0 * sin + x1 * cos), dim=-1).flatten(-2)


class BlossomLayer(nn.Module):
    """site: the first of the two numbers that tell this layer's dropouts from the others'."""

    def __init__(self, hidden, heads, ffn, block, topk, window, native=False, dropout=0.0, site=1, products=False,
                 packed=False):
        super().__init__()
        self.products, self.packed = products, packed
        self.heads, self.block, self.topk, self.window = heads, block, topk, window
        self.native, self.dropout, self.site = native, dropout, site
        self.qkv = nn.Linear(hidden, 3 * hidden)
        self.proj = nn.Linear(hidden, hidden)
        self.gate_logits = nn.Parameter(torch.zeros(heads, 2))
        self.ln1, self.ln2 = nn.LayerNorm(hidden), nn.LayerNorm(hidden)
        self.ff1, self.ff2 = nn.Linear(hidden, ffn), nn.Linear(ffn, hidden)

    def add_norm(self, x, sub, norm, rng, site):
        """norm(x + dropout(sub))"""
        p = self.dropout if self.training else 0.0
        if self.native:
            return blossom_add_norm(sub, x, norm.weight, norm.bias, p=p, rng=rng, site=site, eps=norm.eps)
        return norm(x + F.dropout(sub, p, self.training))

    def linear(self, x, layer, activation="none", packed=False):
        """activation(layer(x))"""
        if self.products:
            return blossom_linear(x, layer.weight, layer.bias, activation=activation, packed=packed)
        return F.gelu(layer(x)) if activation == "gelu" else layer(x)

    def forward(self, x, rng=None):
        B, L, C = x.shape
        q, k, v = self.linear(x, self.qkv).view(B, L, 3, self.heads, C // self.heads).permute(2, 0, 3, 1, 4)
        q, k, v = rope(q).contiguous(), rope(k).contiguous(), v.contiguous()
        a = blossom_attention(q, k, v, self.gate_logits, self.block, self.topk, self.window)
        x = self.add_norm(x, self.linear(a.transpose(1, 2).reshape(B, L, C), self.proj), self.ln1, rng, self.site)
        y = self.linear(self.linear(x, self.ff1, "gelu", self.packed), self.ff2, packed=self.packed)
        return self.add_norm(x, y, self.ln2, rng, self.site + 1)


class BlossomEncoder(nn.Module):
    """native: dropout, residual + LayerNorm and the loss in the library as well.  Its dropouts are a function of
    ``rng`` = (seed, step): call ``next_step`` after each backward.  products: the embedding and the linear layers in the
    library; packed: of these, the feed-forward block's keep their inputs in 8 bits."""

    def __init__(self, n_items=50000, hidden=64, heads=2, ffn=256, layers=2, block=32, topk=8, window=64, native=False,
                 dropout=0.0, seed=0, products=False, packed=False):
        super().__init__()
        if packed and not products:
            raise ValueError("packed: only the library's linear layers (products) keep their inputs in 8 bits")
        self.native, self.dropout, self.products = native, dropout, products
        self.emb = nn.Embedding(n_items + 1, hidden, padding_idx=0)
        nn.init.normal_(self.emb.weight, std=0.02)
        self.layers = nn.ModuleList(BlossomLayer(hidden, heads, ffn, block, topk, window, native, dropout, 1 + 2 * i, products, packed)
                                    for i in range(layers))
        if native:
            self.register_buffer("rng", torch.tensor([seed, 0], dtype=torch.int64))

    def next_step(self):
        """Other dropouts from here on (on the device: a captured step draws anew each time it is replayed)."""
        if self.native:
            self.rng[1] += 1

    def forward(self, ids):
        x = blossom_embedding(ids, self.emb.weight, padding_idx=0) if self.products else self.emb(ids)
        rng = self.rng if self.native else None
        if self.dropout and self.training:
            x = blossom_dropout(x, self.dropout, rng, site=0) if self.native else F.dropout(x, self.dropout)
        for layer in self.layers:
            x = layer(x, rng)
        return x

    def loss(self, ids, targets, negatives):
        """Sampled softmax: the positive against `negatives` [B, L, N] uniform item ids (none of them 0, the
        padding).  With ``native`` positions whose target is 0 take no part."""
        h = self.forward(ids)                                        # [B, L, C]
        if self.native:
            return blossom_sampled_loss(h, self.emb.weight, targets, negatives, ignore_index=0)
        cand = torch.cat((targets[..., None], negatives), dim=-1)   # [B, L, 1 + N]
        logits = (h[:, :, None, :] * self.emb(cand)).sum(-1).float()
        return F.cross_entropy(logits.flatten(0, 1), torch.zeros(logits.shape[0] * logits.shape[1],
                                                                 dtype=torch.long, device=ids.device))


def attention_share(batch=128, seq_len=1024, n_items=50000, negatives=127, steps=5, warmup=2,
                    device="cuda:0", seed=1, native=False, dropout=0.0, products=False, packed=False):
    """Times full forward + backward steps of the layer case and the library kernels inside them.

    Returns a dict: ms per step, ms of the library's attention kernels per step (summed device times from
    the per-launch event profile), their share, the same sum for its other kernels (0 without ``native`` and
    ``products``), the memory that a forward keeps for its backward, the most that is in use during that beside
    the model (its gradients included), and the loss of the last step.
    """
    torch.manual_seed(seed)
    dev = torch.device(device)
    model = BlossomEncoder(n_items=n_items, native=native, dropout=dropout, seed=seed, products=products, packed=packed).to(dev).to(torch.bfloat16)
    seq = zipf_ids(batch, seq_len, n_items, seed=seed).to(dev)
    ids, targets = seq[:, :-1], seq[:, 1:]
    g = torch.Generator(device="cpu").manual_seed(seed)
    neg = torch.randint(1, n_items + 1, (batch, seq_len, negatives), generator=g).to(dev)

    def step():
        model.zero_grad(set_to_none=True)
        loss = model.loss(ids, targets, neg)
        loss.backward()
        model.next_step()
        return loss

    for _ in range(warmup):
        step()
    torch.cuda.synchronize(dev)
    model.zero_grad(set_to_none=True)
    before = torch.cuda.memory_allocated(dev)
    loss = model.loss(ids, targets, neg)
    kept = torch.cuda.memory_allocated(dev) - before
    torch.cuda.reset_peak_memory_stats(dev)
    loss.backward()
    peak = torch.cuda.max_memory_allocated(dev) - before
    del loss
    torch.cuda.synchronize(dev)
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    binding.blossom_profile_start(128 * steps)
    e0.record()
    for _ in range(steps):
        loss = step()
    e1.record()
    torch.cuda.synchronize(dev)
    launches = binding.blossom_profile_stop(128 * steps)
    total = e0.elapsed_time(e1) / steps
    around = ("dropout", "norm_", "loss_", "embed_", "pack_", "unpack_", "linear_")
    ours = sum(ms for name, ms in launches if not name.startswith(around)) / steps
    others = sum(ms for name, ms in launches if name.startswith(around)) / steps
    return {"ms_per_step": total, "attention_ms_per_step": ours, "attention_share": ours / total,
            "rows_and_loss_ms_per_step": others, "library_launches_per_step": len(launches) / steps,
            "kept_mb": kept / 1e6, "peak_mb": peak / 1e6, "loss": float(loss.detach())}


if __name__ == "__main__":
    import argparse
    import json
    args = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    args.add_argument("--native", action="store_true", help="dropout, residual + LayerNorm and loss in the library")
    args.add_argument("--dropout", type=float, default=0.0)
    args.add_argument("--products", action="store_true", help="embedding and linear layers in the library")
    args.add_argument("--packed", action="store_true", help="with --products: the feed-forward block's inputs kept in 8 bits")
    opts = args.parse_args()
    if opts.packed and not opts.products:
        args.error("--packed goes with --products")
    binding.load()
    print(json.dumps(attention_share(native=opts.native, dropout=opts.dropout, products=opts.products, packed=opts.packed)))
