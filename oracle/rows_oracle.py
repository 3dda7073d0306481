"""Double-precision definitions of the operators around the attention, in numpy: dropout from a counter-based
generator, layer norm of residual + dropout(x), the sampled softmax loss; forward and backward.  Shares
no code with the CUDA library."""
from __future__ import annotations

import math

import numpy as np

_M32 = (1 << 32) - 1


def philox4x32(counter, key, rounds=10):
    """Philox 4x32 (Salmon et al. 2011) of counter words (c0, c1, c2, c3), uint64 arrays that hold 32-bit values, under
    the key (k0, k1); returns four such arrays."""
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k = [int(key[0]), int(key[1])]
    for _ in range(rounds):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        hi0, lo0 = p0 >> np.uint64(32), p0 & np.uint64(_M32)
        hi1, lo1 = p1 >> np.uint64(32), p1 & np.uint64(_M32)
        c = [hi1 ^ c[1] ^ np.uint64(k[0]), lo1, hi0 ^ c[3] ^ np.uint64(k[1]), lo0]
        k = [(k[0] + 0x9E3779B9) & _M32, (k[1] + 0xBB67AE85) & _M32]
    return c


def bar(p):
    return int(math.floor(p * 65536.0 + 0.5))


def keep_factor(rows, cols, p, seed, step, site):
    """[rows, cols] float64: 0 where an element is dropped, else the scale of the kept ones."""
    if p == 0.0:
        return np.ones((rows, cols))
    seed, step = int(seed) & ((1 << 64) - 1), int(step) & ((1 << 64) - 1)
    groups = (cols + 7) // 8
    r, g = np.meshgrid(np.arange(rows, dtype=np.uint64), np.arange(groups, dtype=np.uint64), indexing="ij")
    w = philox4x32((g + np.uint64(65536 * site), r, np.full_like(r, step & _M32), np.full_like(r, step >> 32)),
                   (seed & _M32, seed >> 32))
    bits = np.stack([h for x in w for h in (x & np.uint64(0xFFFF), x >> np.uint64(16))], axis=-1)
    bits = bits.reshape(rows, groups * 8)[:, :cols].astype(np.int64)
    t = bar(p)
    return np.where(bits >= t, 65536.0 / (65536 - t) if t < 65536 else 0.0, 0.0)


def add_norm(x, residual, weight, bias, factor, eps):
    """Rows of x, float64; factor from ``keep_factor``.  Returns a dict: out, and what the backward needs."""
    x = np.asarray(x, dtype=np.float64)
    z = np.where(factor == 0.0, 0.0, x * factor)
    if residual is not None:
        z = z + residual
    mean = z.mean(axis=1, keepdims=True)
    rstd = 1.0 / np.sqrt(((z - mean) ** 2).mean(axis=1, keepdims=True) + eps)
    n = (z - mean) * rstd
    w = np.ones(x.shape[1]) if weight is None else np.asarray(weight, dtype=np.float64)
    b = np.zeros(x.shape[1]) if bias is None else np.asarray(bias, dtype=np.float64)
    return {"out": n * w + b, "z": z, "n": n, "mean": mean, "rstd": rstd, "w": w, "factor": factor}


def add_norm_backward(f, dout):
    """Gradients of sum(out * dout) with f as ``add_norm`` returned it."""
    a = dout * f["w"]
    dz = f["rstd"] * (a - a.mean(axis=1, keepdims=True) - f["n"] * (a * f["n"]).mean(axis=1, keepdims=True))
    return {"dx": dz * f["factor"], "dresidual": dz, "dweight": (dout * f["n"]).sum(axis=0), "dbias": dout.sum(axis=0)}


def sampled_loss(hidden, table, targets, negatives, ignore_index=-100, mask_hits=False):
    """Mean over the rows that take part of logsumexp(logits) - target logit, and its gradients; row by row from the
    definition.  negatives: [rows, n] or [n].  Returns a dict: loss, lse [rows], count, dhidden, dtable."""
    hidden, table = np.asarray(hidden, dtype=np.float64), np.asarray(table, dtype=np.float64)
    rows, items = hidden.shape[0], table.shape[0]
    negatives = np.broadcast_to(np.asarray(negatives), (rows, np.shape(negatives)[-1]))
    part = [t for t in range(rows) if 0 <= targets[t] < items and targets[t] != ignore_index]
    res = {"loss": 0.0, "lse": np.zeros(rows), "count": len(part), "dhidden": np.zeros_like(hidden),
           "dtable": np.zeros_like(table)}
    for t in part:
        c = [int(targets[t])] + [int(i) for i in negatives[t]
                                 if 0 <= i < items and not (mask_hits and i == targets[t])]
        l = table[c] @ hidden[t]
        top = l.max()
        e = np.exp(l - top)
        res["lse"][t] = top + math.log(e.sum())
        res["loss"] += (res["lse"][t] - l[0]) / len(part)
        coef = e / e.sum()
        coef[0] -= 1.0
        coef /= len(part)
        res["dhidden"][t] = coef @ table[c]
        np.add.at(res["dtable"], c, coef[:, None] * hidden[t][None, :])
    return res
