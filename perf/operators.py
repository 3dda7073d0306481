"""The operators around the attention of a training step, as plain cases that can be prepared, run and timed.

Three operators: ``dropout`` from a counter-based generator, ``norm`` (layer norm of residual +
dropout(x), the sub-layer ending of a post-norm encoder) and ``loss`` (sampled softmax: one positive
and n negative items per position, scored against the embedding table).  Sizes are those of the
layer case (``layer_step.py``: 128 x 1024 positions, hidden 64, 50,000 items, 127 negatives), of the
short-history configuration (256 x 200 positions), of the paper's data sets (3.7 k to 165 k items) and
their neighbourhood: from one position of one user to a whole training batch, hidden sizes
that are no multiple of anything.

With ``own`` false every operator is computed in its plain form, elementary torch operations in 32
bits; with ``own`` true by the library, through the autograd front end (``entry`` "autograd") or
through the C ABI with the caller's own buffers (``entry`` "abi").
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _norm(**kw):
    # pad: elements between the end of a row of x and the next row (a slice of a wider buffer)
    return dict(dict(op="norm", entry="autograd", train=True, dtype="bf16", rows=1, cols=64, p=0.0, residual=True,
                     pad=0, eps=1e-5, site=1), **kw)


def _dropout(**kw):
    return dict(dict(op="dropout", entry="autograd", train=True, dtype="bf16", rows=1, cols=64, p=0.2, pad=0, site=0),
                **kw)


def _loss(**kw):
    # ignored: share of the positions without a target (padding); zipf: exponent of the targets' popularity;
    # shared: all positions have the same negatives
    return dict(dict(op="loss", entry="autograd", train=True, dtype="bf16", rows=64, cols=64, items=50001, n=127,
                     ignored=0.0, zipf=1.1, shared=False, hits=False), **kw)


def listed():
    return [
        # the last position of one user, evaluated inside a PyTorch program: latency alone
        _norm(name="norm-serve-one", train=False, rows=1),
        # a serving batch of short histories; the runtime keeps its buffers
        _norm(name="norm-serve-batch", entry="abi", train=False, rows=64 * 200),
        # the layer case: 128 x 1024 positions, hidden 64
        _norm(name="norm-train-layer", rows=128 * 1024, p=0.2),
        # short histories with the hidden size of small recommenders, single precision: rows of 200 bytes
        _norm(name="norm-train-odd-fp32", dtype="fp32", rows=128 * 200 - 3, cols=50, p=0.5),
        # a wide encoder
        _norm(name="norm-train-wide", entry="abi", rows=32 * 1024, cols=1024, p=0.1),
        # embeddings of the layer case
        _dropout(name="dropout-train-layer", rows=128 * 1024),
        # embeddings cut out of a wider buffer, an odd size
        _dropout(name="dropout-train-odd-fp32", dtype="fp32", rows=128 * 200 - 3, cols=50, p=0.5, pad=14),
        # evaluation: one position of each of 64 users against 100 sampled items
        _loss(name="loss-eval", train=False, rows=64, n=100),
        # short histories, left-padded, a small catalogue
        _loss(name="loss-train-short", rows=256 * 200, items=3707, n=31, ignored=0.45),
        # single precision, an odd hidden size, negatives shared by the batch
        _loss(name="loss-train-odd-fp32", dtype="fp32", rows=64 * 200 - 5, cols=50, items=12102, n=99, shared=True,
              hits=True),
        # the layer case with the caller's own buffers, and through autograd with a large catalogue
        _loss(name="loss-train-layer", entry="abi", rows=128 * 1024),
        _loss(name="loss-train-large-catalogue", rows=32 * 1024, items=165001, n=127, cols=128),
    ]


# ---- drawn cases: the families above over their ranges ---------------------------------------
def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "dropout", "loss", "loss"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    entry = rng.choice(["autograd", "abi"])
    cols = _log_int(rng, 16, 1024 if kind != "loss" else 256)
    if rng.random() < 0.6:
        cols = (cols + 15) // 16 * 16
    if kind == "loss":
        c = _loss(cols=cols, n=_log_int(rng, 1, 255), items=_log_int(rng, 1000, 165001))
        # no more than a third of the layer case's gathered elements
        most = 128 * 1024 * 128 * 64 // 3 // (cols * (c["n"] + 1))
        c["rows"] = _log_int(rng, 16, max(16, min(most, 128 * 1024)))
        c["ignored"] = rng.choice([0.0, 0.3, 0.6])
        c["zipf"] = rng.choice([0.0, 1.1])
        c["shared"] = rng.random() < 0.2
        c["hits"] = rng.random() < 0.3
    else:
        c = _norm() if kind == "norm" else _dropout()
        c["cols"] = cols
        c["rows"] = _log_int(rng, 1, min(128 * 1024, 32 * 1024 * 1024 // cols))
        c["p"] = rng.choice([0.1, 0.2, 0.5]) if kind == "dropout" or rng.random() < 0.7 else 0.0
        c["pad"] = rng.choice([0, 0, 16, 14])
        if kind == "norm":
            c["residual"] = rng.random() < 0.85
    c["train"] = rng.random() < 0.8
    c["dtype"], c["entry"] = dtype, entry
    return c


# ---- inputs ------------------------------------------------------------------------------------
class _State:
    pass


def _zipf(items, s, shape, g, dev):
    """Ids in [1, items), rank r drawn with weight r^-s."""
    cdf = torch.cumsum(torch.arange(1, items, dtype=torch.float64, device=dev) ** -s, 0)
    u = torch.rand(shape, generator=g, device=dev, dtype=torch.float64) * cdf[-1]
    return torch.searchsorted(cdf, u).clamp_(max=items - 2) + 1


def prepare(case, seed):
    s = _State()
    s.case = c = case
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed) % (1 << 62))
    dt = _TYPES[c["dtype"]]
    R, C = c["rows"], c["cols"]

    def normal(shape, std=1.0, mean=0.0):
        return torch.randn(shape, generator=g, device=dev) * std + mean

    if c["op"] == "loss":
        s.hidden = normal((R, C)).to(dt)             # rows behind a layer norm
        s.table = normal((c["items"], C), 0.1).to(dt)
        s.targets = _zipf(c["items"], c["zipf"], (R,), g, dev)
        if c["ignored"]:
            s.targets[torch.rand((R,), generator=g, device=dev) < c["ignored"]] = -100
        s.negatives = torch.randint(1, c["items"], (1 if c["shared"] else R, c["n"]), generator=g, device=dev)
        s.negatives = s.negatives.expand(R, c["n"])
        s.grad = torch.ones((), device=dev)
    else:
        s.x = normal((R, C + c["pad"])).to(dt)[:, :C]
        s.rng = torch.tensor([int(seed) % (1 << 62) * 2 + 1, int(seed) % 100003], device=dev) if c["p"] else None
        if c["op"] == "norm":
            s.residual = normal((R, C)).to(dt) if c["residual"] else None
            s.weight = normal((C,), 0.2, 1.0).to(dt)
            s.bias = normal((C,), 0.2).to(dt)
        if c["train"]:
            s.dout = normal((R, C)).to(dt)
    if own:
        _prepare_own(s, c, dev, dt)
    return s


def _prepare_own(s, c, dev, dt):
    """What a program keeps from one call to the next: leaves that want gradients, or buffers of its own."""
    if c["entry"] == "autograd":
        if c["train"]:
            for name in ("x", "residual", "weight", "bias", "hidden", "table"):
                t = getattr(s, name, None)
                if t is not None:
                    t.requires_grad_(True)
        return
    from paper_2512_13368_b200 import binding
    R, C = c["rows"], c["cols"]
    f32 = dict(dtype=torch.float32, device=dev)

    def scratch(nbytes):
        return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=dev)

    if c["op"] == "loss":
        s.params = binding.make_loss_params(R, C, c["items"], c["n"], c["dtype"], mask_hits=int(c["hits"]),
                                            negatives_stride=0 if c["shared"] else c["n"])
        s.workspace = scratch(binding.blossom_sampled_loss_workspace_bytes(s.params))
        s.loss, s.lse = torch.empty((), **f32), torch.empty(R + 1, **f32)
        s.grad_hidden = None
        if c["train"]:
            s.grad_hidden = torch.empty((R, C), **f32)
            s.dhidden, s.dtable = torch.empty_like(s.hidden), torch.empty_like(s.table)
        return
    s.params = binding.make_rows_params(R, C, c["dtype"], dropout=c["p"], site=c["site"], eps=c.get("eps", 0.0),
                                        x_stride=C + c["pad"])
    s.out = torch.empty((R, C), dtype=dt, device=dev)
    if c["op"] == "dropout":
        s.params_bwd = binding.make_rows_params(R, C, c["dtype"], dropout=c["p"], site=c["site"])
        s.dx = torch.empty((R, C), dtype=dt, device=dev)
        return
    s.stats = None
    if c["train"]:
        s.stats = torch.empty((R, 2), **f32)
        s.dx = torch.empty((R, C), dtype=dt, device=dev)
        # (without dropout one buffer is the gradient of both)
        s.dresidual = torch.empty_like(s.dx) if c["residual"] and c["p"] else None
        s.dweight, s.dbias = torch.empty_like(s.weight), torch.empty_like(s.bias)
        s.workspace = scratch(binding.blossom_add_norm_workspace_bytes(s.params))


# ---- the plain forms -----------------------------------------------------------------------------
_LOW = 0xFFFFFFFF


def _keep(rows, cols, p, rng, site):
    """(kept [rows, cols], scale): ten rounds of Philox 4x32, a counter per row and eight columns."""
    dev = rng.device
    groups = (cols + 7) // 8
    seed, step = rng[0], rng[1]
    c0 = (torch.arange(groups, device=dev) + (site << 16))[None, :].expand(rows, groups)
    c1 = torch.arange(rows, device=dev)[:, None].expand(rows, groups)
    c2 = (step & _LOW).expand(rows, groups)
    c3 = ((step >> 32) & _LOW).expand(rows, groups)
    k0, k1 = seed & _LOW, (seed >> 32) & _LOW
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # (64-bit products wrap; the masks below take their halves)
        c0, c1, c2, c3 = ((b >> 32) & _LOW) ^ c1 ^ k0, b & _LOW, ((a >> 32) & _LOW) ^ c3 ^ k1, a & _LOW
        k0, k1 = (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW
    words = torch.stack((c0, c1, c2, c3), dim=-1)
    bits = torch.stack((words & 0xFFFF, words >> 16), dim=-1).reshape(rows, groups * 8)[:, :cols]
    bar = math.floor(p * 65536 + 0.5)
    return bits >= bar, 65536.0 / (65536 - bar) if bar < 65536 else 0.0


def _drop(x, keep, scale):
    return torch.where(keep, x * scale, torch.zeros((), device=x.device))


def _plain_dropout(s, c):
    keep, scale = _keep(c["rows"], c["cols"], c["p"], s.rng, c["site"])
    res = {"out": _drop(s.x.float(), keep, scale).to(s.x.dtype)}
    if c["train"]:
        res["dx"] = _drop(s.dout.float(), keep, scale).to(s.x.dtype)
    return res


def _plain_norm(s, c):
    dt = s.x.dtype
    z = s.x.float()
    if c["p"]:
        keep, scale = _keep(c["rows"], c["cols"], c["p"], s.rng, c["site"])
        z = _drop(z, keep, scale)
    if c["residual"]:
        z = z + s.residual.float()
    w = s.weight.float()
    centred = z - z.mean(-1, keepdim=True)
    rstd = 1.0 / torch.sqrt((centred * centred).mean(-1, keepdim=True) + c["eps"])
    xh = centred * rstd
    res = {"out": (xh * w + s.bias.float()).to(dt)}
    if not c["train"]:
        return res
    dout = s.dout.float()
    a = dout * w
    dz = rstd * (a - a.mean(-1, keepdim=True) - xh * (a * xh).mean(-1, keepdim=True))
    res["dx"] = (_drop(dz, keep, scale) if c["p"] else dz).to(dt)
    if c["residual"]:
        res["dresidual"] = dz.to(dt)
    res["dweight"] = (dout * xh).sum(0).to(dt)
    res["dbias"] = dout.sum(0).to(dt)
    return res


def _plain_loss(s, c):
    h, table = s.hidden.float(), s.table.float()
    live = s.targets >= 0
    target = torch.where(live, s.targets, torch.zeros_like(s.targets))
    cand = torch.cat((target[:, None], s.negatives), dim=1)
    rows = table[cand]
    logits = (rows * h[:, None, :]).sum(-1)
    if c["hits"]:
        hit = cand == target[:, None]
        hit[:, 0] = False
        logits = torch.where(hit, torch.full_like(logits, -math.inf), logits)
    top = logits.max(-1, keepdim=True).values
    e = torch.exp(logits - top)
    total = e.sum(-1, keepdim=True)
    each = torch.log(total[:, 0]) + top[:, 0] - logits[:, 0]
    count = live.sum().clamp(min=1)
    loss = torch.where(live, each, torch.zeros_like(each)).sum() / count
    if not c["train"]:
        return {"loss": loss}
    coef = e / total
    coef[:, 0] -= 1.0
    coef = coef * (live[:, None] * (s.grad / count))
    dh = (coef[:, :, None] * rows).sum(1)
    del rows
    dtable = torch.zeros_like(table)
    dtable.index_add_(0, cand.reshape(-1), (coef[:, :, None] * h[:, None, :]).reshape(-1, c["cols"]))
    return {"loss": loss, "dhidden": dh.to(s.hidden.dtype), "dtable": dtable.to(s.table.dtype)}


# ---- the library's calls ---------------------------------------------------------------------------
def _own_abi(s, c):
    from paper_2512_13368_b200 import binding
    if c["op"] == "loss":
        binding.blossom_sampled_loss_fwd(s.params, s.hidden, s.table, s.targets, s.negatives, s.loss, s.lse,
                                         s.grad_hidden, s.workspace)
        if not c["train"]:
            return {"loss": s.loss}
        binding.blossom_sampled_loss_bwd(s.params, s.hidden, s.table, s.targets, s.negatives, s.lse, s.grad_hidden,
                                         s.grad, s.dhidden, s.dtable, s.workspace)
        return {"loss": s.loss, "dhidden": s.dhidden, "dtable": s.dtable}
    if c["op"] == "dropout":
        binding.blossom_dropout(s.params, s.x, s.rng, s.out)
        if not c["train"]:
            return {"out": s.out}
        binding.blossom_dropout(s.params_bwd, s.dout, s.rng, s.dx)
        return {"out": s.out, "dx": s.dx}
    binding.blossom_add_norm_fwd(s.params, s.x, s.residual, s.weight, s.bias, s.rng, s.out, s.stats)
    if not c["train"]:
        return {"out": s.out}
    binding.blossom_add_norm_bwd(s.params, s.x, s.residual, s.weight, s.rng, s.stats, s.dout, s.dx, s.dresidual,
                                 s.dweight, s.dbias, s.workspace)
    res = {"out": s.out, "dx": s.dx}
    if c["residual"]:
        res["dresidual"] = s.dresidual if c["p"] else s.dx
    return dict(res, dweight=s.dweight, dbias=s.dbias)


def _own_autograd(s, c):
    from paper_2512_13368_b200 import autograd as front
    with torch.set_grad_enabled(c["train"]):
        if c["op"] == "loss":
            loss = front.blossom_sampled_loss(s.hidden, s.table, s.targets, s.negatives, mask_hits=c["hits"])
            if not c["train"]:
                return {"loss": loss}
            dh, dtable = torch.autograd.grad(loss, (s.hidden, s.table), s.grad)
            return {"loss": loss, "dhidden": dh, "dtable": dtable}
        if c["op"] == "dropout":
            out = front.blossom_dropout(s.x, c["p"], s.rng, site=c["site"])
            if not c["train"]:
                return {"out": out}
            return {"out": out, "dx": torch.autograd.grad(out, s.x, s.dout)[0]}
        out = front.blossom_add_norm(s.x, s.residual, s.weight, s.bias, p=c["p"], rng=s.rng, site=c["site"], eps=c["eps"])
        if not c["train"]:
            return {"out": out}
        names = [n for n in ("x", "residual", "weight", "bias") if getattr(s, n) is not None]
        grads = torch.autograd.grad(out, [getattr(s, n) for n in names], s.dout)
        return dict({"out": out}, **{"d" + n: t for n, t in zip(names, grads)})


def run(state):
    c = state.case
    if own:
        return _own_abi(state, c) if c["entry"] == "abi" else _own_autograd(state, c)
    return {"loss": _plain_loss, "dropout": _plain_dropout, "norm": _plain_norm}[c["op"]](state, c)


# ---- what a pass cannot do without ---------------------------------------------------------------
def work(case):
    c = case
    R, C = c["rows"], c["cols"]
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "dropout":
        return {"bytes": (4 if c["train"] else 2) * R * C * e, "flops": (2 if c["train"] else 1) * R * C}
    if c["op"] == "norm":
        inputs = 2 if c["residual"] else 1
        # x (and residual) in, out out; for training dout in and the gradients out
        moved = inputs + 1
        if c["train"]:
            moved += 1 + (2 if c["residual"] and c["p"] else 1)
        return {"bytes": moved * R * C * e + (4 if c["train"] else 2) * C * e,
                "flops": (20 if c["train"] else 8) * R * C}
    live = R * (1.0 - c["ignored"])
    pairs = live * (c["n"] + 1)
    moved = live * C * e + min(c["items"], pairs) * C * e + R * 8 + (c["n"] if c["shared"] else live * c["n"]) * 8
    if c["train"]:
        moved += R * C * e + c["items"] * C * e
    return {"bytes": moved + 4, "flops": (6.0 if c["train"] else 2.0) * pairs * C}


# ---- the operators' definitions in 64 bits ---------------------------------------------------------
def _philox_numpy(rows, cols, rng, site):
    """16-bit numbers [rows, cols] from the generator's definition, word by word in numpy."""
    u = np.uint64
    seed, step = (int(v) & ((1 << 64) - 1) for v in rng.tolist())
    groups = -(-cols // 8)
    x = [np.broadcast_to((np.arange(groups, dtype=u) | u(site << 16))[None, :], (rows, groups)),
         np.broadcast_to(np.arange(rows, dtype=u)[:, None], (rows, groups)),
         np.full((rows, groups), step & _LOW, dtype=u), np.full((rows, groups), step >> 32, dtype=u)]
    key = [seed & _LOW, seed >> 32]
    low = u(_LOW)
    for _ in range(10):
        p0, p1 = x[0] * u(0xD2511F53), x[2] * u(0xCD9E8D57)
        x = [(p1 >> u(32)) ^ x[1] ^ u(key[0]), p1 & low, (p0 >> u(32)) ^ x[3] ^ u(key[1]), p0 & low]
        key = [(key[0] + 0x9E3779B9) & _LOW, (key[1] + 0xBB67AE85) & _LOW]
    out = np.empty((rows, groups, 8), dtype=np.int32)
    for i in range(4):
        out[:, :, 2 * i] = (x[i] & u(0xFFFF)).astype(np.int32)
        out[:, :, 2 * i + 1] = (x[i] >> u(16)).astype(np.int32)
    return out.reshape(rows, groups * 8)[:, :cols]


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    dev = torch.device("cuda")
    with torch.no_grad():
        if c["op"] == "loss":
            return _exact_loss(s, c, dev)
        factor = 1.0
        if c["p"]:
            bar = int(math.floor(c["p"] * 65536 + 0.5))
            bits = torch.from_numpy(_philox_numpy(c["rows"], c["cols"], s.rng, c["site"])).to(dev)
            factor = (bits >= bar).double() * (65536.0 / (65536 - bar))
        x = s.x.double()
        if c["op"] == "dropout":
            res = {"out": x * factor}
            if c["train"]:
                res["dx"] = s.dout.double() * factor
            return res
        z = x * factor + (s.residual.double() if c["residual"] else 0.0)
        n = c["cols"]
        mean = z.sum(1) / n
        var = ((z - mean[:, None]) ** 2).sum(1) / n
        sd = torch.sqrt(var + c["eps"])[:, None]
        unit = (z - mean[:, None]) / sd
        res = {"out": unit * s.weight.double() + s.bias.double()}
        if c["train"]:
            dy = s.dout.double()
            dunit = dy * s.weight.double()
            dz = (n * dunit - dunit.sum(1, keepdim=True) - unit * (dunit * unit).sum(1, keepdim=True)) / (n * sd)
            res["dx"] = dz * factor
            if c["residual"]:
                res["dresidual"] = dz
            res["dweight"] = torch.einsum("rc,rc->c", dy, unit)
            res["dbias"] = torch.einsum("rc->c", dy)
        return res


def _exact_loss(s, c, dev):
    R, C, n = c["rows"], c["cols"], c["n"]
    table = s.table.double()
    part = s.targets >= 0
    count = max(int(part.sum()), 1)
    loss = torch.zeros((), dtype=torch.float64, device=dev)
    dh = torch.zeros((R, C), dtype=torch.float64, device=dev)
    dtable = torch.zeros((c["items"], C), dtype=torch.float64, device=dev)
    block = max(1, (1 << 27) // ((n + 1) * C))
    for lo in range(0, R, block):
        at = torch.nonzero(part[lo:lo + block])[:, 0] + lo
        if not len(at):
            continue
        h, pos, neg = s.hidden[at].double(), s.targets[at], s.negatives[at]
        l0 = (h * table[pos]).sum(1)
        picked = table[neg]
        l1 = torch.einsum("tc,tnc->tn", h, picked)
        if c["hits"]:
            l1 = l1.masked_fill(neg == pos[:, None], -math.inf)
        lse = torch.logsumexp(torch.cat((l0[:, None], l1), 1), 1)
        loss += (lse - l0).sum()
        if c["train"]:
            p0, p1 = torch.exp(l0 - lse) - 1.0, torch.exp(l1 - lse[:, None])
            dh[at] = p0[:, None] * table[pos] + torch.einsum("tn,tnc->tc", p1, picked)
            dtable.index_add_(0, pos, p0[:, None] * h)
            dtable.index_add_(0, neg.reshape(-1), (p1[:, :, None] * h[:, None, :]).reshape(-1, C))
    res = {"loss": loss / count}
    if c["train"]:
        res.update(dhidden=dh / count, dtable=dtable / count)
    return res
