"""The sampled loss where its walks and its sort go round more than once: chunks of many windows of entries, items that reach over
windows, chunks and spans, counts of more tiles than a block scans at once; and bf16 rows of 72 to 120 columns on the matrix units.

The 64-bit definition is evaluated on the GPU here, position by position in blocks.  Tolerances as in test_sampled_loss.py, but
for an item's sum: a chunk's up to 512 additions one after another, up to 64 groups of lanes of a block, then the blocks' shares
one after another or side by side: 640 + entries / 128 additions at most."""
import numpy as np
import pytest

from paper_2512_13368_b200 import binding
from test_sampled_loss import U, compare, make, reference


# ---- the shapes of sort and walks, as the library chooses them ------------------------------------------
def plan(entries, lanes, threads):
    """(entries a group of lanes walks, blocks that do)"""
    chunk = 512
    while chunk > (32 if threads == 128 else 8) and entries // chunk * lanes < 2 * 148 * 1024:
        chunk //= 2
    span = chunk * (threads // lanes)
    return chunk, -(-entries // span)


def lanes_of(cols):
    groups = (cols + 7) // 8
    return 4 if groups <= 4 else 8 if groups <= 8 else 16 if groups <= 16 else 32


def workspace(rows, cols, items, n):
    """The bytes that plan and sort come to."""
    entries = rows * (n + 1)
    bits = max(items.bit_length(), 1)
    passes = (bits + 8) // 9
    digits = 1 << -(-bits // passes)
    spans = max(plan(entries, lanes_of(cols), 256)[1], plan(entries, 32, 128)[1])
    parts = [65536] + 4 * [4 * entries] + [4 * -(-entries // 4096) * digits, 4 * 512, 8 * items, 8 * spans * cols]
    return sum(-(-p // 256) * 256 for p in parts)


# rows, cols, items, n, type, what the walk does, entries a chunk has at least, tiles of the sort at least
LONG = [(40000, 64, 300001, 127, "bf16", "sixteens", 512, 1250), (40000, 24, 300001, 127, "bf16", "sixteens", 512, 1250),
        (40000, 128, 300001, 127, "bf16", "sixteens", 512, 1250), (40000, 72, 300001, 127, "bf16", "sixteens", 512, 1250),
        (13500, 8, 30011, 99, "fp32", "one by one", 4 * 4, 300), (13500, 50, 30011, 99, "fp32", "one by one", 4 * 8, 300),
        (13500, 100, 30011, 99, "fp32", "one by one", 4 * 16, 300), (13500, 200, 30011, 99, "fp32", "one by one", 4 * 32, 300),
        (13500, 300, 30011, 99, "fp32", "one by one", 4 * 32, 300), (13500, 600, 30011, 99, "fp32", "one by one", 4 * 32, 300),
        (13500, 64, 200003, 99, "bf16", "one by one", 4 * 8, 300), (13500, 65, 30011, 99, "bf16", "one by one", 4 * 16, 300),
        (66000, 8, 500001, 127, "bf16", "sixteens", 512, 2049), (66000, 8, 500001, 127, "fp32", "one by one", 64, 2049)]


@pytest.mark.parametrize("rows,cols,items,n,dtype,walk,chunk,tiles", LONG)
def test_the_sizes_below_reach_several_rounds(rows, cols, items, n, dtype, walk, chunk, tiles):
    """If the library chooses other shapes, its workspace is another one and the sizes below need a look."""
    binding.load()
    entries = rows * (n + 1)
    prm = binding.make_loss_params(rows, cols, items, n, dtype)
    assert binding.blossom_sampled_loss_workspace_bytes(prm) == workspace(rows, cols, items, n)
    by_sixteens = dtype == "bf16" and cols % 8 == 0 and cols <= 128 and entries // items >= 12
    assert (walk == "sixteens") == by_sixteens
    assert plan(entries, *((32, 128) if by_sixteens else (lanes_of(cols), 256)))[0] >= chunk
    assert -(-entries // 4096) >= tiles


def exact(h, w, t, neg):
    """The definition's results and the bounds, on the GPU: as test_sampled_loss.reference."""
    import torch
    rows, n, items, cols = h.shape[0], neg.shape[1], w.shape[0], h.shape[1]
    hd, wd = h.detach().double(), w.detach().double()
    part = (t >= 0) & (t < items)
    N = max(int(part.sum()), 1)
    z = lambda x: torch.zeros(x.shape, dtype=torch.float64, device="cuda")  # noqa: E731
    loss, tol_loss, dh, tol_h, dw, tol_w = 0.0, 0.0, z(hd), z(hd), z(wd), z(wd)
    count = torch.bincount(torch.cat([t[part], neg[part][(neg[part] >= 0) & (neg[part] < items)]]).long(), minlength=items).double()
    block = max(1, (1 << 28) // (8 * (n + 1) * cols))
    for lo in range(0, rows, block):
        at = torch.nonzero(part[lo:lo + block])[:, 0] + lo
        if not len(at):
            continue
        cand = torch.cat([t[at][:, None], neg[at]], 1).long()
        there = (cand >= 0) & (cand < items)
        cand = torch.where(there, cand, torch.zeros_like(cand))
        rowsw, x = wd[cand], hd[at]
        l = torch.einsum("tc,tnc->tn", x, rowsw)
        size = torch.einsum("tc,tnc->tn", x.abs(), rowsw.abs())
        lse = torch.logsumexp(l.masked_fill(~there, -np.inf), 1)
        eps = (48 * U * size + 8 * U * l.abs()).masked_fill(~there, 0).amax(1) + 8 * U * lse.abs()
        rho = 2 * eps + (n + 24) * U
        p = torch.exp(l - lse[:, None]).masked_fill(~there, 0)
        coef = p.clone()
        coef[:, 0] -= 1
        loss += float((lse - l[:, 0]).sum()) / N
        tol_loss += float(rho.sum()) / N
        dh[at] = torch.einsum("tn,tnc->tc", coef, rowsw) / N
        tol_h[at] = ((rho + (n + 24) * U)[:, None] * torch.einsum("tn,tnc->tc", p, rowsw.abs()) + 8 * U * rowsw[:, 0].abs()) / N
        off = (p * rho[:, None] + 4 * U + (640 + count[cand] / 128) * U * coef.abs()).masked_fill(~there, 0)
        dw.index_add_(0, cand.reshape(-1), (coef[:, :, None] * x[:, None, :]).reshape(-1, cols) / N)
        tol_w.index_add_(0, cand.reshape(-1), (off[:, :, None] * x[:, None, :].abs()).reshape(-1, cols) / N)
    return (loss, dh, dw), (tol_loss + 4 * U * abs(loss), tol_h, tol_w)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,items,n,dtype,walk,chunk,tiles", LONG)
def test_walks_and_sorts_of_several_rounds(rows, cols, items, n, dtype, walk, chunk, tiles):
    """Items with one entry, with some twenty, with thousands; positions without a target, negatives that are no items."""
    import torch
    from paper_2512_13368_b200.autograd import blossom_sampled_loss
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    h = torch.randn(rows, cols, generator=g, device="cuda").to(dt).requires_grad_(True)
    w = (torch.randn(items, cols, generator=g, device="cuda") / cols ** 0.5).to(dt).requires_grad_(True)
    t = torch.randint(0, items, (rows,), generator=g, device="cuda")
    t[torch.rand(rows, generator=g, device="cuda") < 0.1] = -100
    kind = torch.rand(rows, n, generator=g, device="cuda")
    draw = lambda lo, hi: torch.randint(lo, hi, (rows, n), generator=g, device="cuda")  # noqa: E731
    third, few = items // 3, max(items // 1000, 8)
    neg = torch.where(kind < 0.65, draw(third, items), torch.where(kind < 0.95, draw(third - few, third), draw(0, third - few)))
    neg[kind < 0.03] = -1
    (loss0, dh0, dw0), (tol, tol_h, tol_w) = exact(h, w, t, neg)
    entries = torch.bincount(neg[(t >= 0)[:, None].expand_as(neg) & (neg >= 0)], minlength=items)
    assert int((entries == 1).sum()) > 100 and int(entries.max()) > 1000 and (int(((entries > 8) & (entries < 99)).sum()) > 1000)

    def step():
        loss = blossom_sampled_loss(h, w, t, neg)
        return [loss.detach()] + list(torch.autograd.grad(loss, (h, w)))

    loss, dh, dw = first = step()
    assert abs(float(loss) - loss0) <= tol + 4 * U * abs(loss0)
    for got, ref, lim in ((dh, dh0, tol_h), (dw, dw0, tol_w)):
        lim = lim + ref.abs() * (2.0 ** -8 * 1.01 if dtype == "bf16" else 4 * U) + 1e-38
        bad = ~((got.double() - ref).abs() <= lim)
        assert not bad.any(), (int(bad.sum()), float((got.double() - ref).abs()[bad].max()))
    assert all(torch.equal(a, b) for a, b in zip(first, step()))


# ---- between 64 and 128 columns ----------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("cols", [72, 80, 96, 112, 120])
@pytest.mark.parametrize("rows,items,n", [(200, 90, 40), (2000, 90, 15), (300, 5000, 15), (150, 5000, 40), (1300, 4000, 33)])
def test_bf16_rows_of_72_to_120_columns(rows, items, n, cols):
    """A block a position (few positions, from 32 candidates on) and a warp a position; items of many entries and of few; with and
    without the gradient of the positions, and without any."""
    import torch
    from paper_2512_13368_b200.autograd import blossom_sampled_loss
    h, w, t, neg = make(rows, cols, items, n, "bf16", rows + cols + n)
    want, tol = reference(h, w, t, neg, hits=True)
    with torch.no_grad():
        compare({"loss": blossom_sampled_loss(h, w, t, neg, mask_hits=True)}, want, tol, True, "no gradient")
    w.requires_grad_(True)
    loss = blossom_sampled_loss(h, w, t, neg, mask_hits=True)
    compare({"loss": loss, "dtable": torch.autograd.grad(loss, w)[0]}, want, tol, True, "table alone")
    h.requires_grad_(True)
    loss = blossom_sampled_loss(h, w, t, neg, mask_hits=True)
    compare(dict(zip(("dhidden", "dtable"), torch.autograd.grad(loss, (h, w))), loss=loss), want, tol, True, "both")
    loss = blossom_sampled_loss(h, w.detach(), t, neg, mask_hits=True)
    compare({"loss": loss, "dhidden": torch.autograd.grad(loss, h)[0]}, want, tol, True, "positions alone")
