"""Sampled softmax loss on the GPU against the double-precision definition: sizes around the boundaries of the kernels'
shapes and of the sort, ids of either width, ignored positions, ids that are no items, hits, shared negatives, layouts.

Tolerances (u = 2^-24).  A logit is a sum of C <= 1024 products, at most 32 additions in a lane and 5 exchanges, then scaled:
  eps_t = max_j (48 u sum_i |h_i w_ji| + 8 u |l_j|) + 8 u |lse|
bounds what a logit, the log-sum-exp and their difference are off by; a probability's relative error is
  rho_t = 2 eps_t + (n + 24) u          (the sum of n + 1 exponentials, each good to a few units)
so |loss'| <= mean(rho_t) + 4 u |loss|, |dhidden'| <= ((rho_t + (n + 24) u) sum_j p_j |w_j| + 8 u |w_target|) / N and
|dtable'| <= sum over the item's entries of ((p rho_t + 4 u) + (512 + entries / 128) u |p - [target]|) |h_t| / N: a
chunk's sum of up to 128 entries, then the chunks' one after another or 64 side by side.
What is stored in bf16 is rounded once more (2^-8 relative)."""
import numpy as np
import pytest

from oracle import rows_oracle as ro
from paper_2512_13368_b200 import binding

U = 2.0 ** -24


def np64(t):
    return t.detach().double().cpu().numpy()


def reference(h, w, t, neg, ignore=-100, hits=False):
    """The definition's results and the bounds above."""
    h, w, t, neg = np64(h), np64(w), t.cpu().numpy(), neg.cpu().numpy()
    res = ro.sampled_loss(h, w, t, neg, ignore, hits)
    rows, n = h.shape[0], neg.shape[-1]
    neg = np.broadcast_to(neg, (rows, n))
    count = max(res["count"], 1)
    tol = {"loss": 4 * U * abs(res["loss"]), "dhidden": np.zeros_like(h), "dtable": np.zeros_like(w), "lse": np.zeros(rows)}
    entries = np.zeros(w.shape[0])
    pending = []
    for r in range(rows):
        if not (0 <= t[r] < w.shape[0]) or t[r] == ignore:
            continue
        c = [int(t[r])] + [int(i) for i in neg[r] if 0 <= i < w.shape[0] and not (hits and i == t[r])]
        l = w[c] @ h[r]
        eps = float((48 * U * (np.abs(w[c]) @ np.abs(h[r])) + 8 * U * np.abs(l)).max()) + 8 * U * abs(res["lse"][r])
        rho = 2 * eps + (n + 24) * U
        p = np.exp(l - res["lse"][r])
        tol["loss"] += rho / count
        tol["lse"][r] = rho + 4 * U * abs(res["lse"][r])
        tol["dhidden"][r] = ((rho + (n + 24) * U) * (p @ np.abs(w[c])) + 8 * U * np.abs(w[c[0]])) / count
        coef = p.copy()
        coef[0] -= 1
        np.add.at(entries, c, 1)
        pending.append((c, p * rho + 4 * U, np.abs(coef), np.abs(h[r])))
    for c, a, coef, ah in pending:
        np.add.at(tol["dtable"], c, (a + (512 + entries[c] / 128) * U * coef)[:, None] * ah[None, :] / count)
    return res, tol


def compare(got, want, tol, bf16, what=""):
    for key, x in got.items():
        g, ref = np64(x).reshape(np.shape(want[key])), np.asarray(want[key])
        lim = tol[key] + (2.0 ** -8 * 1.01 * np.abs(ref) if bf16 and key[0] == "d" else 4 * U * np.abs(ref)) + 1e-38
        bad = ~(np.abs(g - ref) <= lim)
        assert not bad.any(), (what, key, int(bad.sum()), np.abs(g - ref)[bad].max(), g[bad][:3], ref[bad][:3], np.asarray(lim)[bad][:3])


def make(rows, cols, items, n, dtype, seed, ids="int64", noise=True, shared=False, popular=False):
    import torch
    g = np.random.default_rng(seed)
    dt = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]
    up = lambda a: torch.from_numpy(a.astype(np.float32)).cuda().to(dt)  # noqa: E731
    h, w = up(g.standard_normal((rows, cols))), up(0.3 * g.standard_normal((items, cols)))
    t = g.integers(0, items, rows) if not popular else np.minimum(g.geometric(0.4, rows) - 1, items - 1)
    neg = g.integers(0, items, (n,) if shared else (rows, n))
    if noise and rows > 4:
        t[g.random(rows) < 0.2] = -100
        t[1], t[3] = items, -1
        neg[g.random(neg.shape) < 0.1] = -7
        neg[g.random(neg.shape) < 0.05] = items
        if not shared and n:
            hit = g.random(rows) < 0.3
            neg[hit, 0] = t[hit]
    it = {"int64": torch.int64, "int32": torch.int32}[ids]
    return h, w, torch.from_numpy(t).cuda().to(it), torch.from_numpy(neg).cuda().to(it)


SHAPES = [(1, 64, 10, 1), (1, 1, 1, 0), (2, 3, 2, 5), (5, 8, 3, 7), (64, 64, 50001, 100), (300, 50, 1000, 31), (130, 32, 513, 9),
          (97, 33, 511, 32), (200, 128, 70000, 64), (33, 256, 200, 40), (20, 257, 99, 33), (9, 512, 30, 12), (21, 520, 30, 5),
          (6, 1024, 40, 70), (700, 64, 5000, 63), (4000, 16, 7, 20), (600, 24, 300001, 33), (1170, 64, 255, 6), (1171, 64, 256, 6),
          (3000, 8, 2, 3), (2500, 65, 40, 12),
          (9000, 16, 3000, 31), (9000, 8, 300001, 31), (65, 128, 700, 9), (129, 128, 30, 130)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols,items,n", SHAPES)
def test_loss_and_gradients_over_the_sizes(rows, cols, items, n, dtype):
    import torch
    from paper_2512_13368_b200.autograd import blossom_sampled_loss
    for ids, hits in (("int64", False), ("int32", True)):
        h, w, t, neg = make(rows, cols, items, n, dtype, rows + cols + n, ids)
        want, tol = reference(h, w, t, neg, hits=hits)
        h.requires_grad_(True), w.requires_grad_(True)
        loss = blossom_sampled_loss(h, w, t, neg, mask_hits=hits)
        assert loss.dtype == torch.float32 and loss.dim() == 0
        dh, dw = torch.autograd.grad(loss, (h, w))
        compare({"loss": loss, "dhidden": dh, "dtable": dw}, want, tol, dtype == "bf16", (ids, hits))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,items,n,popular,shared", [(9000, 60, 3, True, False), (6000, 2000, 7, False, True), (20000, 3, 1, True, False),
                                                         (12000, 30000, 2, True, False)])
def test_popular_items_and_shared_negatives(rows, items, n, popular, shared, dtype):
    """Items with thousands of entries: their sums reach over many chunks, and over more than one group joins alone."""
    import torch
    from paper_2512_13368_b200.autograd import blossom_sampled_loss
    h, w, t, neg = make(rows, 16, items, n, dtype, 3, shared=shared, popular=popular)
    want, tol = reference(h, w, t, neg)
    h.requires_grad_(True), w.requires_grad_(True)
    loss = blossom_sampled_loss(h, w, t, neg)
    first = torch.autograd.grad(loss, (h, w), retain_graph=True)
    compare({"loss": loss, "dhidden": first[0], "dtable": first[1]}, want, tol, dtype == "bf16")
    for _ in range(3):
        again = torch.autograd.grad(blossom_sampled_loss(h, w, t, neg), (h, w))
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    if shared:  # the same ids as an expanded matrix, and as one that is written out
        for m in (neg.expand(rows, n), neg.expand(rows, n).contiguous()):
            again = torch.autograd.grad(blossom_sampled_loss(h, w, t, m), (h, w))
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def abi(h, w, t, neg, dtype, **kw):
    """Through the C ABI with a poisoned workspace; returns outputs."""
    import torch
    rows, cols, items, n = h.shape[0], h.shape[1], w.shape[0], neg.shape[1]
    prm = binding.make_loss_params(rows, cols, items, n, dtype, index_bytes=t.element_size(), hidden_stride=h.stride(0),
                                   table_stride=w.stride(0), negatives_stride=neg.stride(0), **kw)
    f = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
    loss, lse, gh = f(1), f(rows + 1), f(rows, cols)
    dh, dw = (torch.full_like(x, float("nan"), memory_format=torch.contiguous_format) for x in (h, w))
    ws = torch.full((binding.blossom_sampled_loss_workspace_bytes(prm),), 0xFF, dtype=torch.uint8, device="cuda")
    binding.blossom_sampled_loss_fwd(prm, h, w, t, neg, loss, lse, gh, ws)
    ws.fill_(0xFF)
    binding.blossom_sampled_loss_bwd(prm, h, w, t, neg, lse, gh, None, dh, dw, ws)
    return {"loss": loss, "lse": lse[:-1], "dhidden": dh, "dtable": dw}, float(lse[-1])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_strides_workspace_contents_and_saved_values(dtype):
    import torch
    h, w, t, neg = make(500, 40, 900, 20, dtype, 9)
    want, tol = reference(h, w, t, neg, ignore=5)
    got, count = abi(h, w, t, neg, dtype, ignore_index=5)
    assert count == want["count"]
    compare(got, want, tol, dtype == "bf16")
    # rows inside wider buffers, at every alignment
    for shift in (0, 1, 2, 8):
        wide = lambda x, s=shift: torch.cat([torch.full((x.shape[0], s), 9, dtype=x.dtype, device="cuda"), x,  # noqa: E731
                                             torch.full((x.shape[0], 3), 9, dtype=x.dtype, device="cuda")], 1)[:, s:s + x.shape[1]]
        again, _ = abi(wide(h), wide(w), t, wide(neg), dtype, ignore_index=5)
        compare(again, want, tol, dtype == "bf16", shift)


@pytest.mark.gpu
def test_layouts_the_front_end_resolves():
    import torch
    from paper_2512_13368_b200.autograd import blossom_sampled_loss
    h, w, t, neg = make(60, 24, 100, 6, "fp32", 2)
    want = blossom_sampled_loss(h, w, t, neg)
    h3, t3, n3 = h.view(5, 12, 24), t.view(5, 12), neg.view(5, 12, 6)
    assert torch.equal(blossom_sampled_loss(h3, w, t3, n3), want)
    perm = lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    a = perm(h3).requires_grad_(True)
    loss = blossom_sampled_loss(a, perm(w), perm(t3), perm(n3))
    assert torch.equal(loss, want)
    b = h3.clone().requires_grad_(True)
    assert torch.equal(torch.autograd.grad(loss, a)[0], torch.autograd.grad(blossom_sampled_loss(b, w, t3, n3), b)[0])
    assert torch.equal(blossom_sampled_loss(h[0], w, t[0], neg[0]), blossom_sampled_loss(h[:1], w, t[:1], neg[:1]))


@pytest.mark.gpu
def test_upstream_gradient_and_only_what_is_wanted():
    import torch
    from paper_2512_13368_b200.autograd import blossom_sampled_loss
    h, w, t, neg = make(300, 64, 1000, 15, "fp32", 6)
    want, tol = reference(h, w, t, neg)
    scaled = {k: want[k] * -2.5 for k in ("dhidden", "dtable")}
    bound = {k: tol[k] * 2.5 for k in scaled}
    h.requires_grad_(True), w.requires_grad_(True)
    (blossom_sampled_loss(h, w, t, neg) * -2.5).backward()
    compare({"dhidden": h.grad, "dtable": w.grad}, scaled, bound, False)
    only_h = torch.autograd.grad(blossom_sampled_loss(h, w.detach(), t, neg) * -2.5, h)[0]
    only_w = torch.autograd.grad(blossom_sampled_loss(h.detach(), w, t, neg) * -2.5, w)[0]
    assert torch.equal(only_h, h.grad) and torch.equal(only_w, w.grad)
    with torch.no_grad():
        assert blossom_sampled_loss(h, w, t, neg).grad_fn is None


@pytest.mark.gpu
def test_positions_and_items_that_take_no_part_are_not_read():
    import torch
    from paper_2512_13368_b200.autograd import blossom_sampled_loss
    h, w, t, neg = make(200, 32, 5000, 4, "bf16", 7)
    used = torch.zeros(5000, dtype=torch.bool, device="cuda")
    live = (t >= 0) & (t < 5000)
    used[t[live]] = True
    cand = neg[live]
    used[cand[(cand >= 0) & (cand < 5000)]] = True
    h2, w2 = h.clone(), w.clone()
    h2[~live], w2[~used] = float("nan"), float("inf")
    a = [x.clone().requires_grad_(True) for x in (h, w)]
    b = [x.clone().requires_grad_(True) for x in (h2, w2)]
    la, lb = blossom_sampled_loss(*a, t, neg), blossom_sampled_loss(*b, t, neg)
    ga, gb = torch.autograd.grad(la, a), torch.autograd.grad(lb, b)
    assert torch.equal(la, lb) and torch.equal(ga[0], gb[0]) and torch.equal(ga[1], gb[1])
    assert not gb[0][~live].any() and not gb[1][~used].any()


@pytest.mark.gpu
def test_a_row_that_is_no_number_shows():
    import torch
    from paper_2512_13368_b200.autograd import blossom_sampled_loss
    for n in (0, 1, 3, 40):
        for bad in (float("nan"), float("inf")):
            h, w, t, neg = make(40, 16, 100, n, "fp32", 8, noise=False)
            h[11] = bad
            h.requires_grad_(True)
            loss = blossom_sampled_loss(h, w, t, neg)
            (dh,) = torch.autograd.grad(loss, h)
            assert not torch.isfinite(loss) and not torch.isfinite(dh[11]).all() and torch.isfinite(dh[:11]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,cols", [("bf16", 64), ("bf16", 50), ("fp32", 64)])
def test_a_row_that_is_no_number_spoils_its_own_items_alone(dtype, cols):
    import torch
    from paper_2512_13368_b200.autograd import blossom_sampled_loss
    h, w, t, neg = make(300, cols, 4000, 6, dtype, 8, noise=False)
    h2 = h.clone()
    h2[57, 3] = float("nan")
    a, b = w.clone().requires_grad_(True), w.clone().requires_grad_(True)
    g = torch.autograd.grad(blossom_sampled_loss(h, a, t, neg), a)[0]
    bad = torch.autograd.grad(blossom_sampled_loss(h2, b, t, neg), b)[0]
    mine = torch.zeros(4000, dtype=torch.bool, device="cuda")
    mine[t[57]] = True
    mine[neg[57]] = True
    assert torch.equal(g[~mine], bad[~mine]) and bool(bad[mine].isnan().any(1).all())


@pytest.mark.gpu
def test_nothing_to_do():
    import torch
    from paper_2512_13368_b200.autograd import blossom_sampled_loss
    w = torch.randn(50, 16, device="cuda", requires_grad=True)
    for rows, t in ((0, []), (3, [-100, 50, -1])):
        h = torch.randn(rows, 16, device="cuda", requires_grad=True)
        t = torch.tensor(t, dtype=torch.int64, device="cuda")
        neg = torch.zeros(rows, 4, dtype=torch.int64, device="cuda")
        loss = blossom_sampled_loss(h, w, t, neg)
        dh, dw = torch.autograd.grad(loss, (h, w))
        assert float(loss.detach()) == 0.0 and not dh.any() and not dw.any() and dh.shape == h.shape
    # no negative at all: the target is certain
    h = torch.randn(3, 16, device="cuda", requires_grad=True)
    loss = blossom_sampled_loss(h, w, torch.tensor([1, 2, 2], device="cuda"), torch.zeros(3, 0, dtype=torch.int64, device="cuda"))
    dh, dw = torch.autograd.grad(loss, (h, w))
    assert abs(float(loss.detach())) < 1e-6 and float(dh.abs().max()) < 1e-6 and float(dw.abs().max()) < 1e-6
    # every negative masked: the same
    loss = blossom_sampled_loss(h, w, torch.tensor([1, 2, 2], device="cuda"), torch.tensor([[1], [2], [-5]], device="cuda"), mask_hits=True)
    assert abs(float(loss.detach())) < 1e-6


@pytest.mark.gpu
def test_logits_far_apart():
    """Logits of some hundreds: exponentials that vanish, a maximum that comes late."""
    import torch
    from paper_2512_13368_b200.autograd import blossom_sampled_loss
    h, w, t, neg = make(100, 64, 300, 50, "fp32", 10, noise=False)
    h = h * 40
    want, tol = reference(h, w, t, neg)
    h.requires_grad_(True), w.requires_grad_(True)
    loss = blossom_sampled_loss(h, w, t, neg)
    dh, dw = torch.autograd.grad(loss, (h, w))
    compare({"loss": loss, "dhidden": dh, "dtable": dw}, want, tol, False)


@pytest.mark.gpu
def test_gradient_against_differences_of_the_kernel():
    """Central differences with step h = 2^-4 along a unit direction: the loss (about 3) is stored with an error below 2^-20, so
    the quotient is off by 2^-20 / 2^-4 = 2^-16 and by h^2 / 6 times a third derivative of at most |table row|^3 / N ~ 2^3 / 64:
    2^-8 2^-3 / 6 < 2^-13.  Both stay below 2^-12."""
    import torch
    from paper_2512_13368_b200.autograd import blossom_sampled_loss
    h, w, t, neg = make(64, 16, 200, 20, "fp32", 11, noise=False)
    a, b = h.clone().requires_grad_(True), w.clone().requires_grad_(True)
    dh, dw = torch.autograd.grad(blossom_sampled_loss(a, b, t, neg), (a, b))
    torch.manual_seed(0)
    s = 2.0 ** -4
    v = torch.randn_like(h)
    v /= v.norm()
    f = lambda x, y: float(blossom_sampled_loss(x, y, t, neg).double())  # noqa: E731
    assert abs((f(h + s * v, w) - f(h - s * v, w)) / (2 * s) - float((dh.double() * v.double()).sum())) < 2.0 ** -12
    v = torch.randn_like(w)
    v /= v.norm()
    assert abs((f(h, w + s * v) - f(h, w - s * v)) / (2 * s) - float((dw.double() * v.double()).sum())) < 2.0 ** -12


@pytest.mark.gpu
def test_another_stream_and_a_captured_step():
    import torch
    from paper_2512_13368_b200.autograd import blossom_sampled_loss
    h, w, t, neg = make(3000, 64, 5000, 9, "bf16", 12)
    h.requires_grad_(True), w.requires_grad_(True)
    want = blossom_sampled_loss(h, w, t, neg)
    grads = torch.autograd.grad(want, (h, w))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        loss = blossom_sampled_loss(h, w, t, neg)
        g = torch.autograd.grad(loss, (h, w))
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(loss, want) and torch.equal(g[0], grads[0]) and torch.equal(g[1], grads[1])
    # (leaves of the graph's own: autograd remembers the stream on which a leaf was first used)
    h, w = h.detach().requires_grad_(True), w.detach().requires_grad_(True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = blossom_sampled_loss(h, w, t, neg)
        g = torch.autograd.grad(loss, (h, w))
    for _ in range(2):
        graph.replay()
        assert torch.equal(loss, want) and torch.equal(g[0], grads[0]) and torch.equal(g[1], grads[1])


@pytest.mark.gpu
def test_rows_further_apart_than_32_bits_reach():
    """Row strides of 2^30 + 8 elements: the third row starts behind 2^31 elements."""
    import torch
    from paper_2512_13368_b200.autograd import blossom_add_norm, blossom_dropout, blossom_sampled_loss
    st = (1 << 30) + 8
    buf = torch.empty(2 * st + 64, dtype=torch.bfloat16, device="cuda")
    far = buf.as_strided((3, 64), (st, 1))
    x = torch.randn(3, 64, device="cuda").bfloat16()
    far.copy_(x)
    rng = torch.tensor([1, 2], device="cuda")
    w = torch.randn(64, device="cuda").bfloat16()
    for f in (lambda y: blossom_dropout(y, 0.5, rng), lambda y: blossom_add_norm(y, y, w, w, p=0.5, rng=rng)):
        a, b = x.clone().requires_grad_(True), far.detach().requires_grad_(True)
        oa, ob = f(a), f(b)
        assert torch.equal(oa, ob) and torch.equal(torch.autograd.grad(oa, a, x)[0], torch.autograd.grad(ob, b, x)[0])
    t, neg = torch.tensor([2, 0, 1], device="cuda"), torch.tensor([[0, 1], [2, 2], [0, 2]], device="cuda")
    a, b = x.clone().requires_grad_(True), far.detach().requires_grad_(True)
    la, lb = blossom_sampled_loss(a, a, t, neg), blossom_sampled_loss(b, b, t, neg)
    assert torch.equal(la, lb) and torch.equal(torch.autograd.grad(la, a)[0], torch.autograd.grad(lb, b)[0])
    out = blossom_dropout(x, 0.5, rng)
    far.fill_(7)
    prm = binding.make_rows_params(3, 64, "bf16", dropout=0.5, out_stride=st)
    binding.blossom_dropout(prm, x, rng, far)
    assert torch.equal(far, out)


@pytest.mark.gpu
def test_front_end_refusals():
    import torch
    from paper_2512_13368_b200.autograd import blossom_sampled_loss
    h, w, t, neg = make(6, 8, 20, 3, "fp32", 1)
    for args, exc in (((h.cpu(), w, t, neg), ValueError), ((h.half(), w.half(), t, neg), TypeError), ((h, w[:, :4], t, neg), ValueError),
                      ((h, w.bfloat16(), t, neg), TypeError), ((h, w, t[:3], neg), ValueError), ((h, w, t, neg[:3]), ValueError),
                      ((h, w, t.int(), neg), TypeError), ((h, w, t.float(), neg.float()), TypeError), ((h, w, t.cpu(), neg), ValueError),
                      ((h, w[:0], t, neg), ValueError), ((h, w, t, None), ValueError),
                      ((torch.zeros(2, 1025, device="cuda"), torch.zeros(2, 1025, device="cuda"), t[:2], neg[:2]), binding.BlossomError)):
        with pytest.raises(exc):
            blossom_sampled_loss(*args)
    a = h.requires_grad_(True)
    (g,) = torch.autograd.grad(blossom_sampled_loss(a, w, t, neg), a, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivative"):
        g.sum().backward()


def test_arguments_are_checked_before_any_launch():
    binding.load()
    E, A = binding, 1 << 20
    good = lambda **kw: E.make_loss_params(**dict(dict(rows=10, cols=64, items=100, negatives=5, dtype="bf16"), **kw))  # noqa: E731
    n = E.blossom_sampled_loss_workspace_bytes(good())
    assert n > E.LOSS_FORWARD_BYTES and n % 256 == 0
    assert E.blossom_sampled_loss_workspace_bytes(good(rows=0)) >= E.LOSS_FORWARD_BYTES
    for bad, rc in ((dict(rows=-1), 1), (dict(cols=0), 1), (dict(cols=1025), 2), (dict(items=0), 1), (dict(items=1 << 30), 2),
                    (dict(negatives=-1), 1), (dict(dtype=4), 1), (dict(index_bytes=2), 1), (dict(mask_hits=2), 1),
                    (dict(hidden_stride=63), 1), (dict(table_stride=-64), 1), (dict(dhidden_stride=1), 1), (dict(dtable_stride=1), 1),
                    (dict(negatives_stride=-1), 1), (dict(rows=1 << 31), 2), (dict(rows=1 << 29, negatives=3), 2),
                    (dict(negatives_stride=1 << 31), 2)):
        p = good(**bad)
        assert E.blossom_sampled_loss_workspace_bytes(p) == 0, bad
        assert E.blossom_sampled_loss_fwd(p, A, A, A, A, A, A, A, A, 1 << 40, stream=0, check=False) == rc, bad
        assert E.blossom_sampled_loss_bwd(p, A, A, A, A, A, A, A, A, A, A, 1 << 40, stream=0, check=False) == rc, bad
    p = good()
    for i, v in ((0, None), (0, A + 1), (1, None), (1, A + 1), (2, None), (2, A + 4), (3, None), (3, A + 4), (4, None), (4, A + 2),
                 (5, None), (5, A + 2), (6, A + 8)):
        args = [A] * 7
        args[i] = v
        assert E.blossom_sampled_loss_fwd(p, *args, A, n, stream=0, check=False) == E.BLOSSOM_ERR_INVALID_ARG, (i, v)
    for i, v in ((0, None), (1, None), (2, None), (3, None), (4, None), (5, None), (5, A + 4), (6, A + 2), (7, A + 1), (8, A + 1)):
        args = [A] * 9
        args[i] = v
        assert E.blossom_sampled_loss_bwd(p, *args, A, n, stream=0, check=False) == E.BLOSSOM_ERR_INVALID_ARG, (i, v)
    assert E.blossom_sampled_loss_bwd(p, *[A] * 7, None, None, A, n, stream=0, check=False) == E.BLOSSOM_ERR_INVALID_ARG
    for ws, size in ((None, n), (A + 128, n)):
        assert E.blossom_sampled_loss_fwd(p, *[A] * 7, ws, size, stream=0, check=False) == E.BLOSSOM_ERR_WORKSPACE
        assert E.blossom_sampled_loss_bwd(p, *[A] * 9, ws, size, stream=0, check=False) == E.BLOSSOM_ERR_WORKSPACE
    assert E.blossom_sampled_loss_fwd(p, *[A] * 7, A, E.LOSS_FORWARD_BYTES - 1, stream=0, check=False) == E.BLOSSOM_ERR_WORKSPACE
    assert E.blossom_sampled_loss_bwd(p, *[A] * 9, A, n - 1, stream=0, check=False) == E.BLOSSOM_ERR_WORKSPACE


def test_loss_params_layout_matches_the_header():
    import ctypes
    f = binding.blossom_loss_params
    assert ctypes.sizeof(f) == 80 and f.mask_hits.offset == 28 and f.ignore_index.offset == 32 and f.negatives_stride.offset == 72
