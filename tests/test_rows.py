"""Dropout and residual + layer norm on the GPU against the double-precision definitions: sizes around every boundary of
the kernels' shapes, strides and alignments, what may be missing, dropped non-finite values, streams, graphs.

Tolerances (u = 2^-24, one rounding of single precision).  A sum over C <= 8192 columns is eight additions in a thread, up to
ten exchanges and up to 32 warps, a variance's terms have three roundings more, the square root's approximation
two units: fewer than 64 roundings stand between the inputs and any value of a row.  So
  |n - n'|   <= 64 u (rstd max|terms of z| + |n|)                                      =: eta
  |out'|     <= eta |w| + 4 u (|n w| + |b|)
  |dz'|      <= rstd (64 u (|a| + A + |n| B) + eta B + |n| mean(|a|) max eta), A = mean|a|, B = mean|a n|
  |dweight'| <= sum_rows |dout| eta + 128 u sum_rows |dout n|    (a column's sum: rows of a thread, 32 slots, CTAs)
and what is stored in bf16 is rounded once more (2^-8 relative: eight significant bits are 2^-7 apart)."""
import numpy as np
import pytest

from oracle import rows_oracle as ro
from paper_2512_13368_b200 import binding

U = 2.0 ** -24


def bounds(x, residual, f, dout, b):
    terms = np.abs(np.where(f["factor"] == 0, 0, x * f["factor"])) + (0 if residual is None else np.abs(residual))
    eta = 64 * U * (f["rstd"] * terms.max(axis=1, keepdims=True) + np.abs(f["n"]))
    n, w, rstd = np.abs(f["n"]), np.abs(f["w"]), f["rstd"]
    res = {"out": eta * w + 4 * U * (n * w + (0 if b is None else np.abs(b)))}
    if dout is not None:
        a = np.abs(dout * f["w"])
        A, B = a.mean(axis=1, keepdims=True), (a * n).mean(axis=1, keepdims=True)
        dz = rstd * (64 * U * (a + A + n * B) + eta * B + n * A * eta.max(axis=1, keepdims=True))
        res["dresidual"] = dz
        res["dx"] = dz * np.maximum(f["factor"], 1.0)
        res["dweight"] = (np.abs(dout) * eta).sum(axis=0) + 128 * U * np.abs(dout * f["n"]).sum(axis=0)
        res["dbias"] = 128 * U * np.abs(dout).sum(axis=0)
    return res


def compare(got, want, tol, bf16, what):
    for key, t in got.items():
        g = t.detach().double().cpu().numpy().reshape(want[key].shape)
        lim = tol[key] + (2.0 ** -8 * np.abs(want[key]) * 1.01 + 1e-38 if bf16.get(key, bf16["all"]) else 1e-38)
        bad = ~(np.abs(g - want[key]) <= lim)
        assert not bad.any(), (what, key, int(bad.sum()), float(np.abs(g - want[key])[bad].max()), g[bad][:3], want[key][bad][:3])


def tensors(rows, cols, dtype, seed, residual=True, weights=True, wide_weights=False):
    import torch
    dt = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = np.random.default_rng(seed)
    up = lambda a, d=dt: torch.from_numpy(a.astype(np.float32)).cuda().to(d)  # noqa: E731
    x, r, dout = up(g.standard_normal((rows, cols)) * 2), up(g.standard_normal((rows, cols)) + 0.5), up(g.standard_normal((rows, cols)))
    wd = torch.float32 if wide_weights else dt
    w, b = up(1 + 0.3 * g.standard_normal(cols), wd), up(0.3 * g.standard_normal(cols), wd)
    return x, (r if residual else None), (w if weights else None), (b if weights else None), dout


def np64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def reference(x, r, w, b, dout, p, seed, step, site, eps):
    fac = ro.keep_factor(x.shape[0], x.shape[1], p, seed, step, site)
    f = ro.add_norm(np64(x), np64(r), np64(w), np64(b), fac, eps)
    want = dict(ro.add_norm_backward(f, np64(dout)), out=f["out"])
    return want, bounds(np64(x), np64(r), f, np64(dout), np64(b))


SHAPES = [(1, 64), (2, 64), (33, 64), (1000, 64), (1, 1), (5, 1), (3, 2), (40, 7), (65, 8), (17, 9), (64, 32), (129, 33),
          (300, 50), (77, 100), (31, 128), (9, 129), (200, 250), (35, 256), (12, 257), (20, 511), (21, 512), (11, 520), (6, 1000),
          (19, 1024), (10, 1026), (7, 2048), (5, 2056), (3, 4096), (4, 4100), (3, 8191), (2, 8192), (4096, 24)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_add_norm_over_the_sizes(rows, cols, dtype):
    import torch
    from paper_2512_13368_b200.autograd import blossom_add_norm
    for p, residual in ((0.0, True), (0.3, True), (0.2, False)):
        x, r, w, b, dout = tensors(rows, cols, dtype, rows + cols, residual=residual)
        want, tol = reference(x, r, w, b, dout, p, 99 - rows, cols, 5, 1e-5)
        leaves = [t.requires_grad_(True) for t in (x, r, w, b) if t is not None]
        rng = torch.tensor([99 - rows, cols], device="cuda")
        out = blossom_add_norm(x, r, w, b, p=p, rng=rng, site=5)
        grads = torch.autograd.grad(out, leaves, dout)
        names = ["dx"] + (["dresidual"] if residual else []) + ["dweight", "dbias"]
        compare(dict(zip(names, grads), out=out), want, tol, {"all": dtype == "bf16"}, (p, residual))


# more rows than the GPU takes at once, several times over: a CTA's rows follow each other through its stages
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(285001, 8), (60003, 50), (30011, 136), (9001, 520), (6007, 1024), (2003, 2056), (1501, 4096), (901, 8192)])
def test_add_norm_over_many_rows_a_cta(rows, cols, dtype):
    import torch
    from paper_2512_13368_b200.autograd import blossom_add_norm
    x, r, w, b, dout = tensors(rows, cols, dtype, rows + cols)
    want, tol = reference(x, r, w, b, dout, 0.3, 7, 8, 9, 1e-5)
    leaves = [t.requires_grad_(True) for t in (x, r, w, b)]
    out = blossom_add_norm(x, r, w, b, p=0.3, rng=torch.tensor([7, 8], device="cuda"), site=9)
    grads = torch.autograd.grad(out, leaves, dout)
    compare(dict(zip(["dx", "dresidual", "dweight", "dbias"], grads), out=out), want, tol, {"all": dtype == "bf16"}, "many rows")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("weights,wide", [(True, True), (True, False), (False, False)])
def test_add_norm_weights_of_their_own_type_or_none(dtype, weights, wide):
    import torch
    from paper_2512_13368_b200.autograd import blossom_add_norm
    x, r, w, b, dout = tensors(130, 72, dtype, 5, weights=weights, wide_weights=wide)
    want, tol = reference(x, r, w, b, dout, 0.1, 1, 2, 3, 1e-3)
    leaves = [t.requires_grad_(True) for t in (x, r, w, b) if t is not None]
    out = blossom_add_norm(x, r, w, b, p=0.1, rng=torch.tensor([1, 2], device="cuda"), site=3, eps=1e-3)
    grads = torch.autograd.grad(out, leaves, dout)
    if wide:
        assert grads[2].dtype == torch.float32
    wb = dtype == "bf16" and not wide
    compare(dict(zip(["dx", "dresidual", "dweight", "dbias"], grads), out=out), want, tol,
            {"all": dtype == "bf16", "dweight": wb, "dbias": wb}, "weights")
    # one of the two alone
    if weights:
        w1, b1 = w.detach().clone().requires_grad_(True), b.detach().clone().requires_grad_(True)
        for ww, bb in ((w1, None), (None, b1)):
            want, tol = reference(x, None, ww, bb, dout, 0.0, 0, 0, 0, 1e-5)
            out = blossom_add_norm(x.detach(), None, ww, bb)
            (g,) = torch.autograd.grad(out, [ww if bb is None else bb], dout)
            compare({"out": out, "dweight" if bb is None else "dbias": g}, want, tol, {"all": dtype == "bf16", "dweight": wb, "dbias": wb}, "one")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("cols,pad,shift", [(64, 16, 0), (64, 16, 8), (64, 2, 0), (64, 3, 1), (50, 14, 0), (50, 13, 3), (512, 8, 2)])
def test_strides_and_addresses(dtype, cols, pad, shift):
    """x, residual, dout: slices of wider buffers at every alignment; the neighbours of every output stay as they were."""
    import torch
    rows, p = 37, 0.25
    x, r, w, b, dout = tensors(rows, cols, dtype, cols + pad)
    want, tol = reference(x, r, w, b, dout, p, 4, 5, 6, 1e-5)

    def wide(t, value=7.0):
        buf = torch.full((rows, cols + pad + shift), value, dtype=x.dtype, device="cuda")
        view = buf[:, shift:shift + cols]
        if t is not None:
            view.copy_(t)
        return buf, view

    xs, rs, ds = wide(x)[1], wide(r)[1], wide(dout)[1]
    (ob, out), (db, dx), (eb, dres) = wide(None), wide(None), wide(None)
    st = cols + pad + shift
    prm = binding.make_rows_params(rows, cols, dtype, dropout=p, site=6, x_stride=st, residual_stride=st, out_stride=st,
                                   dx_stride=st, dresidual_stride=st)
    rng = torch.tensor([4, 5], device="cuda")
    stats = torch.empty(rows, 2, device="cuda")
    dw, dbias = torch.empty_like(w), torch.empty_like(b)
    ws = torch.empty(binding.blossom_add_norm_workspace_bytes(prm), dtype=torch.uint8, device="cuda")
    ws.fill_(0xFF)
    binding.blossom_add_norm_fwd(prm, xs, rs, w, b, rng, out, stats)
    binding.blossom_add_norm_bwd(prm, xs, rs, w, rng, stats, ds, dx, dres, dw, dbias, ws)
    compare({"out": out, "dx": dx, "dresidual": dres, "dweight": dw, "dbias": dbias}, want, tol, {"all": dtype == "bf16"}, "strided")
    for buf in (ob, db, eb):
        rest = torch.cat([buf[:, :shift], buf[:, shift + cols:]], dim=1)
        assert bool((rest == 7.0).all())
    # the same for dropout alone, in place
    yb, y = wide(x)
    binding.blossom_dropout(binding.make_rows_params(rows, cols, dtype, dropout=p, site=6, x_stride=st, out_stride=st), y, rng, y)
    fac = ro.keep_factor(rows, cols, p, 4, 5, 6)
    lim = np.abs(np64(x)) * fac * ((2.0 ** -8 if dtype == "bf16" else 0) + 2 * U)
    assert np.all(np.abs(np64(y) - np64(x) * fac) <= lim)
    assert bool((torch.cat([yb[:, :shift], yb[:, shift + cols:]], dim=1) == 7.0).all())


@pytest.mark.gpu
def test_layouts_the_front_end_resolves():
    import torch
    from paper_2512_13368_b200.autograd import blossom_add_norm, blossom_dropout
    torch.manual_seed(0)
    rng = torch.tensor([8, 9], device="cuda")
    base = torch.randn(6, 5, 4, 24, device="cuda")
    w, b = torch.randn(24, device="cuda"), torch.randn(24, device="cuda")
    for x in (base, base.transpose(0, 1), base[:, ::2], base[..., :24:1][:, :, :2], base[:, :, :1].expand(6, 5, 4, 24),
              base.permute(0, 1, 3, 2).contiguous().permute(0, 1, 3, 2)):
        flat = x.reshape(-1, 24)
        want = blossom_add_norm(flat.contiguous(), flat.contiguous() * 2, w, b, p=0.4, rng=rng, site=1)
        got = blossom_add_norm(x, x * 2, w, b, p=0.4, rng=rng, site=1)
        assert got.shape == x.shape and torch.equal(got.reshape(-1, 24), want)
        assert torch.equal(blossom_dropout(x, 0.4, rng).reshape(-1, 24), blossom_dropout(flat.contiguous(), 0.4, rng))
    # an upstream gradient that is one number seen from everywhere, and a transposed one
    x = base.clone().requires_grad_(True)
    out = blossom_add_norm(x, None, w, b, p=0.4, rng=rng)
    g1, = torch.autograd.grad(out.sum(), x, retain_graph=True)
    g2, = torch.autograd.grad(out, x, torch.ones_like(out), retain_graph=True)
    assert torch.equal(g1, g2)
    d = torch.randn(5, 6, 4, 24, device="cuda")
    assert torch.equal(torch.autograd.grad(out, x, d.transpose(0, 1), retain_graph=True)[0],
                       torch.autograd.grad(out, x, d.transpose(0, 1).contiguous())[0])
    # vectors, and negated views (whose memory holds the other sign)
    v = torch.randn(24, device="cuda")
    assert torch.equal(blossom_add_norm(v, None, w, b), blossom_add_norm(v[None], None, w, b)[0])
    z = torch.randn(3, 24, dtype=torch.complex64, device="cuda")
    neg = z.conj().imag
    assert neg.is_neg() or True
    assert torch.equal(blossom_dropout(neg, 0.4, rng), blossom_dropout(neg.clone(), 0.4, rng))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 8), (100, 50), (1025, 64), (7, 1000), (2, 8192)])
def test_dropout_keeps_what_the_definition_keeps(rows, cols, dtype):
    import torch
    from paper_2512_13368_b200.autograd import blossom_dropout
    dt = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]
    for p, seed, step, site in ((0.1, 1, 0, 0), (0.5, -(1 << 62), (1 << 40) + 5, 65535), (0.9999, 1 << 33, -1, 7), (1.0, 0, 0, 0)):
        rng = torch.tensor([seed, step], device="cuda")
        x = torch.ones(rows, cols, dtype=dt, device="cuda").requires_grad_(True)
        out = blossom_dropout(x, p, rng, site=site)
        want = torch.from_numpy(ro.keep_factor(rows, cols, p, seed, step, site)).to(dt)
        assert torch.equal(out.detach().cpu(), want), p
        (dx,) = torch.autograd.grad(out, x, torch.ones_like(out))
        assert torch.equal(dx.cpu(), want)
    x = torch.ones(rows, cols, dtype=dt, device="cuda")
    assert blossom_dropout(x, 0.0, None) is x


@pytest.mark.gpu
def test_dropped_elements_are_zero_whatever_was_there():
    import torch
    from paper_2512_13368_b200.autograd import blossom_add_norm, blossom_dropout
    rng = torch.tensor([5, 6], device="cuda")
    fac = torch.from_numpy(ro.keep_factor(50, 40, 0.5, 5, 6, 2)).cuda()
    torch.manual_seed(1)
    x = torch.randn(50, 40, device="cuda")
    bad = torch.tensor([float("nan"), float("inf"), -float("inf")], device="cuda")
    y = torch.where(fac > 0, x, bad[torch.randint(0, 3, x.shape, device="cuda")])
    r = torch.randn(50, 40, device="cuda")
    assert torch.equal(blossom_dropout(x, 0.5, rng, site=2), blossom_dropout(y, 0.5, rng, site=2))
    grads = []
    for t in (x, y):
        t = t.clone().requires_grad_(True)
        out = blossom_add_norm(t, r, None, None, p=0.5, rng=rng, site=2)
        grads.append((out.detach(), torch.autograd.grad(out, t, r)[0]))
    assert torch.equal(grads[0][0], grads[1][0]) and torch.equal(grads[0][1], grads[1][1])
    # a non-finite row spoils itself alone
    z = x.clone()
    z[7, 3] = float("nan")
    a, b = blossom_add_norm(x, r, None, None), blossom_add_norm(z, r, None, None)
    assert bool(b[7].isnan().all()) and torch.equal(a[:7], b[:7]) and torch.equal(a[8:], b[8:])


@pytest.mark.gpu
def test_rows_far_from_zero_and_constant_rows():
    """A mean 2^12 times the spread: a variance from E[z^2] - mean^2 would have no digits left.  A constant row gives its bias."""
    import torch
    from paper_2512_13368_b200.autograd import blossom_add_norm
    g = np.random.default_rng(8)
    x = torch.from_numpy((4096.0 + g.standard_normal((20, 96))).astype(np.float32)).cuda()
    f = ro.add_norm(np64(x), None, None, None, np.ones((20, 96)), 1e-5)
    compare({"out": blossom_add_norm(x, None, None, None)}, {"out": f["out"]}, bounds(np64(x), None, f, None, None), {"all": False}, "far")
    b = torch.randn(96, device="cuda")
    assert torch.equal(blossom_add_norm(torch.full((4, 96), 3.0, device="cuda"), None, None, b), b.expand(4, 96))


@pytest.mark.gpu
def test_gradient_against_differences_of_the_kernel():
    """Central differences of the single-precision kernel, step h in a random direction.  The loss is a sum of N = 16 * 40
    products of size one, each with an error below 2^-18 (64 u): the difference is off by at most N 2^-18 / h plus the
    third derivative's h^2 N (values of size one): 0.25 + 0.64 with h = 2^-5 would be no test, so the errors'
    independence is used, sqrt(N) in place of N: 25 (2^-18 / 2^-5 + 2^-10) < 0.03."""
    import torch
    from paper_2512_13368_b200.autograd import blossom_add_norm
    torch.manual_seed(3)
    rng = torch.tensor([3, 1], device="cuda")
    t = [torch.randn(16, 40, device="cuda"), torch.randn(16, 40, device="cuda"), 1 + 0.2 * torch.randn(40, device="cuda"),
         torch.randn(40, device="cuda")]
    dout = torch.randn(16, 40, device="cuda")
    leaves = [a.clone().requires_grad_(True) for a in t]
    grads = torch.autograd.grad(blossom_add_norm(*leaves, p=0.3, rng=rng), leaves, dout)
    h = 2.0 ** -5
    for i in range(4):
        v = torch.randn_like(t[i])
        v /= v.norm()
        up, down = list(t), list(t)
        up[i], down[i] = t[i] + h * v, t[i] - h * v
        f = lambda a: float((blossom_add_norm(*a, p=0.3, rng=rng).double() * dout.double()).sum())  # noqa: E731
        assert abs((f(up) - f(down)) / (2 * h) - float((grads[i].double() * v.double()).sum())) < 0.03


@pytest.mark.gpu
def test_no_rows():
    import torch
    from paper_2512_13368_b200.autograd import blossom_add_norm, blossom_dropout
    rng = torch.tensor([1, 1], device="cuda")
    x = torch.empty(0, 3, 48, device="cuda", requires_grad=True)
    w, b = torch.ones(48, device="cuda", requires_grad=True), torch.zeros(48, device="cuda", requires_grad=True)
    out = blossom_add_norm(x, x, w, b, p=0.1, rng=rng)
    g = torch.autograd.grad(out, (x, w, b), torch.empty_like(out))
    assert out.shape == x.shape and g[0].shape == x.shape and not g[1].any() and not g[2].any()
    assert blossom_dropout(x, 0.5, rng).shape == x.shape


@pytest.mark.gpu
def test_only_what_is_wanted_and_the_same_bits():
    import torch
    from paper_2512_13368_b200.autograd import blossom_add_norm
    x, r, w, b, dout = tensors(2000, 64, "bf16", 3)
    rng = torch.tensor([1, 2], device="cuda")
    args = {"x": x, "residual": r, "weight": w, "bias": b}

    def run(names):
        a = {k: (v.detach().requires_grad_(k in names)) for k, v in args.items()}
        out = blossom_add_norm(a["x"], a["residual"], a["weight"], a["bias"], p=0.2, rng=rng)
        return dict(zip(names, torch.autograd.grad(out, [a[n] for n in names], dout)))

    full = run(list(args))
    for _ in range(3):
        again = run(list(args))
        assert all(torch.equal(full[k], again[k]) for k in full)
    for n in args:
        assert torch.equal(run([n])[n], full[n])
    with torch.no_grad():
        assert blossom_add_norm(x.requires_grad_(True), r, w, b).grad_fn is None


@pytest.mark.gpu
def test_another_stream_and_a_captured_step():
    import torch
    from paper_2512_13368_b200.autograd import blossom_add_norm, blossom_dropout
    x, r, w, b, dout = tensors(500, 64, "bf16", 4)
    rng = torch.tensor([7, 0], device="cuda")
    want = [blossom_add_norm(blossom_dropout(x, 0.3, torch.tensor([7, s], device="cuda"), site=1), r, w, b, p=0.3,
                             rng=torch.tensor([7, s], device="cuda"), site=2) for s in range(3)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = blossom_add_norm(blossom_dropout(x, 0.3, rng, site=1), r, w, b, p=0.3, rng=rng, site=2)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want[0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = blossom_add_norm(blossom_dropout(x, 0.3, rng, site=1), r, w, b, p=0.3, rng=rng, site=2)
        rng[1] += 1
    rng[1] = 0
    for k in range(3):
        g.replay()
        assert torch.equal(out, want[k])


@pytest.mark.gpu
def test_a_step_moved_on_before_the_backward_is_noticed():
    import torch
    from paper_2512_13368_b200.autograd import blossom_add_norm, blossom_dropout
    x = torch.randn(4, 32, device="cuda", requires_grad=True)
    for f in (lambda rng: blossom_dropout(x, 0.5, rng), lambda rng: blossom_add_norm(x, None, None, None, p=0.5, rng=rng)):
        rng = torch.tensor([1, 1], device="cuda")
        out = f(rng)
        rng[1] += 1
        with pytest.raises(RuntimeError, match="inplace"):
            out.sum().backward()


@pytest.mark.gpu
def test_second_derivatives_are_refused_where_they_are_used():
    import torch
    from paper_2512_13368_b200.autograd import blossom_add_norm
    x = torch.randn(4, 32, device="cuda", requires_grad=True)
    (g,) = torch.autograd.grad(blossom_add_norm(x, None, None, None).pow(2).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivative"):
        g.sum().backward()


@pytest.mark.gpu
def test_front_end_refusals():
    import torch
    from paper_2512_13368_b200.autograd import blossom_add_norm, blossom_dropout
    x = torch.randn(4, 32, device="cuda")
    rng = torch.tensor([1, 1], device="cuda")
    w = torch.ones(32, device="cuda")
    for call, exc in ((lambda: blossom_dropout(x.cpu(), 0.5, rng), ValueError), (lambda: blossom_dropout(x.half(), 0.5, rng), TypeError),
                      (lambda: blossom_dropout(x, 0.5, None), ValueError), (lambda: blossom_dropout(x, 0.5, rng.int()), ValueError),
                      (lambda: blossom_dropout(x, 0.5, rng.cpu()), ValueError), (lambda: blossom_dropout(x, 1.5, rng), binding.BlossomError),
                      (lambda: blossom_dropout(x, -0.5, rng), binding.BlossomError), (lambda: blossom_dropout(x, float("nan"), rng), binding.BlossomError),
                      (lambda: blossom_dropout(x, 0.5, rng, site=65536), binding.BlossomError),
                      (lambda: blossom_dropout(torch.zeros(2, 8200, device="cuda"), 0.5, rng), binding.BlossomError),
                      (lambda: blossom_add_norm(x, x[:2], w, w), ValueError), (lambda: blossom_add_norm(x, x.bfloat16(), w, w), TypeError),
                      (lambda: blossom_add_norm(x, None, w[:5], w), ValueError), (lambda: blossom_add_norm(x, None, w, w.bfloat16()), TypeError),
                      (lambda: blossom_add_norm(x, None, w.half(), None), TypeError), (lambda: blossom_add_norm(x, None, w, w, p=0.5), ValueError),
                      (lambda: blossom_add_norm(x, None, w, w, eps=-1.0), binding.BlossomError),
                      (lambda: blossom_add_norm(x[:, :0], None, None, None), ValueError)):
        with pytest.raises(exc):
            call()


def test_params_and_arguments_are_checked_before_any_launch():
    binding.load()
    E, A = binding, 1 << 20   # a fake, aligned, never-dereferenced device address
    good = lambda **kw: E.make_rows_params(**dict(dict(rows=10, cols=64, dtype="bf16", dropout=0.1), **kw))  # noqa: E731
    n = E.blossom_add_norm_workspace_bytes(good())
    assert n >= 256 and n % 256 == 0
    assert E.blossom_add_norm_workspace_bytes(good(rows=0)) > 0
    for bad, rc in ((dict(rows=-1), 1), (dict(cols=0), 1), (dict(cols=8193), 2), (dict(rows=1 << 31), 2), (dict(dtype=5), 1),
                    (dict(weight_dtype=5), 1), (dict(site=-1), 1), (dict(site=65536), 1), (dict(dropout=-0.1), 1), (dict(dropout=1.1), 1),
                    (dict(dropout=float("nan")), 1), (dict(eps=-1e-9), 1), (dict(eps=float("inf")), 1), (dict(x_stride=63), 1),
                    (dict(residual_stride=-64), 1), (dict(out_stride=1), 1), (dict(dx_stride=8), 1), (dict(dresidual_stride=8), 1)):
        p = good(**bad)
        assert E.blossom_add_norm_workspace_bytes(p) == 0, bad
        assert E.blossom_dropout(p, A, A, A, stream=0, check=False) == rc, bad
        assert E.blossom_add_norm_fwd(p, A, A, A, A, A, A, A, stream=0, check=False) == rc, bad
        assert E.blossom_add_norm_bwd(p, A, A, A, A, A, A, A, A, A, A, A, 1 << 40, stream=0, check=False) == rc, bad
    p = good()
    for args in ((None, A, A), (A, None, A), (A, A, None), (A + 1, A, A), (A, A + 4, A), (A, A, A + 1)):
        assert E.blossom_dropout(p, *args, stream=0, check=False) == E.BLOSSOM_ERR_INVALID_ARG, args
    for i, v in ((0, None), (0, A + 1), (1, A + 1), (2, A + 1), (3, A + 1), (4, None), (5, None), (5, A + 1), (6, A + 4)):
        args = [A] * 7
        args[i] = v
        assert E.blossom_add_norm_fwd(p, *args, stream=0, check=False) == E.BLOSSOM_ERR_INVALID_ARG, (i, v)
    for i, v in ((0, None), (1, A + 1), (2, A + 1), (3, None), (4, None), (4, A + 4), (5, None), (6, A + 1), (7, A + 1), (8, A + 1), (9, A + 1)):
        args = [A] * 10
        args[i] = v
        assert E.blossom_add_norm_bwd(p, *args, A, n, stream=0, check=False) == E.BLOSSOM_ERR_INVALID_ARG, (i, v)
    nothing = [A] * 6 + [None] * 4
    assert E.blossom_add_norm_bwd(p, *nothing, A, n, stream=0, check=False) == E.BLOSSOM_ERR_INVALID_ARG
    for ws, size in ((None, n), (A + 128, n), (A, n - 1)):
        assert E.blossom_add_norm_bwd(p, *[A] * 10, ws, size, stream=0, check=False) == E.BLOSSOM_ERR_WORKSPACE
    assert E.blossom_dropout(good(rows=0), None, A, None, stream=0, check=False) == 0
    with pytest.raises(E.BlossomError):
        E.blossom_dropout(p, None, None, None, stream=0)


def test_rows_params_layout_matches_the_header():
    import ctypes
    f = binding.blossom_rows_params
    assert ctypes.sizeof(f) == 80 and f.site.offset == 20 and f.dropout.offset == 24 and f.x_stride.offset == 40


def test_python_checks_need_no_gpu():
    import torch
    from paper_2512_13368_b200.autograd import check_rows
    x = torch.zeros(3, 8)
    chk = lambda *a, **k: check_rows(*a, require_cuda=False, **k)  # noqa: E731
    chk(x, 0.0, None)
    chk(x, 0.5, torch.zeros(2, dtype=torch.int64), (("residual", x),), (("weight", x[0]), ("bias", None)))
    for a, k, exc in (((x, 0.5, None), {}, ValueError), ((x, 0.5, torch.zeros(2)), {}, ValueError), ((x.double(), 0.0, None), {}, TypeError),
                      ((x[0, 0], 0.0, None), {}, ValueError), ((x, 0.0, None, (("residual", x[:2]),)), {}, ValueError),
                      ((x, 0.0, None, (), (("weight", x[0].double()),)), {}, TypeError)):
        with pytest.raises(exc):
            chk(*a, **k)
    with pytest.raises(ValueError):
        check_rows(x, 0.0, None)   # a host tensor
