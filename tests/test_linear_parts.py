"""The upstream gradient behind an activation between the products of large bf16 layers: a sum of two bf16, whatever the size."""
import numpy as np
import pytest

from oracle import linear_oracle as lo
from paper_2512_13368_b200 import binding

F32, BF16 = 2.0 ** -24, 2.0 ** -8   # half a step, relative


def half_step(v):
    """Of a bf16 result: half a step of the power of two at or below v."""
    import torch
    return torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -100))) - 8)


def backward(x, w, b, dout, act):
    import torch
    rows, cols = x.shape
    outs = w.shape[0]
    p = binding.make_linear_params(rows, cols, outs, "bf16", act)
    ws = torch.full((binding.blossom_linear_workspace_bytes(p),), 0xa5, dtype=torch.uint8, device="cuda")
    dx, dw, db = (torch.full_like(t, 7.0) for t in (x, w, b))
    binding.blossom_linear_bwd(p, x, None, w, b, dout, dx, dw, db, ws)
    assert binding.blossom_device_status(ws) == 0
    return dx, dw, db


LARGE = [(8192, 1024, 4096), (8191, 1024, 4096), (33000, 2048, 512), (300, 520, 640)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,outs", LARGE)
def test_sums_of_one_slope(rows, cols, outs):
    """The activation's arguments are the biases, so that a column of the upstream gradient is one number c between 1 and 1.03:
    rounded to bf16, alone, it would be off by up to 2^-8, and so would the sums: a whole step of theirs where they begin with
    1.95.  In two parts it is off by 2^-16.  The slope's own error is 4.4e-5 at most, and sums that are cut lose 2^-23 a step of
    16."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows)
    there = int(1.951 * 2 ** int(np.log2(rows / 2)))     # rows with a gradient
    assert there <= rows
    x, w = torch.zeros(rows, cols, device="cuda"), torch.zeros(outs, cols, device="cuda")
    x[:there, 0] = 1.0
    for _ in range(3):                                   # three ones down a column of the weight, but for the first
        w[torch.randint(0, outs, (cols - 1,), generator=g, device="cuda"), torch.arange(1, cols, device="cuda")] += 1.0
    dout = torch.zeros(rows, outs, device="cuda")
    dout[:there] = 1.0
    b = 0.75 + 0.08 * torch.rand(outs, generator=g, device="cuda")
    x, w, b, dout = (t.bfloat16() for t in (x, w, b, dout))
    dx, dw, db = backward(x, w, b, dout, "gelu")
    c = torch.from_numpy(lo.activation("gelu", b.double().cpu().numpy())[1]).cuda()
    assert float(c.min()) >= 0.99 and float(c.max()) <= 1.04

    def good(got, want):
        off = (got.double() - want).abs()
        tol = half_step(want) + (4.4e-5 + 2.0 ** -16 + (rows / 16 + 64) * 2.0 ** -23) * want.abs()
        assert bool((off <= 1.001 * tol).all()), (int((off > 1.001 * tol).sum()), float((off / tol).max()))

    good(db, there * c)
    good(dw[:, 0], there * c)
    good(dx[:there], (c @ w.double()).expand(there, cols))
    assert bool((dx[there:] == 0).all()) and bool((dw[:, 1:] == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("rows,cols,outs", LARGE)
def test_gradients_of_large_layers(rows, cols, outs, act):
    """Rows of dx, rows of dweight and dbias against 64 bits; the bounds are those of smaller layers: k + 4 roundings or cuts of
    sums over k terms, the slope's error, two parts of the upstream gradient, and the result's rounding."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)

    def t(*s, std=1.0):
        return (torch.randn(*s, generator=g, device="cuda") * std).bfloat16()

    x, w, b, dout = t(rows, cols), t(outs, cols, std=cols ** -0.5), t(outs, std=0.3), t(rows, outs)
    dx, dw, db = backward(x, w, b, dout, act)
    x, w, b, dout = (v.double() for v in (x, w, b, dout))

    def behind(rows_, outs_):
        """G and what it may be off by."""
        p = x[rows_] @ w[outs_].t() + b[outs_]
        size = x[rows_].abs() @ w[outs_].abs().t() + b[outs_].abs()
        if act == "gelu":
            cdf = 0.5 * torch.special.erfc(-p / 2 ** 0.5)
            d = cdf + p * torch.exp(-p * p / 2) * (2 * np.pi) ** -0.5
        else:
            s = torch.sigmoid(p)
            d = s * (1 + p * (1 - s))
        G = dout[rows_][:, outs_] * d
        off = dout[rows_][:, outs_].abs() * (0.8 * (cols + 4) * 2 * F32 * size + 2.0 ** -14 * (1 + p.abs())) + BF16 ** 2 * G.abs()
        return G, off

    def good(got, want, tol, what):
        off = (got.double() - want).abs()
        assert bool((off <= 1.01 * tol).all()), (what, int((off > 1.01 * tol).sum()), float((off / tol).max()))

    every = slice(None)
    some = torch.tensor([0, 1, 127, 128, rows // 2, rows - 2, rows - 1], device="cuda")
    G, off = behind(some, every)
    good(dx[some], G @ w, BF16 * (G @ w).abs() + off @ w.abs() + (outs + 4) * 2 * F32 * ((G.abs() + off) @ w.abs()), "dx")
    some = torch.tensor([0, 127, 128, outs // 2, outs - 1], device="cuda")
    G, off = behind(every, some)
    for got, want, size, slack in ((dw[some], G.t() @ x, (G.abs() + off).t() @ x.abs(), off.t() @ x.abs()),
                                   (db[some], G.sum(0), (G.abs() + off).sum(0), off.sum(0))):
        good(got, want, BF16 * want.abs() + slack + (rows + 4) * 2 * F32 * size, "dweight or dbias")


def size(*a):
    return binding.blossom_linear_workspace_bytes(binding.make_linear_params(*a))


def test_how_many_steps_an_accumulator_adds_up():
    """Over rows 16384, over columns and outs 65536, those of both parts of the upstream gradient behind an activation: seen by the
    partial sums that the workspace has room for, beside the upstream gradient's parts."""
    binding.load()
    tiles = 4096 * 4096 * 4
    assert size(16384, 4096, 4096, "bf16", "none") < tiles
    assert size(8192, 4096, 4096, "bf16", "gelu") < 2 * 8192 * 4096 * 2 + tiles
    for rows, act, parts, splits in ((35000, "none", 0, 3), (17500, "gelu", 2, 3), (75000, "silu", 2, 10)):
        assert size(rows, 4096, 4096, "bf16", act) >= parts * rows * 4096 * 2 + splits * tiles, (rows, act)
    # dx over very many outs
    rows = 40000
    assert size(rows, 64, 60000, "bf16", "gelu") >= 2 * rows * 60000 * 2 + 2 * rows * 64 * 4
    assert size(400000, 64, 8200, "bf16", "none") < 2 * 400000 * 64 * 4


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,outs", [(1212416 * 2 + 777, 16, 8), (1212416 + 129, 32, 24), (9699328 + 7, 16, 8), (140000, 520, 264), (20000, 48, 40000)])
def test_long_sums_behind_an_activation(rows, cols, outs):
    """Of one sign.  An accumulator's steps, by 16 at a time, are off by 2^-23 each, and so are the terms; two parts of the
    upstream gradient leave 2^-16 of it, its slope is off by 2^-20."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(0)

    def t(*s):
        return (torch.rand(*s, generator=g, device="cuda") + 0.5).bfloat16()

    x, w, dout = t(rows, cols), t(outs, cols), t(rows, outs)
    b = torch.full((outs,), -0.9 * cols, device="cuda").bfloat16()
    dx, dw, db = backward(x, w, b, dout, "silu")

    def behind(rows_):
        p = x[rows_].double() @ w.double().t() + b.double()
        s = torch.sigmoid(p)
        return dout[rows_].double() * (s * (1 + p * (1 - s))), p

    want_w = torch.zeros(outs, cols, dtype=torch.float64, device="cuda")
    want_b = torch.zeros(outs, dtype=torch.float64, device="cuda")
    size_w, size_b = want_w.clone(), want_b.clone()
    for r0 in range(0, rows, 1 << (27 - max(outs, 64).bit_length())):
        part = slice(r0, r0 + (1 << (27 - max(outs, 64).bit_length())))
        G, _ = behind(part)
        want_w += G.t() @ x[part].double()
        want_b += G.sum(0)
        size_w += G.abs().t() @ x[part].double()
        size_b += G.abs().sum(0)
    steps = (max(16384, 2 * outs) / 16 + 64) * 2.0 ** -23 + 2.0 ** -16 + 2.0 ** -20
    # (the argument, a sum over cols of numbers of up to 2.25, is off by 2^-23 a step of its magnitudes, its slope by as much)
    argument = 0.5 * (cols + 4) * 2.0 ** -23 * 3.2 * cols
    for got, want, mag in ((dw, want_w, size_w), (db, want_b, size_b)):
        off = (got.double() - want).abs()
        tol = half_step(want) + steps * mag + argument * mag.max() * 2
        assert bool((off <= 1.01 * tol).all()), float((off / tol).max())
    at = torch.tensor([0, 1, rows // 2, rows - 1], device="cuda")
    G, _ = behind(at)
    want, mag = G @ w.double(), G.abs() @ w.double()
    off = (dx[at].double() - want).abs()
    tol = half_step(want) + steps * mag + argument * (dout[at].double() @ w.double())
    assert bool((off <= 1.01 * tol).all()), float((off / tol).max())


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["none", "silu"])
def test_how_much_is_cut_from_long_sums(act):
    """dweight of 32768 rows of one sign, over elements of all sizes between two powers of two, whose roundings cancel in the mean
    (1.7e-3 by the root of their number, 512).  1024 products of 16 rows cut less than 2^-23 of the sum so far, half the
    sum in the mean: 2^-14 in all; the terms are off by 2^-20."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(2)
    rows, cols, outs = 32768, 1024, 4096

    def t(n, c):
        return ((torch.rand(n, c, generator=g, device="cuda") + 0.5) * (1 + torch.rand(c, generator=g, device="cuda"))).bfloat16()

    x, dout = t(rows, cols), t(rows, outs)
    w, b = torch.zeros(outs, cols, device="cuda").bfloat16(), torch.full((outs,), 0.5, device="cuda").bfloat16()
    _, dw, _ = backward(x, w, b, dout, act)
    slope = lo.activation(act, np.array([0.5]))[1][0]
    some = slice(0, 256)
    want = slope * (dout[:, some].double().t() @ x.double())
    off = float((dw[some].double() / want - 1).mean())
    assert abs(off) <= 2.0 ** -14 + 2.0 ** -20 + 4 * 1.7e-3 / 512, off
