"""What is no number, and infinities, in one column of a linear layer: the other columns' results keep their bits."""
import pytest

from paper_2512_13368_b200 import binding

# few rows; the narrow layers' backward in one kernel; products of any size by TMA and by plain loads; odd numbers of outs
SHAPES = [(3, 64, 64), (12, 300, 70), (5, 64, 64), (64, 256, 64), (200, 64, 256), (333, 256, 63), (190, 50, 71), (300, 512, 640), (130, 520, 333)]


def tensors(rows, cols, outs, dtype):
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows)
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    return [(torch.randn(*s, generator=g, device="cuda") * f).to(dt)
            for s, f in (((rows, cols), 1.0), ((outs, cols), cols ** -0.5), ((outs,), 0.3), ((rows, outs), 1.0))]


def step(x, w, b, dout, act):
    import torch
    rows, cols = x.shape
    p = binding.make_linear_params(rows, cols, w.shape[0], "fp32" if x.dtype == torch.float32 else "bf16", act)
    ws = torch.empty(binding.blossom_linear_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    out, dx, dw, db = (torch.full_like(t, 7.0) for t in (dout, x, w, b))
    binding.blossom_linear_fwd(p, x, w, b, None, out, ws)
    assert binding.blossom_device_status(ws) == 0
    binding.blossom_linear_bwd(p, x, None, w, b, dout, dx, dw, db, ws)
    assert binding.blossom_device_status(ws) == 0
    return dict(out=out, dx=dx, dw=dw, db=db)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("rows,cols,outs", SHAPES)
def test_a_column_that_is_no_number_stays_alone(rows, cols, outs, act, dtype):
    """A NaN in one bias, or in one row of the weight: its column of the output, its row of dweight and its dbias (where the slope
    is one too), and nothing of another column."""
    import torch
    x, w, b, dout = tensors(rows, cols, outs, dtype)
    clean = step(x, w, b, dout, act)
    for n in sorted({0, 1, outs // 2, outs // 2 + 1, outs - 1}):
        keep = torch.arange(outs, device="cuda") != n
        for where in ("bias", "weight"):
            w1, b1 = w.clone(), b.clone()
            (b1 if where == "bias" else w1[n])[n if where == "bias" else cols // 2] = float("nan")
            got = step(x, w1, b1, dout, act)
            assert torch.equal(got["out"][:, keep], clean["out"][:, keep]), (n, where)
            assert torch.equal(got["dw"][keep], clean["dw"][keep]) and torch.equal(got["db"][keep], clean["db"][keep]), (n, where)
            assert bool(got["out"][:, n].isnan().all()), (n, where)
            if act in ("gelu", "silu"):
                assert bool(got["dw"][n].isnan().all()) and bool(got["db"][n].isnan()), (n, where)


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("rows,cols,outs", SHAPES)
def test_an_infinite_row_has_the_limits(rows, cols, outs, act):
    """bf16: arguments of plus and minus infinity, in the last of an odd number of columns too, whose neighbour is not there: an
    infinity, or what the smallest arguments have."""
    import torch
    x, w, b, dout = tensors(rows, cols, outs, "bf16")
    w[:, 3] = torch.where(w[:, 3] == 0, torch.ones_like(w[:, 3]), w[:, 3])
    clean = step(x, w, b, dout, act)
    x = x.clone()
    x[1, 3] = float("inf")
    got = step(x, w, b, dout, act)
    up = w[:, 3] > 0
    assert bool((got["out"][1][up] == float("inf")).all()) and bool((got["out"][1][~up].abs() <= 6e-9).all())
    keep = torch.arange(rows, device="cuda") != 1
    assert torch.equal(got["out"][keep], clean["out"][keep]) and torch.equal(got["dx"][keep], clean["dx"][keep])
    # its slopes are 1 and 0: what reaches dx is the sum of the upstream gradients of the first
    want = (dout[1].double() * up) @ w.double()
    size = dout[1].double().abs() @ w.double().abs()
    assert bool(((got["dx"][1].double() - want).abs() <= 2.0 ** -8 * want.abs() + (outs + 64) * 2.0 ** -23 * size + 1e-6 * size).all())


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
@pytest.mark.parametrize("rows,cols,outs", SHAPES)
def test_an_infinite_upstream_gradient(rows, cols, outs, act):
    """bf16: one infinite element makes its row of dx, its row of dweight and its dbias infinite, of the signs of the terms, and
    nothing else."""
    import torch
    x, w, b, dout = tensors(rows, cols, outs, "bf16")
    x, w = (torch.where(t == 0, torch.ones_like(t), t) for t in (x, w))
    clean = step(x, w, b, dout, act)
    for n, big in ((0, float("inf")), (outs // 2 + 1, float("-inf")), (outs - 1, 3.3895e38)):
        d = dout.clone()
        d[1, n] = big
        got = step(x, w, b, d, act)
        p = x[1].double() @ w[n].double() + b[n].double()
        s = torch.sigmoid(p)
        slope = {"none": 1.0, "silu": float(s * (1 + p * (1 - s))),
                 "gelu": float(0.5 * torch.special.erfc(-p / 2 ** 0.5) + p * torch.exp(-p * p / 2) * 0.3989422804)}[act]
        assert abs(slope) > 1e-3
        others, rest = torch.arange(outs, device="cuda") != n, torch.arange(rows, device="cuda") != 1
        assert torch.equal(got["dw"][others], clean["dw"][others]) and torch.equal(got["db"][others], clean["db"][others])
        assert torch.equal(got["dx"][rest], clean["dx"][rest])
        if big == big + 1 and abs(big) > 3.4e38:
            sign = slope * big
            assert torch.equal(got["db"][n].float(), torch.tensor(sign, device="cuda"))
            assert torch.equal(got["dw"][n].float(), sign * x[1].float()) and torch.equal(got["dx"][1].float(), sign * w[n].float())
        else:   # the largest bf16: products with it may pass the largest number, but none is no number
            assert not bool(got["db"][n].isnan()) and not bool(got["dw"][n].isnan().any()) and not bool(got["dx"][1].isnan().any())
