"""GELU and its derivative: the terms of the logit of Phi in double precision, and the kernels' results over the arguments."""
import os
import re

import numpy as np
import pytest

from oracle import linear_oracle as lo
from paper_2512_13368_b200 import binding

F32, BF16 = 2.0 ** -24, 2.0 ** -8   # half a step, relative


def terms():
    """{name: numbers} of linear.cuh, as single precision adds them up."""
    with open(os.path.join(os.path.dirname(binding.__file__), "csrc", "linear.cuh")) as f:
        text = f.read()
    lists = {}
    for name in ("value", "value_rest", "both", "both_rest"):
        numbers = re.search(rf"constexpr float {name}\[\d\] = \{{(.*?)\}}", text, re.S).group(1)
        lists[name] = np.array([float(v.strip().rstrip("f")) for v in numbers.split(",")], dtype=np.float32)
    res = {}
    for name in ("value", "both"):
        t = lists[name + "_rest"].copy()
        t[:len(lists[name])] = lists[name] + t[:len(lists[name])]
        res[name] = t.astype(np.float64)
    return res


def value_of(t, x):
    low = np.maximum(x, -6.0)
    return low / (1.0 + np.exp(-low * np.polyval(t[::-1], low * low)))


def test_the_terms():
    """Nine terms for bf16 results: within 9e-4 of x Phi(x) relative to it down to x = -6, an absolute error of 7.6e-8; seven for
    results in single precision, 7.1e-8, and for the derivative Phi(x) + x phi(x), in which Phi alone is theirs: 4.8e-8.  From
    x = -6 down all of it is nearer to 0 than 6e-9 (the value) and 4e-8 (the derivative)."""
    t = terms()
    assert len(t["value"]) == 9 and len(t["both"]) == 7
    x = np.linspace(-6.0, 6.0, 240001)
    want, _ = lo.activation("gelu", x)
    got = value_of(t["value"], x)
    assert np.abs(got - want).max() < 7.6e-8 and (np.abs(got - want)[x < 0] <= 9e-4 * np.abs(want)[x < 0]).all()
    assert np.abs(value_of(t["both"], x) - want).max() < 7.1e-8
    phi = 1.0 / (1.0 + np.exp(-x * np.polyval(t["both"][::-1], x * x)))
    assert np.abs(phi - lo._cdf(x)).max() < 4.8e-8
    # beyond: the value is not cut on the right, where every term counts; the derivative is cut at 6
    far = np.concatenate([np.linspace(6.0, 100.0, 94001), 10.0 ** np.arange(2, 39)])
    with np.errstate(over="ignore", invalid="ignore"):
        assert (np.polyval(t["value"][::-1], far[far < 1e10] ** 2) > 1.5).all() and t["value"][-1] > 0
        assert (np.polyval(t["both"][::-1], far[far < 1e10] ** 2) > 1.5).all() and t["both"][-1] > 0
    assert np.abs(value_of(t["value"], np.array([-6.0]))) < 6.01e-9
    edge = lo.activation("gelu", np.array([-6.0, 6.0]))[1]
    assert abs(edge[0]) < 4e-8 and abs(edge[1] - 1.0) < 4e-8


def layer(x, w, act, rows, dtype):
    """x a number, w [outs]: every row of x the same, so that the argument of out n is x w_n; (out, dbias / rows)."""
    import torch
    outs = len(w)
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    xs = torch.full((rows, 1), x, dtype=dt, device="cuda")
    wt = torch.from_numpy(w).to(dt).cuda()[:, None]
    b, dout = torch.zeros(outs, dtype=dt, device="cuda"), torch.ones(rows, outs, dtype=dt, device="cuda")
    p = binding.make_linear_params(rows, 1, outs, dtype, act)
    ws = torch.empty(binding.blossom_linear_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    out, db = torch.empty_like(dout), torch.empty_like(b)
    binding.blossom_linear_fwd(p, xs, wt, b, None, out, ws)
    binding.blossom_linear_bwd(p, xs, None, wt, b, dout, None, None, db, ws)
    assert binding.blossom_device_status(ws) == 0
    assert torch.equal(out, out[:1].expand(rows, outs))
    return out[0].double().cpu().numpy(), db.double().cpu().numpy() / rows


def every_bf16(least, most):
    v = np.arange(65536, dtype=np.uint32) << 16
    v = v.view(np.float32)
    with np.errstate(invalid="ignore"):
        return v[(np.abs(v) >= least) & (np.abs(v) <= most)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 4, 128, 300])
@pytest.mark.parametrize("outs", [64, 200, 4000])
def test_values_relative_to_themselves(rows, outs):
    """bf16: off by half a step and 9e-4 of the value from x = -6 on, by 6e-9 below; 2^-18 besides, for the logit of up to 30 in
    single precision and its exponential."""
    w = every_bf16(2.0 ** -40, 1e4)
    for i in range(0, len(w), outs):
        part = w[i:i + outs]
        got, _ = layer(1.0, part, "gelu", rows, "bf16")
        x = part.astype(np.float64)
        want = lo.activation("gelu", x)[0]
        tol = (BF16 * (1 + 2.0 ** -9) + 9e-4 + 2.0 ** -18) * np.abs(want) + np.where(x < -6.0, 6.1e-9, 0.0)
        bad = ~(np.abs(got - want) <= tol)
        assert not bad.any(), (x[bad][:4], got[bad][:4], want[bad][:4])


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 16, 128, 300])
@pytest.mark.parametrize("outs", [64, 4000])
def test_values_in_single_precision(rows, outs):
    """Of the value: the sum in the denominator, the shared reciprocal's product, the reciprocal (two halves of a step), and the
    products behind it, six halves of a step; 7.1e-8 of the polynomial; and through the change of Phi the logit, two roundings a
    term of the powers and the sums, and the exponential, 2^-22."""
    rng = np.random.default_rng(0)
    t = np.abs(terms()["both"])
    w = np.concatenate([every_bf16(2.0 ** -40, 1e4), rng.uniform(-8, 8, 5000).astype(np.float32)])
    for i in range(0, len(w), outs):
        got, _ = layer(1.0, w[i:i + outs], "gelu", rows, "fp32")
        x = w[i:i + outs].astype(np.float64)
        want = lo.activation("gelu", x)[0]
        low = np.clip(x, -6.0, 6.0)
        logit = np.abs(low) * sum((2 * k + 4) * c * low ** (2 * k) for k, c in enumerate(t)) * F32
        cdf = lo._cdf(low)
        tol = 6 * F32 * np.abs(want) + 7.1e-8 + np.abs(low) * cdf * (1 - cdf) * (logit + 2.0 ** -22)
        bad = ~(np.abs(got - want) <= tol)
        assert not bad.any(), (x[bad][:4], got[bad][:4], want[bad][:4])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows", [1, 64, 512])
@pytest.mark.parametrize("outs", [64, 4000])
def test_derivatives_near_their_zero(rows, outs, dtype):
    """Where the derivative is 0 (x = -0.7518) a result in bf16 has steps small enough for the error of the derivative itself to
    show: 4.8e-8 of Phi; its roundings and those of phi, of the sum and of the argument, 16 halves of a step in all; two bf16 of 2^-16 between the products,
    and the result's rounding.  Powers of two of rows: their sums are exact but for the cuts, 2^-23 a step of 16."""
    rng = np.random.default_rng(1)
    w = np.concatenate([every_bf16(0.7, 0.8), -0.7518 + 0.01 * rng.standard_normal(4000).astype(np.float32)]).astype(np.float32)
    w = (w.view(np.uint32) & 0xffff0000).view(np.float32) if dtype == "bf16" else w   # (exact in the type)
    x1 = 1.0 + 2.0 ** -7
    u = BF16 if dtype == "bf16" else F32
    for x in (1.0, x1):
        for i in range(0, len(w), outs):
            _, got = layer(x, w[i:i + outs], "gelu", rows, dtype)
            want = lo.activation("gelu", x * w[i:i + outs].astype(np.float64))[1]
            tol = (u + (2.0 ** -16 if dtype == "bf16" else 2 * F32) + (rows / 16 + 8) * 2.0 ** -23) * np.abs(want) + 4.8e-8 + 16 * F32
            bad = ~(np.abs(got - want) <= 1.01 * tol)
            assert not bad.any(), (w[i:i + outs][bad][:4], got[bad][:4], want[bad][:4])
