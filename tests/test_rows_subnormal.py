"""Dropout of subnormal numbers: a kept one is scaled like any other."""
import numpy as np
import pytest

from oracle import rows_oracle as ro


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("cols", [64, 50, 7, 1024])
def test_kept_subnormal_elements_are_scaled(cols, dtype):
    """fp32: the product rounded once, which double precision holds exactly before; bf16: that product rounded once more."""
    import torch
    from paper_2512_13368_b200.autograd import blossom_dropout
    g = np.random.default_rng(cols)
    x = (g.standard_normal((40, cols)) * 2.0 ** g.integers(-148, -120, (40, cols))).astype(np.float32)
    x = torch.from_numpy(x)
    if dtype == "bf16":
        x = x.bfloat16()
    small = (x != 0) & (x.float().abs() < 2.0 ** -126)
    assert small.float().mean() > 0.25   # (in bf16 the smallest are zeros)
    fac = ro.keep_factor(40, cols, 0.3, 5, 6, 1)
    scale = float(np.float32(fac.max()))
    want = np.where(fac > 0, x.double().numpy() * scale, 0.0).astype(np.float32)
    want = torch.from_numpy(want).to(x.dtype)
    assert ((want != 0) & (want.float().abs() < 2.0 ** -126)).any()
    leaf = x.cuda().requires_grad_(True)
    out = blossom_dropout(leaf, 0.3, torch.tensor([5, 6], device="cuda"), site=1)
    (dx,) = torch.autograd.grad(out, leaf, x.cuda())
    assert torch.equal(out.detach().cpu(), want) and torch.equal(dx.cpu(), want)
