"""Residual + layer norm where something is not there: what its params say about it does not matter."""
import pytest

from paper_2512_13368_b200 import binding


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("cols", [64, 512, 1024, 4096])
def test_the_stride_of_an_absent_residual_does_not_matter(cols, dtype):
    """An odd stride would make odd addresses, which an asynchronous copy of no bytes may not have either."""
    import torch
    torch.manual_seed(cols)
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    rows = 70
    x, dout = (torch.randn(rows, cols, device="cuda").to(dt) for _ in range(2))
    w, b = (torch.randn(cols, device="cuda").to(dt) for _ in range(2))
    rng = torch.tensor([3, 4], device="cuda")

    def step(p, **strides):
        prm = binding.make_rows_params(rows, cols, dtype, dropout=p, **strides)
        out, dx, dw, db = (torch.empty_like(t) for t in (x, x, w, b))
        stats = torch.empty(rows, 2, device="cuda")
        ws = torch.empty(binding.blossom_add_norm_workspace_bytes(prm), dtype=torch.uint8, device="cuda")
        binding.blossom_add_norm_fwd(prm, x, None, w, b, rng, out, stats)
        binding.blossom_add_norm_bwd(prm, x, None, w, rng, stats, dout, dx, None, dw, db, ws)
        return out, dx, dw, db, stats

    for p in (0.0, 0.3, 1.0):
        want = step(p)
        for stride in (cols + 1, cols + 3, (1 << 62) + 1):
            assert all(torch.equal(a, c) for a, c in zip(step(p, residual_stride=stride, dresidual_stride=stride), want)), (p, stride)
