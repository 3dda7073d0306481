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


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,dtype", [(70, 64, "bf16"), (33, 1000, "fp32"), (0, 64, "bf16")])
def test_no_workspace_without_a_gradient_of_weight_or_bias(rows, cols, dtype):
    import torch
    torch.manual_seed(cols)
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    x, r, dout = (torch.randn(rows, cols, device="cuda").to(dt) for _ in range(3))
    w = torch.randn(cols, device="cuda").to(dt)
    rng = torch.tensor([3, 4], device="cuda")
    prm = binding.make_rows_params(rows, cols, dtype, dropout=0.2)
    ws = torch.empty(binding.blossom_add_norm_workspace_bytes(prm), dtype=torch.uint8, device="cuda")
    out, stats, want, wres, dx, dres = (torch.empty_like(t) for t in (x, torch.empty(rows, 2, device="cuda"), x, x, x, x))
    dw, db = torch.empty_like(w), torch.empty_like(w)
    binding.blossom_add_norm_fwd(prm, x, r, w, None, rng, out, stats)
    binding.blossom_add_norm_bwd(prm, x, r, w, rng, stats, dout, want, wres, dw, db, ws)
    binding.blossom_add_norm_bwd(prm, x, r, w, rng, stats, dout, dx, dres, None, None, None)
    assert torch.equal(dx, want) and torch.equal(dres, wres)
    for one in ((dw, None), (None, db)):
        if rows:
            rc = binding.blossom_add_norm_bwd(prm, x, r, w, rng, stats, dout, dx, dres, *one, None, check=False)
            assert rc == binding.BLOSSOM_ERR_WORKSPACE


def test_no_workspace_is_one_of_no_bytes():
    """The refusal is the library's, before any launch, not an error of the binding."""
    binding.load()
    E, A = binding, 1 << 20
    p = E.make_rows_params(10, 64, "bf16", dropout=0.1)
    assert E.blossom_add_norm_bwd(p, *[A] * 10, None, stream=0, check=False) == E.BLOSSOM_ERR_WORKSPACE
    q = E.make_loss_params(10, 64, 100, 5, "bf16")
    assert E.blossom_sampled_loss_fwd(q, *[A] * 7, None, stream=0, check=False) == E.BLOSSOM_ERR_WORKSPACE
    assert E.blossom_sampled_loss_bwd(q, *[A] * 9, None, stream=0, check=False) == E.BLOSSOM_ERR_WORKSPACE
