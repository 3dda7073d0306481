"""The sampled loss at its limits: how many candidates a row may have, upstream gradients that are no numbers."""
import pytest

from paper_2512_13368_b200 import binding


def test_rows_of_more_candidates_than_a_sum_takes_are_refused():
    """Numbers of candidates near 2^31 would leave the walk's 32-bit counter behind, and single-precision sums stop at 2^24 ones."""
    binding.load()
    E, A = binding, 1 << 20
    good = lambda n, rows=1: E.make_loss_params(rows, 64, 100, n, "bf16", negatives_stride=0)  # noqa: E731
    for n in ((1 << 31) - 2, (1 << 31) - 40, (1 << 30), 1 << 24):
        p = good(n)
        assert E.blossom_sampled_loss_workspace_bytes(p) == 0, n
        assert E.blossom_sampled_loss_fwd(p, A, A, A, A, A, A, A, A, 1 << 50, stream=0, check=False) == E.BLOSSOM_ERR_UNSUPPORTED, n
        assert E.blossom_sampled_loss_bwd(p, *[A] * 9, A, 1 << 50, stream=0, check=False) == E.BLOSSOM_ERR_UNSUPPORTED, n
    assert E.blossom_sampled_loss_workspace_bytes(good((1 << 24) - 1)) > 0
    assert E.blossom_sampled_loss_workspace_bytes(good((1 << 24) - 1, 127)) > 0
    assert E.blossom_sampled_loss_workspace_bytes(good((1 << 24) - 1, 128)) == 0
    assert E.blossom_sampled_loss_workspace_bytes(good(1 << 24, 0)) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols,items,n", [(300, 64, 5000, 6), (300, 50, 5000, 6), (400, 128, 60, 40), (40, 600, 900, 3)])
@pytest.mark.parametrize("g", [float("inf"), float("nan")])
def test_what_takes_no_part_has_zero_gradients_whatever_the_upstream_gradient_is(g, rows, cols, items, n, dtype):
    """An overflowed loss scale: padding and items that are nobody's candidate stay at zero, the others show it."""
    import torch
    from paper_2512_13368_b200.autograd import blossom_sampled_loss
    torch.manual_seed(1)
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    h = torch.randn(rows, cols, device="cuda").to(dt).requires_grad_(True)
    w = (0.3 * torch.randn(items, cols, device="cuda")).to(dt).requires_grad_(True)
    t = torch.randint(0, items // 2, (rows,), device="cuda")
    t[::3] = -100
    neg = torch.randint(0, items // 2, (rows, n), device="cuda")
    live = t >= 0
    used = torch.zeros(items, dtype=torch.bool, device="cuda")
    used[t[live]] = True
    used[neg[live]] = True
    loss = blossom_sampled_loss(h, w, t, neg)
    dh, dw = torch.autograd.grad(loss, (h, w), torch.full_like(loss, g))
    assert not dh[~live].any() and not dw[~used].any()
    assert not torch.isfinite(dh[live]).any() and not torch.isfinite(dw[used]).any()
