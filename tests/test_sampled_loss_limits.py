"""How many candidates a row of the sampled loss may have."""
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
