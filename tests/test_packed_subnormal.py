"""Rows in 8 bits at their limits: elements that are subnormal beside a largest one that is not, and how far values may be off."""
import numpy as np
import pytest

from oracle import linear_oracle as lo
from paper_2512_13368_b200 import binding


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("cols", [32, 50, 256, 1000])
def test_subnormal_elements(cols, dtype):
    import torch
    g = torch.Generator().manual_seed(cols)
    rows = 40
    # multiples of 2^-130 up to 2^-124, in groups whose largest is from 2^-121 (all zeros) to 2^-117
    x = torch.randint(-63, 64, (rows, cols), generator=g).float() * 2.0 ** -130
    x[:, ::32] = torch.exp2(torch.randint(-121, -116, (rows, 1), generator=g).float()) * 1.5
    x[:, 1::32] = 2.0 ** -127                    # half a unit of the smallest: to even, zero
    x[:, 2::32] = -(2.0 ** -127) * 1.03125       # more than half
    x = x.to(torch.float32 if dtype == "fp32" else torch.bfloat16)
    want_codes, want_scales = lo.pack(x.float().numpy())
    assert (np.abs(want_codes[:, 2::32]) == 1).any()
    p = binding.make_rows_params(rows, cols, dtype)
    x = x.cuda()
    codes = torch.empty(rows, cols, dtype=torch.int8, device="cuda")
    scales = torch.empty(rows, (cols + 31) // 32, dtype=torch.uint8, device="cuda")
    binding.blossom_pack_rows(p, x, codes, scales)
    assert np.array_equal(codes.cpu().numpy(), want_codes) and np.array_equal(scales.cpu().numpy(), want_scales)
    out = torch.empty_like(x)
    binding.blossom_unpack_rows(p, codes, scales, out)
    assert np.array_equal(out.double().cpu().numpy(), lo.unpack(want_codes, want_scales))


def test_how_far_a_value_may_be_off():
    """2^-7 of a group's largest magnitude and no less: half a unit where that begins with 1, a unit at the limit of 127."""
    x = np.full((2, 32), 0.0, dtype=np.float32)
    x[0, :2] = 1.0, 0.9999 * 2.0 ** -7     # (half a unit is 2^-7: zero)
    x[1, :2] = 1.9999, 1.0                 # 127.99 units
    off = np.abs(lo.unpack(*lo.pack(x)) - x)
    assert off[0, 1] > 0.99 * 2.0 ** -7 and off[1, 0] > 0.99 * 2.0 ** -7 * x[1, 0]
    g = np.random.default_rng(0)
    x = (g.standard_normal((2000, 64)) * np.exp2(g.integers(-100, 100, (2000, 1)))).astype(np.float32)
    off, top = np.abs(lo.unpack(*lo.pack(x)) - x), np.abs(x)
    for c in (0, 32):
        assert (off[:, c:c + 32] <= 2.0 ** -7 * top[:, c:c + 32].max(axis=1, keepdims=True)).all()
