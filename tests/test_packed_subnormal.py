"""Rows in 8 bits whose elements are subnormal beside a largest one that is not: codes of 1, not zeros."""
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
