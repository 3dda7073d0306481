"""The linear layer's workspace: as much as the kernels that run need."""
import pytest

from paper_2512_13368_b200 import binding

A = 1 << 20   # an address, never read


def sizes(rows, cols, outs, dtype, act, packed=False, x=A, w=A, dout=A, **kw):
    """(for tensors anywhere, for tensors at these addresses)"""
    p = binding.make_linear_params(rows, cols, outs, dtype, act, packed, **kw)
    return binding.blossom_linear_workspace_bytes(p), binding.blossom_linear_bwd_workspace_bytes(p, x, w, dout)


def test_sizes():
    binding.load()
    MB = 1 << 20
    # narrow layers: partial sums of 148 blocks, not the upstream gradient behind the activation nor x from its codes
    for rows, cols, outs, act, packed in ((131072, 64, 256, "gelu", False), (131072, 256, 64, "none", True), (131072, 64, 192, "none", False)):
        anywhere, here = sizes(rows, cols, outs, "bf16", act, packed)
        sums = 148 * outs * (cols + 1) * 4
        assert sums <= here <= sums + 4096, (rows, cols, outs)
        assert here <= anywhere and (act == "none" and not packed or anywhere > 60 * MB)
    # codes behind an activation become rows first
    _, here = sizes(131072, 64, 256, "bf16", "gelu", True)
    assert 131072 * 64 * 2 <= here <= 131072 * 64 * 2 + 11 * MB
    # as many rows at a time as an accumulator may add up
    for rows, cols, outs, act, splits in ((148 * 16384, 256, 64, "none", 148), (148 * 16384 + 1, 256, 64, "none", 149),
                                          (148 * 8192, 64, 256, "gelu", 148), (148 * 16384, 64, 256, "gelu", 296)):
        _, here = sizes(rows, cols, outs, "bf16", act)
        sums = splits * outs * (cols + 1) * 4
        assert sums <= here <= sums + 4096, (rows, act)
    # tensors that the kernel cannot take, wide layers, few rows, float32: what fits anywhere
    for kw in (dict(w=A + 2), dict(dout=A + 8), dict(x=A + 2), dict(x_stride=68), dict(out_stride=260), dict(weight_stride=65)):
        anywhere, here = sizes(131072, 64, 256, "bf16", "gelu", **kw)
        assert here == anywhere, kw
    for a in ((131072, 264, 256, "bf16", "gelu"), (3, 64, 64, "bf16", "gelu"), (131072, 64, 256, "fp32", "gelu"), (0, 64, 64, "bf16", "gelu")):
        anywhere, here = sizes(*a)
        assert here == anywhere and here >= binding.LINEAR_FORWARD_BYTES, a
    # x that is not read does not matter
    assert sizes(131072, 256, 64, "bf16", "none", True, x=None)[1] == sizes(131072, 256, 64, "bf16", "none", True)[1]
    # refused params
    assert sizes(10, 0, 64, "bf16", "none") == (0, 0) and sizes(10, 64, 65537, "bf16", "none") == (0, 0)


def test_a_workspace_for_other_addresses_is_refused():
    binding.load()
    p = binding.make_linear_params(4096, 64, 256, "bf16", "gelu")
    here = binding.blossom_linear_bwd_workspace_bytes(p, A, A, A)
    for kw in (dict(x=A + 2), dict(w=A + 2), dict(dout=A + 2)):
        a = dict(dict(x=A, w=A, dout=A), **kw)
        rc = binding.blossom_linear_bwd(p, a["x"], None, a["w"], A, a["dout"], A, A, A, A, here, stream=0, check=False)
        assert rc == binding.BLOSSOM_ERR_WORKSPACE, kw
    assert binding.blossom_linear_bwd(p, A, None, A, A, A, A, A, A, A, here - 1, stream=0, check=False) == binding.BLOSSOM_ERR_WORKSPACE


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols,outs", [(3, 64, 64), (16, 300, 64), (100, 256, 256), (129, 64, 200), (1500, 64, 256), (1500, 256, 64),
                                            (700, 50, 200), (200, 40, 2466), (1500, 264, 520)])
def test_the_same_bits_within_the_smaller_workspace(rows, cols, outs, dtype):
    import torch
    torch.manual_seed(0)
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16

    def at(t, offset):     # at an address that is that many elements behind a multiple of 256 bytes
        big = torch.empty(t.numel() + 256, dtype=t.dtype, device="cuda")
        v = big[offset:offset + t.numel()].view(t.shape)
        v.copy_(t)
        return v

    x, w, b, dout = (torch.randn(*s, device="cuda").to(dt) for s in ((rows, cols), (outs, cols), (outs,), (rows, outs)))
    for act, packed in (("none", False), ("none", True), ("gelu", False), ("gelu", True)):
        p = binding.make_linear_params(rows, cols, outs, dtype, act, packed)
        codes, scales = (torch.zeros(rows, n, dtype=t, device="cuda") for n, t in ((cols, torch.int8), ((cols + 31) // 32, torch.uint8)))
        if packed:
            binding.blossom_pack_rows(binding.make_rows_params(rows, cols, dtype), x, codes, scales)
        for offset in (0, 3):
            xs, ws_, ds = at(codes if packed else x, offset), at(w, offset), at(dout, offset)
            for want in ((1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1)):
                reads_x = act != "none" or want[1]
                need = binding.blossom_linear_bwd_workspace_bytes(p, xs if reads_x else None, ws_, ds)
                got = []
                for size in (binding.blossom_linear_workspace_bytes(p), need):
                    room = torch.full((size + (1 << 16),), 0xee, dtype=torch.uint8, device="cuda")
                    res = [torch.full_like(t, 7.0) if k else None for t, k in zip((x, w, b), want)]
                    binding.blossom_linear_bwd(p, xs if reads_x else None, scales if packed else None, ws_, b, ds, *res, room[:size])
                    assert binding.blossom_device_status(room) == 0 and bool((room[size:] == 0xee).all()), (act, packed, offset, want)
                    got.append(res)
                assert all(u is None or torch.equal(u, v) for u, v in zip(*got)), (act, packed, offset, want)


@pytest.mark.gpu
@pytest.mark.parametrize("cols,outs,act,packed", [(64, 256, "gelu", False), (256, 64, "none", True)])
def test_what_a_backward_takes_for_itself(cols, outs, act, packed):
    """Through autograd: the gradients and the partial sums."""
    import torch
    from paper_2512_13368_b200.autograd import blossom_linear
    rows = 65536
    leaves = [torch.randn(*s, device="cuda").bfloat16().requires_grad_(True) for s in ((rows, cols), (outs, cols), (outs,))]
    y = blossom_linear(*leaves, activation=act, packed=packed)
    dout = torch.ones_like(y)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    torch.autograd.grad(y, leaves, dout)
    assert torch.cuda.max_memory_allocated() - before <= rows * cols * 2 + 148 * outs * (cols + 1) * 4 + (1 << 21)
