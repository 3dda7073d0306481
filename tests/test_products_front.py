"""The embedding and the linear layer under transforms, tangents and tensors that hold no plain memory: refused, or resolved."""
import pytest


def calls():
    """(function of its tensors, tensors, how many of them in front are differentiable)"""
    import torch
    from paper_2512_13368_b200.autograd import blossom_embedding, blossom_linear
    g = torch.Generator(device="cuda").manual_seed(3)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    ids = torch.randint(0, 40, (30, 3), generator=g, device="cuda")
    return [(lambda table, i: blossom_embedding(i, table, scale=2.0, padding_idx=0), [mk(40, 48), ids], 1),
            (lambda x, w, b, r: blossom_linear(x, w, b, residual=r, activation="gelu"), [mk(30, 48), mk(24, 48), mk(24), mk(30, 24)], 4),
            (lambda x, w, b, r: blossom_linear(x, w, b, residual=r, packed=True), [mk(30, 48), mk(24, 48), mk(24), mk(30, 24)], 4),
            (lambda x, w: blossom_linear(x, w, activation="silu", packed=True), [mk(3, 48), mk(24, 48)], 2)]


@pytest.mark.gpu
def test_transforms_without_a_rule_are_refused():
    import torch
    for f, args, n in calls():
        for i, x in enumerate(args):
            one = lambda t: f(*args[:i], t, *args[i + 1:])  # noqa: E731,B023
            with pytest.raises(RuntimeError):
                torch.func.vmap(one)(torch.stack([x, x]))
            if i < n:
                with pytest.raises(RuntimeError):
                    torch.func.grad(lambda t: one(t).sum())(x)  # noqa: B023
        # several upstream gradients at once
        a = [t.detach().requires_grad_(t.is_floating_point()) for t in args]
        out = f(*a)
        for i in range(n):
            if i == 3:
                continue      # (the residual's gradient is the upstream one, whatever that is)
            with pytest.raises(RuntimeError):
                torch.autograd.grad(out, a[i], torch.ones((2, *out.shape), device="cuda"), is_grads_batched=True, retain_graph=True)
        assert torch.isfinite(f(*args)).all()     # (and the interpreter is in order)


@pytest.mark.gpu
@pytest.mark.parametrize("train", [False, True])
def test_forward_mode_is_refused(train):
    import torch
    import torch.autograd.forward_ad as fwd
    for f, args, n in calls():
        args = [t.detach().requires_grad_(train and t.is_floating_point()) for t in args]
        with fwd.dual_level():
            for i in range(n):
                a = list(args)
                a[i] = fwd.make_dual(a[i], torch.ones_like(a[i]))
                with pytest.raises(NotImplementedError):
                    f(*a)
        assert torch.isfinite(f(*args)).all()


@pytest.mark.gpu
def test_negated_and_zero_tensors_are_resolved():
    """Views that are negated when they are read, and tensors of zeros without memory, as every argument and upstream gradient."""
    import torch

    def step(f, args, dout):
        a = [t.detach().requires_grad_(True) if t.is_floating_point() else t for t in args]
        out = f(*a)
        return [out.detach()] + list(torch.autograd.grad(out, [t for t in a if t.requires_grad], dout))

    for f, args, _ in calls():
        dout = torch.randn_like(f(*args))
        want = step(f, args, dout)
        for i, t in enumerate([*args, dout]):
            neg = torch._neg_view(-t)
            zero = torch._efficientzerotensor(t.shape, dtype=t.dtype, device="cuda")
            assert neg.is_neg() and zero._is_zerotensor()
            for other, plain in ((neg, None), (zero, torch.zeros_like(t))):
                def put(v):
                    a = list(args)
                    if i < len(args):  # noqa: B023
                        a[i] = v       # noqa: B023
                    return step(f, a, v if i == len(args) else dout)  # noqa: B023
                ref = want if plain is None else put(plain)
                assert all(torch.equal(x, y) for x, y in zip(put(other), ref)), i


@pytest.mark.gpu
@pytest.mark.parametrize("packed", [False, True])
def test_a_backward_captured_while_an_eager_graph_of_other_leaves_lives(packed):
    """Captured with leaves of its own (one of the same leaves is refused by PyTorch's engine), and replayed on changed inputs."""
    import torch
    from paper_2512_13368_b200.autograd import blossom_embedding, blossom_linear
    torch.manual_seed(0)
    ids = torch.randint(0, 50, (70,), device="cuda")
    table, w, b = torch.randn(50, 64, device="cuda"), torch.randn(48, 64, device="cuda"), torch.randn(48, device="cuda")

    def step(leaves):
        y = blossom_linear(blossom_embedding(ids, leaves[0]), *leaves[1:], activation="gelu", packed=packed)
        return y, torch.autograd.grad(y, leaves, torch.ones_like(y), retain_graph=True)

    own, captured = ([t.clone().requires_grad_(True) for t in (table, w, b)] for _ in range(2))
    alive = step(own)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(captured)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(captured)
    for k in (1.0, 0.5):
        with torch.no_grad():
            for a, c in zip(own, captured):
                a.mul_(k)
                c.mul_(k)
        graph.replay()
        want = step(own)
        assert torch.equal(got[0], want[0]) and all(torch.equal(x, y) for x, y in zip(got[1], want[1]))
    assert alive[0].requires_grad


def test_inputs_in_8_bits_are_for_the_librarys_layers():
    """A layer case that would ignore `packed` says so."""
    import subprocess
    import sys

    from paper_2512_13368_b200.layer_step import BlossomEncoder
    with pytest.raises(ValueError, match="products"):
        BlossomEncoder(n_items=10, hidden=32, packed=True)
    BlossomEncoder(n_items=10, hidden=32, products=True, packed=True)
    run = subprocess.run([sys.executable, "-m", "paper_2512_13368_b200.layer_step", "--native", "--packed"], capture_output=True, text=True)
    assert run.returncode == 2 and "--products" in run.stderr
