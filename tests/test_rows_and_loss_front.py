"""The autograd nodes of dropout, residual + layer norm and the sampled loss beyond the ordinary call: saved tensors that come
back in another layout or as something else, integers that do not fit, tensors that are not plain memory, transforms without a
rule, host threads."""
import threading

import pytest

from paper_2512_13368_b200 import build


def operators(offset=3, pads=(16, 7, 16, 9), seed=0):
    """(name, function of the leaves, leaves, ids of the loss): every tensor that is saved is a slice of a wider buffer."""
    import torch
    from paper_2512_13368_b200.autograd import blossom_add_norm, blossom_dropout, blossom_sampled_loss
    g = torch.Generator(device="cuda").manual_seed(seed)

    def sliced(rows, cols, pad, dtype):
        return torch.randn(rows, cols + pad, generator=g, device="cuda").to(dtype)[:, offset:offset + cols].detach()

    def ids(hi, *shape, pad=0):
        t = torch.randint(0, hi, (*shape[:-1], shape[-1] + pad), generator=g, device="cuda")
        return t[..., :shape[-1]]

    rng = torch.tensor([[5, 0], [9, 0]], device="cuda")[:, 0]   # (its two numbers are not next to each other)
    res = []
    for dtype, cols in ((torch.bfloat16, 64), (torch.float32, 50)):
        x, r, h, w = (sliced(n, cols, pad, dtype) for n, pad in zip((90, 90, 90, 40), pads))
        weight, bias = (torch.randn(2 * cols, generator=g, device="cuda").to(dtype)[::2] for _ in range(2))
        t, own, shared = ids(40, 180)[::2], ids(40, 90, 7, pad=5), ids(40, 14)[::2]
        res += [("dropout", lambda a: blossom_dropout(a, 0.3, rng, site=4), [x], None),
                ("norm", lambda a, b, c, d: blossom_add_norm(a, b, c, d, p=0.3, rng=rng, site=4), [x, r, weight, bias], None),
                ("norm, no dropout", lambda a, b, c, d: blossom_add_norm(a, b, c, d), [x, r, weight, bias], None),
                ("norm alone", lambda a: blossom_add_norm(a, None, None, None), [x], None),
                ("loss", lambda a, b, t=t, n=own: blossom_sampled_loss(a, b, t, n), [h, w], (t, own)),
                ("loss, shared", lambda a, b, t=t, n=shared: blossom_sampled_loss(a, b, t, n), [h, w], (t, shared)),
                ("loss, no negatives", lambda a, b, t=t, n=own: blossom_sampled_loss(a, b, t, n[:, :0]), [h, w], (t, own[:, :0]))]
    return res


def step(f, leaves, make=None):
    """Output and gradients; make: what calls f."""
    import torch
    a = [t.detach().requires_grad_(True) for t in leaves]
    assert all(x.stride() == y.stride() for x, y in zip(a, leaves))
    out = f(*a) if make is None else make(f, *a)
    return [out.detach()] + list(torch.autograd.grad(out, a, torch.full_like(out, 0.75)))


@pytest.mark.gpu
def test_saved_tensors_may_come_back_in_another_layout():
    """Offloaded to the host and brought back a slice has lost its gaps; computed again it may lie elsewhere.  The same bits, but for
    the loss in layouts of another alignment, by which its kernels (the order of their sums) go: there within the
    definition's bounds."""
    import torch
    from test_sampled_loss import compare, reference
    from torch.utils.checkpoint import checkpoint

    def offload(pin):
        def make(f, *a):
            with torch.autograd.graph.save_on_cpu(pin_memory=pin):
                return f(*a)
        return make

    def gaps(t):    # the same numbers with gaps between rows, elements of a vector apart
        if t.dim() == 0:
            return t
        big = torch.zeros(*t.shape[:-1], 2 * t.shape[-1] + 6, dtype=t.dtype, device=t.device)
        view = big[..., 2:2 + t.shape[-1]] if t.dim() > 1 else big[2:2 + 2 * t.shape[-1]:2]
        return view.copy_(t) if t.numel() else t

    def widen(f, *a):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, gaps):
            return f(*a)

    for offset, pads in ((3, (16, 7, 16, 9)), (0, (16, 8, 16, 8))):
        for name, f, leaves, ids in operators(offset, pads):
            want = step(f, leaves)
            if ids:
                exact, tol = reference(*leaves, *ids)
                exact, tol = ({k: d[k] * (1.0 if k == "loss" else 0.75) for k in ("loss", "dhidden", "dtable")} for d in (exact, tol))
            for make in (offload(False), offload(True), widen, lambda f, *a: checkpoint(f, *a, use_reentrant=False)):
                got = step(f, leaves, make)
                if ids:
                    compare(dict(zip(exact, got)), exact, tol, leaves[0].dtype == torch.bfloat16, name)
                if not ids or (offset == 0 and make is not widen):
                    assert all(torch.equal(a, b) for a, b in zip(got, want)), name


@pytest.mark.gpu
def test_saved_tensors_that_are_something_else_are_refused():
    """Fewer rows, other types, another device: an error, whichever of the saved tensors it is."""
    import torch
    change = {"shorter": lambda t: t[:-1], "wider": lambda t: torch.cat([t, t], -1),
              "type": lambda t: t.to(torch.float64 if t.is_floating_point() else torch.int16), "device": lambda t: t.cpu()}
    for name, f, leaves, _ in operators():
        for how, other in change.items():
            which, count = 0, 1
            while which < count:
                packed = []

                def pack(t):
                    packed.append(t)  # noqa: B023
                    return len(packed) - 1, t  # noqa: B023

                a = [t.detach().requires_grad_(True) for t in leaves]
                with torch.autograd.graph.saved_tensors_hooks(pack, lambda it: other(it[1]) if it[0] == which else it[1]):  # noqa: B023
                    out = f(*a)
                with pytest.raises(RuntimeError, match="hook"):
                    torch.autograd.grad(out, a, torch.full_like(out, 0.75))
                which, count = which + 1, len(packed)
            assert count >= 1, (name, how)


def test_integers_of_more_than_32_bits_are_refused():
    """Their low half must not pass for the number, in the attention's arguments neither."""
    import torch
    build.build()
    from paper_2512_13368_b200 import autograd
    front = autograd._module()
    x, rng, ids = torch.zeros(4, 8), torch.zeros(2, dtype=torch.int64), torch.zeros(4, dtype=torch.int64)
    q, gate = torch.zeros(1, 1, 8, 32), torch.zeros(1, 2)
    tail = (8, 2, 8, 0.0, 0, 8, 0, 0, 0, 0, 1, 0.0)
    assert front.dropout(x, 0.5, rng, 5) is None      # (a host tensor: the caller says what is wrong)
    assert front.attention(q, q, q, gate, None, None, *tail) is None
    for wide in ((1 << 32) + 5, 1 << 31, -(1 << 31) - 1, 1 << 62, 1 << 70, torch.tensor((1 << 32) + 5)):
        for call in (lambda: front.dropout(x, 0.5, rng, wide), lambda: front.add_norm(x, None, None, None, 0.5, rng, wide, 1e-5),  # noqa: B023
                     lambda: front.sampled_loss(x, x, ids, ids, -100, wide),  # noqa: B023
                     lambda: front.attention(q, q, q, gate, None, None, wide, *tail[1:])):  # noqa: B023
            with pytest.raises(OverflowError):
                call()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,cols", [("bf16", 64), ("fp32", 50)])
def test_negated_views_and_zero_tensors_that_need_no_copy_for_their_layout(dtype, cols):
    """Every input, the generator's state among them, and the upstream gradient: what plain copies give."""
    import torch
    from paper_2512_13368_b200.autograd import blossom_add_norm, blossom_dropout, blossom_sampled_loss
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(cols)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda").to(dt)  # noqa: E731
    ids = lambda *s: torch.randint(0, 40, s, generator=g, device="cuda")  # noqa: E731
    rng = torch.tensor([7, 3], device="cuda")
    cases = [(lambda x, rng: blossom_dropout(x, 0.4, rng, site=2), dict(x=mk(30, cols), rng=rng), mk(30, cols)),
             (lambda x, r, w, b, rng: blossom_add_norm(x, r, w, b, p=0.4, rng=rng, site=2),
              dict(x=mk(30, cols), r=mk(30, cols), w=mk(cols), b=mk(cols), rng=rng), mk(30, cols)),
             (blossom_sampled_loss, dict(hidden=mk(30, cols), table=mk(40, cols), targets=ids(30), negatives=ids(30, 5)),
              torch.tensor(0.75, device="cuda")),
             (blossom_sampled_loss, dict(hidden=mk(30, cols), table=mk(40, cols), targets=ids(30), negatives=ids(5)),
              torch.tensor(0.75, device="cuda"))]

    def step(f, args, dout):
        a = {k: (t.detach().requires_grad_(True) if t.is_floating_point() else t) for k, t in args.items()}
        out = f(**a)
        return [out.detach()] + list(torch.autograd.grad(out, [t for t in a.values() if t.requires_grad], dout))

    for f, args, dout in cases:
        want = step(f, args, dout)
        for k, t in dict(args, dout=dout).items():
            neg = torch._neg_view(-t)
            assert neg.is_neg() and torch.equal(neg, t) and neg.stride() == t.stride()
            zero = torch._efficientzerotensor(t.shape, dtype=t.dtype, device="cuda")
            assert zero._is_zerotensor()
            plain = torch.zeros_like(t)
            ref = step(f, args, plain) if k == "dout" else step(f, dict(args, **{k: plain}), dout)
            for other, res in ((neg, want), (zero, ref)):
                got = step(f, args, other) if k == "dout" else step(f, dict(args, **{k: other}), dout)
                assert all(torch.equal(x, y) for x, y in zip(got, res)), k


def calls():
    """(function of its tensors, tensors): every operator, with what is differentiable in front."""
    import torch
    from paper_2512_13368_b200.autograd import blossom_add_norm, blossom_dropout, blossom_sampled_loss
    g = torch.Generator(device="cuda").manual_seed(3)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    ids = lambda *s: torch.randint(0, 40, s, generator=g, device="cuda")  # noqa: E731
    rng = torch.tensor([7, 3], device="cuda")
    return [(lambda x, rng: blossom_dropout(x, 0.4, rng), [mk(30, 48), rng], 1),
            (lambda x, r, w, b, rng: blossom_add_norm(x, r, w, b, p=0.4, rng=rng), [mk(30, 48), mk(30, 48), mk(48), mk(48), rng], 4),
            (lambda x, r, w, b: blossom_add_norm(x, r, w, b), [mk(30, 48), mk(30, 48), mk(48), mk(48)], 4),
            (blossom_sampled_loss, [mk(30, 48), mk(40, 48), ids(30), ids(30, 5)], 2),
            (blossom_sampled_loss, [mk(30, 48), mk(40, 48), ids(30), ids(5)], 2)]


@pytest.mark.gpu
def test_transforms_without_a_rule_are_refused():
    """Batched tensors (vmap) and those of functional gradients have no memory that the library could read."""
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
        with pytest.raises(RuntimeError):
            torch.autograd.grad(out, a[0], torch.ones((2, *out.shape), device="cuda"), is_grads_batched=True)
        assert f(*args).shape == out.shape     # (and the interpreter is in order)


@pytest.mark.gpu
@pytest.mark.parametrize("train", [False, True])
def test_forward_mode_is_refused(train):
    """There is no forward-mode rule: a tangent is an error, never dropped."""
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
def test_threads_do_not_disturb_each_other():
    """Host threads that train at once, each on a stream of its own, with sizes whose kernels want different amounts of shared
    memory: the bits of the same steps one after another."""
    import torch
    from paper_2512_13368_b200.autograd import blossom_add_norm, blossom_dropout, blossom_sampled_loss
    g = torch.Generator(device="cuda").manual_seed(4)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()  # noqa: E731
    problems = []
    for rows, cols, items, n in ((400, 64, 700, 9), (900, 512, 300, 3), (300, 1024, 90, 20), (5000, 128, 4000, 15)):
        problems.append([mk(rows, cols), mk(rows, cols), mk(cols), mk(cols), mk(items, cols),
                         torch.randint(0, items, (rows,), generator=g, device="cuda"),
                         torch.randint(0, items, (rows, n), generator=g, device="cuda"), torch.tensor([rows, 1], device="cuda")])

    def step(x, r, w, b, table, targets, negatives, rng):
        leaves = [t.detach().requires_grad_(True) for t in (x, r, w, b, table)]
        y = blossom_add_norm(blossom_dropout(leaves[0], 0.2, rng), *leaves[1:4], p=0.1, rng=rng, site=1)
        loss = blossom_sampled_loss(y, leaves[4], targets, negatives)
        return [loss.detach()] + list(torch.autograd.grad(loss, leaves))

    want = [step(*p) for p in problems]
    torch.cuda.synchronize()
    failures, start = [], threading.Barrier(len(problems))

    def work(p, ref):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait()
                for _ in range(60):
                    got = step(*p)
                torch.cuda.current_stream().synchronize()
                assert all(torch.equal(a, b) for a, b in zip(got, ref))
        except BaseException as e:  # noqa: BLE001
            failures.append(e)

    threads = [threading.Thread(target=work, args=a) for a in zip(problems, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures, failures
