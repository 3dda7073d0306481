"""The layer case with everything around the attention in the library: the same model step by step as with PyTorch's
operators, dropouts that are the definition's, a step captured in a graph.  GPU only."""
import numpy as np
import pytest

from oracle import rows_oracle as ro

pytestmark = pytest.mark.gpu


def models(dtype, **kw):
    import torch
    from paper_2512_13368_b200 import layer_step
    torch.manual_seed(0)
    args = dict(n_items=300, hidden=64, heads=2, ffn=96, layers=2, block=16, topk=3, window=24)
    plain = layer_step.BlossomEncoder(**args).cuda().to(dtype)
    native = layer_step.BlossomEncoder(native=True, seed=5, **args, **kw).cuda().to(dtype)
    native.load_state_dict(plain.state_dict(), strict=False)
    ids = layer_step.zipf_ids(4, 96, 300, seed=2).cuda()
    neg = torch.randint(1, 301, (4, 96, 15), device="cuda")
    return plain, native, ids[:, :-1], ids[:, 1:], neg


def test_the_same_step_as_with_pytorch_operators():
    """Without dropout, in single precision: the same sums in another order.  Two layers of sums over at most 256 terms, each to
    a few units of 2^-24: 1e-4 relative to the largest gradient of a parameter leaves a factor of some tens."""
    import torch
    plain, native, ids, targets, neg = models(torch.float32)
    a, b = plain.loss(ids, targets, neg), native.loss(ids, targets, neg)
    a.backward(), b.backward()
    assert abs(float(a.detach()) - float(b.detach())) < 1e-5 * abs(float(a.detach()))
    for (name, p), (_, q) in zip(plain.named_parameters(), native.named_parameters()):
        assert float((p.grad - q.grad).abs().max()) <= 1e-4 * float(p.grad.abs().max()) + 1e-9, name


def test_dropouts_are_those_of_the_definition(monkeypatch):
    """The PyTorch operators with the definition's masks in place of random ones give the native step."""
    import torch
    from paper_2512_13368_b200 import layer_step
    plain, native, ids, targets, neg = models(torch.float32, dropout=0.3)
    plain.dropout = 0.3
    for layer in plain.layers:
        layer.dropout = 0.3
    native.rng[1] = 17
    site = iter(range(100))

    def masked(x, p, training=True):
        f = ro.keep_factor(x[..., 0].numel(), x.shape[-1], p, 5, 17, next(site))
        return x * torch.from_numpy(f.astype(np.float32)).cuda().view(x.shape)

    b = native.loss(ids, targets, neg)
    b.backward()
    monkeypatch.setattr(layer_step.F, "dropout", masked)
    a = plain.loss(ids, targets, neg)
    a.backward()
    assert next(site) == 5   # embeddings, twice two layers
    assert abs(float(a.detach()) - float(b.detach())) < 1e-5 * abs(float(a.detach()))
    for (name, p), (_, q) in zip(plain.named_parameters(), native.named_parameters()):
        assert float((p.grad - q.grad).abs().max()) <= 1e-4 * float(p.grad.abs().max()) + 1e-9, name
    native.eval()
    with torch.no_grad():
        plain.eval()
        assert torch.allclose(native(ids), plain(ids), rtol=1e-4, atol=1e-5)


def test_training_steps_and_a_captured_one():
    import torch
    _, native, ids, targets, neg = models(torch.bfloat16, dropout=0.1)
    losses = []
    for _ in range(30):
        native.zero_grad(set_to_none=True)
        loss = native.loss(ids, targets, neg)
        loss.backward()
        native.next_step()
        with torch.no_grad():
            for p in native.parameters():
                p -= 0.5 * p.grad
        losses.append(float(loss.detach()))
    assert int(native.rng[1]) == 30 and losses[0] > 2.7 and losses[-1] < losses[0] - 0.05

    def step():
        return native.loss(ids, targets, neg)

    with torch.no_grad():
        want = []
        native.rng[1] = 100
        for _ in range(3):
            want.append(step().clone())
            native.next_step()
        native.rng[1] = 100
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
            native.next_step()
        native.rng[1] = 100
        for k in range(3):
            graph.replay()
            assert torch.equal(out, want[k])
        assert not torch.equal(want[0], want[1])


def test_the_share_is_reported_with_the_native_rows():
    from paper_2512_13368_b200 import layer_step
    r = layer_step.attention_share(batch=8, seq_len=256, n_items=2000, negatives=15, steps=2, warmup=1, native=True, dropout=0.2)
    assert np.isfinite(r["loss"]) and 0.0 < r["attention_share"] < 1.0 and r["rows_and_loss_ms_per_step"] > 0.0
    # two layers x (attention, two layer norms in three launches each), a dropout each way, the loss
    assert r["library_launches_per_step"] >= 2 * (7 + 6) + 2 + 5
