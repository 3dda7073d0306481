"""The double-precision definitions of the rows around the attention: the generator against its published vectors,
gradients against differences.  CPU only."""
import numpy as np
import pytest

from oracle import rows_oracle as ro


@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_generator_gives_its_published_vectors(counter, key, want):
    assert tuple(int(x) for x in ro.philox4x32(counter, key)) == want


@pytest.mark.parametrize("p", [0.1, 0.5, 0.9])
def test_share_of_kept_elements_and_their_mean(p):
    f = ro.keep_factor(400, 333, p, seed=7, step=3, site=2)
    n, keep = f.size, 1.0 - ro.bar(p) / 65536.0
    assert abs((f > 0).mean() - keep) < 6.0 * np.sqrt(keep * (1 - keep) / n)   # six standard deviations
    assert np.all((f == 0) | (f == 65536.0 / (65536 - ro.bar(p))))


def test_seed_step_site_row_and_column_all_count():
    base = ro.keep_factor(64, 40, 0.5, 1, 2, 3) > 0
    for other in (ro.keep_factor(64, 40, 0.5, 2, 2, 3), ro.keep_factor(64, 40, 0.5, 1, 3, 3),
                  ro.keep_factor(64, 40, 0.5, 1, 2, 4), ro.keep_factor(64, 40, 0.5, 1 + (1 << 32), 2, 3),
                  ro.keep_factor(64, 40, 0.5, 1, 2 + (1 << 32), 3)):
        assert 0.4 < (base == (other > 0)).mean() < 0.6
    # what is drawn for an element does not depend on how many rows or columns there are
    assert np.array_equal(ro.keep_factor(10, 17, 0.5, 1, 2, 3) > 0, base[:10, :17])
    assert np.all(ro.keep_factor(8, 8, 1.0, 1, 2, 3) == 0.0)


def _difference(f, x, v, h=1e-6):
    return (f(x + h * v) - f(x - h * v)) / (2 * h)


@pytest.mark.parametrize("p", [0.0, 0.3])
def test_add_norm_gradients_against_differences(p):
    rng = np.random.default_rng(3)
    x, r, dout = rng.standard_normal((3, 5, 13))
    w, b = 1 + 0.2 * rng.standard_normal(13), 0.2 * rng.standard_normal(13)
    fac = ro.keep_factor(5, 13, p, 1, 1, 1)
    g = ro.add_norm_backward(ro.add_norm(x, r, w, b, fac, 1e-5), dout)
    loss = lambda x=x, r=r, w=w, b=b: float((ro.add_norm(x, r, w, b, fac, 1e-5)["out"] * dout).sum())  # noqa: E731
    for key, arg, f in (("dx", x, lambda y: loss(x=y)), ("dresidual", r, lambda y: loss(r=y)),
                        ("dweight", w, lambda y: loss(w=y)), ("dbias", b, lambda y: loss(b=y))):
        v = rng.standard_normal(arg.shape)
        # a central difference of step 1e-6: truncation ~ h^2, cancellation ~ 1e-16 |loss| / h
        assert abs(_difference(f, arg, v) - float((g[key] * v).sum())) < 1e-7, key


@pytest.mark.parametrize("hits", [False, True])
def test_sampled_loss_gradients_against_differences(hits):
    rng = np.random.default_rng(4)
    h, w = rng.standard_normal((6, 5)), rng.standard_normal((9, 5))
    t = np.array([3, 0, -100, 8, 3, 9])          # one ignored, one out of range
    neg = rng.integers(-1, 10, size=(6, 4))      # some out of range, some hits
    neg[0, 1] = 3
    f = ro.sampled_loss(h, w, t, neg, mask_hits=hits)
    assert f["count"] == 4 and np.all(f["dhidden"][[2, 5]] == 0) and np.all(f["lse"][[2, 5]] == 0)
    v, u = rng.standard_normal(h.shape), rng.standard_normal(w.shape)
    loss = lambda a, b: ro.sampled_loss(a, b, t, neg, mask_hits=hits)["loss"]  # noqa: E731
    assert abs(_difference(lambda y: loss(y, w), h, v) - float((f["dhidden"] * v).sum())) < 1e-7
    assert abs(_difference(lambda y: loss(h, y), w, u) - float((f["dtable"] * u).sum())) < 1e-7


def test_sampled_loss_without_rows_or_negatives():
    rng = np.random.default_rng(5)
    h, w = rng.standard_normal((2, 3)), rng.standard_normal((4, 3))
    none = ro.sampled_loss(h, w, np.array([-100, 4]), np.array([[0, 1], [2, 3]]))
    assert none["loss"] == 0.0 and none["count"] == 0 and not none["dtable"].any()
    alone = ro.sampled_loss(h, w, np.array([1, 2]), np.zeros((2, 0), dtype=int))
    assert abs(alone["loss"]) < 1e-15 and np.abs(alone["dhidden"]).max() < 1e-15
