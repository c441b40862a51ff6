"""The float64 losses against central differences and against what their definitions say at the corners."""
import numpy as np
import pytest

from oracle import losses


def _inputs(rows, C, seed):
    rng = np.random.default_rng(seed)
    x = rng.normal(0, 2, (rows, C))
    label = rng.integers(0, C, rows)
    lp = np.array([losses.log_softmax(x[r])[label[r]] for r in range(rows)])
    return rng, x, label, lp


def _differences(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += h
        down[i] -= h
        g[i] = (f(up) - f(down)) / (2 * h)
    return g


@pytest.mark.parametrize("kl", ["none", "sampled", "full"])
@pytest.mark.parametrize("weighted", [False, True])
def test_policy_gradient_is_the_derivative(kl, weighted):
    rng, x, label, lp = _inputs(7, 5, 3)
    label[2], label[5] = -1, 5                                   # masked on either side
    kw = dict(clip_low=0.2, clip_high=0.3, kl_coef=0.7, weight=rng.uniform(0.1, 2, 7) if weighted else None)
    # ratios on both sides of both borders, with advantages of either sign
    old, A = lp - np.array([0.5, -0.5, 0, 0.1, 0.6, 0, -0.6]), np.array([1.0, -1.0, 1, 0.5, -0.7, 1, 0.9])
    if kl == "sampled":
        kw["ref_logp"] = lp + rng.normal(0, 0.4, 7)
    if kl == "full":
        kw["ref_logits"] = x + rng.normal(0, 0.5, x.shape)
    r = losses.policy_loss(x, label, old, A, **kw)
    want = _differences(lambda v: losses.policy_loss(v, label, old, A, **kw)["loss"], x)
    # h = 1e-6: truncation 1e-12 times third derivatives of order 1, rounding 1e-16 / 1e-6
    np.testing.assert_allclose(r["grad"], want, rtol=0, atol=1e-8)
    assert not r["grad"][2].any() and not r["grad"][5].any()
    assert r["stats"][2] > 0 and (r["stats"][1] > 0) == (kl != "none")


def test_policy_clips_only_where_the_smaller_product_is_constant():
    x, label = np.zeros((4, 2)), np.zeros(4, int)
    lp = np.log(0.5)
    old = np.array([lp - 1, lp - 1, lp + 1, lp + 1])             # ratios e, e, 1/e, 1/e
    r = losses.policy_loss(x, label, old, np.array([1.0, -1.0, 1.0, -1.0]), 0.2, 0.2, 0.0)
    assert np.allclose(r["stats"], [(1.2 - np.e + np.exp(-1) - 0.8) / 4, 0, 0.5])
    assert [bool(g.any()) for g in r["grad"]] == [False, True, True, False]


@pytest.mark.parametrize("eps", [0.0, 0.15])
def test_preference_gradient_is_the_derivative(eps):
    rng, x, label, _ = _inputs(9, 4, 5)
    label[1] = -1
    offsets, ref = [0, 3, 4, 4, 8], rng.normal(-4, 2, 4)         # an empty sequence, a row behind the last
    f = lambda v: losses.preference_loss(v, label, offsets, 0.3, eps, ref)  # noqa: E731
    r = f(x)
    want = _differences(lambda v: f(v)["loss"], x)
    np.testing.assert_allclose(r["grad"][:8], want[:8], rtol=0, atol=1e-8)
    assert not want[8].any() and np.isnan(r["grad"][8]).all() and not r["grad"][1].any()
    assert r["logp"][2] == 0.0


def test_rows_without_a_distribution():
    x = np.full((2, 3), -np.inf)
    x[1] = 0
    r = losses.policy_loss(x, np.array([0, 0]), np.zeros(2), np.ones(2), 0.2, 0.2, 0.0)
    assert r["logp"][0] == -np.inf and not r["grad"][0].any() and np.isclose(r["loss"], -(1 / 3) / 2)
    p = losses.preference_loss(x, np.array([0, 0]), [0, 1, 2], 1.0)
    assert p["logp"][0] == 0 and not p["grad"][0].any() and p["grad"][1].any()


def test_clipping_scales_down_to_the_norm_and_never_up():
    g = [np.array([3.0, 0.0]), np.array([[4.0]]), np.zeros(0)]
    norm, each, clipped = losses.grad_clip(g, 2.5)
    assert norm == 5.0 and list(each) == [3.0, 4.0, 0.0] and np.allclose(clipped[0], [1.5, 0]) and np.allclose(clipped[1], 2)
    assert all((a == b).all() for a, b in zip(losses.grad_clip(g, 5.0)[2], g))
    assert np.isinf(losses.grad_clip([np.array([np.inf, 1.0])], 1.0)[2][0][0])
