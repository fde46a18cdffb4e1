"""Pins of the oracle's density, policy loss, preference loss and advantages."""
import numpy as np
import pytest

import oracle


def _rows(rng, n, d, spread=0.1):
    old = rng.uniform(1.0, 5.0, (n, 2 * d))
    return old * np.exp(spread * rng.standard_normal(old.shape)), old


def test_density_is_the_derivative_of_the_cdf_and_integrates_to_one():
    for a, b in ((2.0, 5.0), (1.5, 3.0), (1.0, 1.0), (4.2, 1.3)):
        x = np.linspace(0.02, 0.98, 97)
        h = 1e-6
        num = (oracle.kumaraswamy_cdf(x + h, a, b) - oracle.kumaraswamy_cdf(x - h, a, b)) / (2 * h)
        l, _, _ = oracle.event_logp(np.array([[a, b]]), x[:, None])
        np.testing.assert_allclose(np.exp(l), num, rtol=1e-7, atol=1e-9)   # 2^-53 over 2e-6, the difference quotient
        mid = (np.arange(200000) + 0.5) / 200000
        assert abs(np.mean(np.exp(oracle.event_logp(np.array([[a, b]]), mid[:, None])[0])) - 1.0) < 1e-4


@pytest.mark.parametrize("d", [2, 3])
def test_density_gradient_by_differences(d):
    rng = np.random.default_rng(d)
    th, _ = _rows(rng, 1, d)
    x = rng.uniform(0.01, 0.99, (50, d))
    _, g, terms = oracle.event_logp(th, x)
    assert np.all(terms >= np.abs(g) * (1.0 - 1e-12))
    for j in range(2 * d):
        e = np.zeros_like(th)
        e[0, j] = 1e-6
        num = (oracle.event_logp(th + e, x)[0] - oracle.event_logp(th - e, x)[0]) / 2e-6
        np.testing.assert_allclose(g[:, j], num, rtol=1e-6, atol=1e-7)


@pytest.mark.parametrize("average", ["events", "rows"])
@pytest.mark.parametrize("ref", [False, True])
def test_policy_gradient_by_differences(average, ref):
    rng = np.random.default_rng(5)
    R, E, d = 4, 30, 2
    th, old = _rows(rng, R, d)
    kw = dict(theta_ref=old * 1.1 if ref else None, mask=rng.random((R, E)) < 0.7, clip_low=0.1, clip_high=0.3, kl_coef=0.3,
              average=average)
    kw["mask"][2] = False
    x, A = rng.uniform(0.02, 0.98, (R, E, d)), rng.standard_normal((R, E))
    o = oracle.policy_loss(th, old, x, A, **kw)
    assert 0.0 < o["clip_frac"] < 1.0
    assert np.all(o["dtheta"][2] == 0.0)
    for i in range(R):
        for j in range(2 * d):
            e = np.zeros_like(th)
            e[i, j] = 1e-7
            num = (oracle.policy_loss(th + e, old, x, A, **kw)["loss"] - oracle.policy_loss(th - e, old, x, A, **kw)["loss"]) / 2e-7
            assert abs(num - o["dtheta"][i, j]) < 2e-7, (i, j)


def test_policy_at_equal_rows():
    """Nothing has moved: the ratio is one, the loss is minus the mean advantage, no event is clipped."""
    rng = np.random.default_rng(6)
    _, old = _rows(rng, 3, 2)
    x, A = rng.uniform(0.02, 0.98, (3, 11, 2)), rng.standard_normal((3, 11))
    o = oracle.policy_loss(old, old, x, A, theta_ref=old, kl_coef=1.0)
    assert abs(o["loss"] + A.mean()) < 1e-14 and o["kl"] == 0.0 and o["clip_frac"] == 0.0


@pytest.mark.parametrize("eps", [0.0, 0.1])
def test_preference_gradient_by_differences(eps):
    rng = np.random.default_rng(7)
    R, P, d = 3, 6, 2
    th, ref = _rows(rng, R, d)
    ch, rj = rng.uniform(0.02, 0.98, (P, 5, d)), rng.uniform(0.02, 0.98, (P, 4, d))
    kw = dict(len_chosen=np.array([5, 0, 3, 9, -2, 1]), len_rejected=np.array([4, 4, 0, 2, 0, 4]), beta=0.7, label_smoothing=eps)
    o = oracle.preference_loss(th, ref, ch, rj, **kw)
    assert o["margin"][4] == 0.0     # both sets empty
    for i in range(R):
        for j in range(2 * d):
            e = np.zeros_like(th)
            e[i, j] = 1e-6
            num = (oracle.preference_loss(th + e, ref, ch, rj, **kw)["loss"] - oracle.preference_loss(th - e, ref, ch, rj, **kw)["loss"]) / 2e-6
            assert abs(num - o["dtheta"][i, j]) < 1e-8, (i, j)


def test_preference_at_equal_rows():
    rng = np.random.default_rng(8)
    _, ref = _rows(rng, 2, 3)
    o = oracle.preference_loss(ref, ref, rng.uniform(0.1, 0.9, (4, 3, 3)), rng.uniform(0.1, 0.9, (4, 3, 3)))
    assert abs(o["loss"] - np.log(2.0)) < 1e-15 and np.all(o["margin"] == 0.0)


def test_group_advantage():
    rng = np.random.default_rng(9)
    r = rng.standard_normal((5, 40))
    m = rng.random((5, 40)) < 0.5
    m[3] = False
    a = oracle.group_advantage(r, m, eps=0.0)
    assert np.all(a[~m] == 0.0)
    for i in (0, 1, 2, 4):
        assert abs(a[i, m[i]].mean()) < 1e-14 and abs(a[i, m[i]].std() - 1.0) < 1e-14
    c = oracle.group_advantage(r, m, normalise=False)
    np.testing.assert_allclose(c[0, m[0]], r[0, m[0]] - r[0, m[0]].mean(), rtol=1e-14)
    assert np.all(oracle.group_advantage(np.full((2, 7), 3.25)) == 0.0)


@pytest.mark.parametrize("shape", [(1, 1), (5, 9), (9, 5), (3, 16, 16), (2, 40, 7)])
def test_orthogonalise_against_its_products(shape):
    rng = np.random.default_rng(10)
    u = rng.standard_normal(shape)
    a, b, c = oracle.learn.NS_COEF
    x = u.reshape((-1,) + shape[-2:])
    x = np.swapaxes(x, 1, 2) if shape[-2] > shape[-1] else x
    x = x / (np.sqrt((x * x).sum((1, 2), keepdims=True)) + 1e-7)
    for _ in range(5):
        A = x @ np.swapaxes(x, 1, 2)
        x = a * x + (b * A + c * (A @ A)) @ x
    x = (np.swapaxes(x, 1, 2) if shape[-2] > shape[-1] else x).reshape(shape)
    np.testing.assert_allclose(oracle.orthogonalise(u), x, atol=1e-12)


def test_muon_step():
    rng = np.random.default_rng(11)
    p, g = rng.standard_normal((2, 6, 4)), rng.standard_normal((2, 6, 4))
    p1, m1 = oracle.muon_step(p, g, np.zeros_like(p), 0.1, weight_decay=0.5)
    np.testing.assert_array_equal(m1, g)
    np.testing.assert_allclose(p1, 0.95 * p - 0.1 * np.sqrt(1.5) * oracle.orthogonalise(1.95 * g), rtol=1e-12, atol=1e-14)
    s = np.linalg.svd((0.95 * p - p1) / (0.1 * np.sqrt(1.5)), compute_uv=False)
    assert s.min() > 0.6 and s.max() < 1.21
