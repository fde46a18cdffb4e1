"""Pins of the mixture oracle: closed forms, scipy, torch autograd, central differences and a
sort in pure Python."""
import numpy as np
import pytest
from scipy.special import log_softmax
from scipy.stats import entropy

from oracle import mixture as mx
from workloads import gen


def test_log_probs_and_entropy_against_scipy():
    x = 3.0 * np.random.default_rng(0).standard_normal((7, 19))
    f = mx.choice_logprob(x, np.arange(7), 3, 0.7)
    lp = log_softmax(0.7 * x, axis=1)
    np.testing.assert_allclose(f["logp"], lp[np.arange(7), np.arange(7)], rtol=1e-13)
    np.testing.assert_allclose(f["entropy"], entropy(np.exp(lp), axis=1), rtol=1e-12)
    np.testing.assert_allclose(f["top_logp"], -np.sort(-lp, axis=1)[:, :3], rtol=1e-13)


def test_masks_ties_and_padding():
    inf = np.inf
    x = np.array([[1.0, 2.0, 2.0, -inf], [-inf, -inf, -inf, -inf], [0.0, -0.0, 0.0, -inf]])
    f = mx.choice_logprob(x, np.array([3, 0, 7]), 5)
    assert f["top_choice"].tolist() == [[1, 2, 0, -1, -1], [-1] * 5, [0, 1, 2, -1, -1]]
    assert f["logp"].tolist() == [-inf, -inf, 0.0] and f["entropy"][1] == 0.0
    np.testing.assert_allclose(f["entropy"][2], np.log(3.0))


@pytest.mark.parametrize("scale", [1.0, 0.6])
def test_choice_gradient_against_autograd_and_differences(scale):
    import torch
    r = np.random.default_rng(1)
    x = 2.0 * r.standard_normal((5, 9))
    c, gl, gH, gt = np.array([0, 3, -1, 8, 2]), r.standard_normal(5), r.standard_normal(5), r.standard_normal((5, 2))
    got = mx.choice_backward(x, c, gl, gH, gt, scale)
    idx = mx.choice_logprob(x, c, 2, scale)["top_choice"]
    t = torch.tensor(x, requires_grad=True)
    lp = torch.log_softmax(scale * t, 1)
    on = torch.tensor(c >= 0)
    loss = (torch.tensor(gl) * torch.where(on, lp[torch.arange(5), torch.tensor(c).clamp(min=0)], torch.zeros(()))).sum()
    loss = loss - (torch.tensor(gH) * (lp.exp() * lp).sum(1)).sum() + (torch.tensor(gt) * lp.gather(1, torch.tensor(idx))).sum()
    loss.backward()
    np.testing.assert_allclose(got, t.grad.numpy(), rtol=1e-10, atol=1e-12)

    def value(y):
        f = mx.choice_logprob(y, c, 0, scale)
        return (gl * f["logp"]).sum() + (gH * f["entropy"]).sum() + (gt * np.take_along_axis(mx.log_probs(y, scale), idx, 1)).sum()
    h = 1e-5
    for r_, v in ((0, 0), (1, 5), (2, 2), (3, 8)):
        up, down = x.copy(), x.copy()
        up[r_, v] += h
        down[r_, v] -= h
        assert abs((value(up) - value(down)) / (2 * h) - got[r_, v]) < 1e-8


def test_route_against_a_plain_sort():
    m = np.random.default_rng(2).integers(-1, 6, (40, 3))
    p = mx.route(m, 5)
    want = sorted((int(v), i) for i, v in enumerate(m.reshape(-1)) if 0 <= v < 5)
    assert [i for _, i in want] == p["order"][:len(want)].tolist() and (p["order"][len(want):] == -1).all()
    for k in range(5):
        assert p["offsets"][k + 1] - p["offsets"][k] == sum(v == k for v, _ in want)
    flat = p["place"].reshape(-1)
    assert all(flat[i] == j for j, (_, i) in enumerate(want)) and (flat[m.reshape(-1) >= 5] == -1).all()


def test_combine_and_its_gradient():
    r = np.random.default_rng(3)
    m = r.integers(-1, 4, (9, 2))
    p = mx.route(m, 4)
    y, w, g = r.standard_normal((18, 5)), r.standard_normal((9, 2)), r.standard_normal((9, 5))
    out, _ = mx.combine(y, p["place"], w)
    dy, dw, _ = mx.combine_backward(g, y, p["place"], w)
    on = ~np.isnan(dy[:, 0])
    # out is bilinear in y and w: <g, out> is both inner products
    np.testing.assert_allclose((g * out).sum(), (dy[on] * y[on]).sum(), rtol=1e-12)
    np.testing.assert_allclose((g * out).sum(), (dw * w).sum(), rtol=1e-12)
    assert on.sum() == p["offsets"][-1]
    # dispatch and combine without weights are each other's transpose
    x = r.standard_normal((9, 5))
    s = np.zeros((18, 5))
    for row in range(9):
        for k in range(2):
            if p["place"][row, k] >= 0:
                s[p["place"][row, k]] = x[row]
    np.testing.assert_allclose((s[on] * y[on]).sum(), (x * mx.combine(y, p["place"])[0]).sum(), rtol=1e-12)


def test_members_gradients_against_differences():
    W, b = gen.generator_stack((3, 8, 8, 2), 3, seed=4)
    W, b = [w.astype(np.float64) for w in W], [v.astype(np.float64) for v in b]
    r = np.random.default_rng(5)
    x, g, off = r.standard_normal((10, 3)), r.standard_normal((10, 2)), np.array([0, 4, 4, 9])
    dW, db, dx = mx.members_backward(W, b, x, off, g)
    assert (dW[0][1] == 0).all() and np.isnan(dx[9]).all()

    def value(W, x):
        t = mx.members_forward(W, b, x, off)
        return (g[:9] * t[:9]).sum()
    h = 1e-6
    up, down = x.copy(), x.copy()
    up[6, 1] += h
    down[6, 1] -= h
    assert abs((value(W, up) - value(W, down)) / (2 * h) - dx[6, 1]) < 1e-6
    Wu, Wd = [w.copy() for w in W], [w.copy() for w in W]
    Wu[1][2, 3, 4] += h
    Wd[1][2, 3, 4] -= h
    assert abs((value(Wu, x) - value(Wd, x)) / (2 * h) - dW[1][2, 3, 4]) < 1e-6
