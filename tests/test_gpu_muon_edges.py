"""Ends of the ranges that the orthogonalisation accepts, against the float64 oracle.

Tolerances as derived in test_gpu_muon: a perturbation of X grows by at most 3.4445 a step, and a
step's own rounding is at most 8 units in the last place of fp32 of ||X||_F."""
import numpy as np
import pytest

import oracle
from tests.parity import to_np
from tests.test_gpu_muon import _assert_close

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

UNIT = 8 * 2.0 ** -24


def _norm(a):
    return np.sqrt((np.asarray(a, np.float64) ** 2).sum((-2, -1)))


@pytest.mark.parametrize("shape", [(20, 30), (60, 64), (128, 128), (200, 150)])
@pytest.mark.parametrize("steps,coef", [(2, (2.9, -0.25, 0.0)), (1, (3.89, 0.0, 0.0)), (2, (2.95, -0.26, 0.0))])
def test_coefficients_up_to_the_bound(gpu_ctx, shape, steps, coef):
    """A matrix of rank one starts with a singular value of 1, the largest there is; the accepted
    coefficients take it up to 3.9 whatever the matrix's size."""
    print(f"case coefficients {shape} {coef}", flush=True)
    x = np.zeros((2,) + shape, np.float32)
    x[0, 3, 5] = 2.0
    x[1] = np.outer(np.sin(np.arange(shape[0]) + 1.0), np.cos(np.arange(shape[1])))
    got = to_np(gpu_ctx.orthogonalise(torch.tensor(x, device="cuda:0"), steps=steps, coef=coef)).astype(np.float64)
    ref = oracle.orthogonalise(x.astype(np.float64), steps, coef)
    assert _norm(ref)[0] > 2.8
    # slopes are at most coef[0] + 3 |b| s^2 + 5 |c| s^4 below 8 for the s of these steps (at most 2.7)
    tol = sum(8.0 ** k for k in range(steps + 1)) * UNIT * 3.9
    assert np.all(_norm(got - ref) <= tol), _norm(got - ref) / tol


@pytest.mark.parametrize("shape", [(20, 30), (128, 128), (200, 150)])
def test_norms_and_eps_at_the_ends(gpu_ctx, shape):
    """Zero matrices, subnormal ones and ones near the largest number, at an eps below fp32's range."""
    print(f"case norms {shape}", flush=True)
    rng = np.random.default_rng(7)
    g = rng.standard_normal(shape)
    x = np.stack([g, 0.0 * g, np.sign(g) * 3e38, 1e-42 * g, 1e-39 * g]).astype(np.float32)
    got = to_np(gpu_ctx.orthogonalise(torch.tensor(x, device="cuda:0"), eps=1e-60))
    assert np.all(got[1] == 0.0)
    _assert_close(got, oracle.orthogonalise(x.astype(np.float64), eps=1e-60), False)
