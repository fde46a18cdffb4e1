"""Ends of the ranges that the orthogonalisation accepts, against the float64 oracle.

Tolerances as derived in test_gpu_muon: a perturbation of X grows by at most 3.4445 a step, and a
step's own rounding is at most 8 units in the last place of fp32 of ||X||_F."""
import numpy as np
import pytest

import oracle
from tests.parity import to_np
from tests.test_gpu_muon import _assert_close, _gradients

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


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("shape", [(20, 30), (128, 128), (70, 60), (300, 200)])
def test_norms_far_below_eps(gpu_ctx, shape, bf16):
    """X starts at ||U|| / eps instead of 1, and is held no worse for it: of the result the same part
    is rounding as at ordinary norms."""
    print(f"case norms below eps {shape} bf16={bf16}", flush=True)
    rng = np.random.default_rng(8)
    ratio = 10.0 ** -np.arange(0, 13)
    g = rng.standard_normal((len(ratio),) + shape)
    x = torch.tensor(g * (ratio * 1e-7 / _norm(g))[:, None, None], dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda:0")
    got = to_np(gpu_ctx.orthogonalise(x, eps=1e-7).float()).astype(np.float64)
    ref = oracle.orthogonalise(to_np(x.double()), eps=1e-7)
    tol = 485 * UNIT * ratio + 5 * UNIT * _norm(ref) + (2.0 ** -9 * _norm(ref) if bf16 else 0.0)
    err = _norm(got - ref)
    print(f"  worst of error / tolerance {np.max(err / tol):.3f}", flush=True)
    assert np.all(err <= tol), err / tol


def test_momenta_far_below_eps(gpu_ctx):
    """The step on them: each matrix of a stack at its own scale."""
    rng = np.random.default_rng(9)
    for r, c in ((128, 128), (300, 200)):
        p, m = rng.standard_normal((3, r, c)).astype(np.float32) * 1e-4, np.zeros((3, r, c), np.float32)
        g = rng.standard_normal((3, r, c))
        g = (g * (np.array([1.0, 1e-9, 1e-13]) / _norm(g))[:, None, None]).astype(np.float32)
        tp, tm = torch.tensor(p, device="cuda:0"), torch.tensor(m, device="cuda:0")
        gpu_ctx.muon_step([tp], [torch.tensor(g, device="cuda:0")], [tm], 1.0)
        want, _ = oracle.muon_step(p, g, m, 1.0)
        moved = want - p
        first = np.array([1.0, 1.95e-2, 1.95e-6])          # ||U|| / eps, U = (1 + 0.95) g
        tol = (max(1.0, r / c) ** 0.5 * 485 * first + 5 * _norm(moved)) * UNIT + 2.0 ** -23 * (_norm(p) + _norm(moved))
        err = _norm(to_np(tp) - want)
        assert np.all(err <= tol), err / tol


def test_stacks_beyond_one_part(gpu_ctx):
    """Matrices go in parts of 2 GiB of workspace (255 of 1 x 16,384); a part may begin inside a tensor."""
    rng = np.random.default_rng(10)
    shape = (1, 16384)
    x = rng.standard_normal((300,) + shape).astype(np.float32)
    t = torch.tensor(x, device="cuda:0")
    got = gpu_ctx.orthogonalise(t)
    _assert_close(to_np(got), oracle.orthogonalise(x.astype(np.float64)), False)
    assert torch.equal(got[:150], gpu_ctx.orthogonalise(t[:150].clone())) and torch.equal(got[150:], gpu_ctx.orthogonalise(t[150:].clone()))
    p = [torch.randn((150,) + shape, device="cuda:0") for _ in range(2)]
    m = [torch.zeros_like(v) for v in p]
    own = [[v.clone() for v in s] for s in (p, m)]
    gpu_ctx.muon_step(p, [t[:150], t[150:]], m, 0.1)
    for i in range(2):
        gpu_ctx.muon_step([own[0][i]], [t[150 * i:150 * i + 150].clone()], [own[1][i]], 0.1)
        assert torch.equal(p[i], own[0][i]) and torch.equal(m[i], own[1][i])


def test_coefficients_come_in_threes(gpu_ctx):
    x = torch.zeros((8, 8), device="cuda:0")
    for coef in ((1.5, -0.5), (1.5,), (1.5, -0.5, 0.0, 0.0)):
        with pytest.raises(ValueError, match="three"):
            gpu_ctx.orthogonalise(x, coef=coef)
        with pytest.raises(ValueError, match="three"):
            gpu_ctx.muon_step([x], [torch.zeros_like(x)], [torch.zeros_like(x)], 0.1, coef=coef)


@pytest.mark.parametrize("shape", [(3, 1, 7), (4, 33, 65), (3, 65, 64), (7, 128, 128), (1, 129, 300), (2, 300, 129), (1, 40, 3000),
                                   (300, 16, 20)])
def test_bf16_is_rounded_once(gpu_ctx, shape):
    """bf16 matrices are taken exactly and held in the same terms as fp32 ones; what is left is the
    rounding of the result, 2^-9 of each value."""
    print(f"case bf16 {shape}", flush=True)
    rng = np.random.default_rng(shape[1])
    x = torch.tensor(_gradients(rng, shape), dtype=torch.bfloat16, device="cuda:0")
    got, ref = to_np(gpu_ctx.orthogonalise(x).float()), oracle.orthogonalise(to_np(x.double()))
    tol = (485 + 5 * _norm(ref)) * UNIT + 2.0 ** -9 * _norm(ref)
    assert np.all(_norm(got - ref) <= tol), _norm(got - ref) / tol
