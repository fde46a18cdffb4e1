"""Orthogonalisation and the optimiser step on it on the GPU against the float64
oracle (a singular value decomposition): sizes from 1 to beyond every tile, both
orientations, stacks, several tensors, rank deficiency, extreme scales, NaN.

Tolerances, derived from the arithmetic.  A perturbation of X grows by at most
3.4445 a step (the slope of the polynomial at 0; it is below 3.9 everywhere up to
1.2), 485 in five.  A step's own rounding is at most 8 units in the last place of
fp32 of ||X||_F (three-term products and terms are exact to 2^-24, sums of K terms in
fp32), which starts at 1 and never exceeds 1.3 sqrt(n): so the result's Frobenius
error is at most 485 * 8 * 2^-24 from the first steps and 5 * 8 * 2^-24 * ||O||_F from
the last.  Two-term operands: 4 * 2^-17 instead of 8 * 2^-24, and the rounding to
bf16, 2^-9 of each value."""
import numpy as np
import pytest

import oracle
from tests.parity import to_np

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2407_00051_amd as sg  # noqa: E402

SHAPES = [(1, 1, 1), (3, 1, 7), (2, 7, 1), (5, 5, 5), (4, 33, 65), (2, 64, 64), (3, 65, 64), (7, 128, 128), (2, 100, 127),
          (1, 129, 300), (2, 300, 129), (5, 6, 128), (5, 128, 6), (1, 513, 40), (2, 31, 700), (1, 257, 255), (1, 512, 512),
          (1, 40, 3000), (300, 16, 20)]


def _tol(ref, bf16):
    unit = 4 * 2.0 ** -17 if bf16 else 8 * 2.0 ** -24
    norm = np.sqrt((ref ** 2).sum((-2, -1)))
    return 485 * unit + 5 * unit * norm + (2.0 ** -9 * norm if bf16 else 0.0)


def _gradients(rng, shape):
    """A few strong directions over a noise floor."""
    n, r, c = shape
    k = min(4, r, c)
    return (rng.standard_normal((n, r, k)) * 0.5 ** np.arange(k)) @ rng.standard_normal((n, k, c)) + 0.1 * rng.standard_normal(shape)


def _assert_close(got, ref, bf16, scale=1.0):
    err = np.sqrt(((got.astype(np.float64) - ref) ** 2).sum((-2, -1)))
    tol = scale * _tol(ref / scale, bf16)
    print(f"  worst of error / tolerance {np.max(err / tol):.3f}", flush=True)
    assert np.all(err <= tol), (err / tol).max()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_orthogonalise(gpu_ctx, shape, bf16):
    print(f"case orthogonalise {shape} bf16={bf16}", flush=True)
    rng = np.random.default_rng(shape[1] * 31 + shape[2])
    x = torch.tensor(_gradients(rng, shape), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda:0")
    got = gpu_ctx.orthogonalise(x)
    assert got.dtype == x.dtype and got.shape == x.shape
    _assert_close(to_np(got.float()), oracle.orthogonalise(to_np(x.double())), bf16)
    assert torch.equal(got, gpu_ctx.orthogonalise(x))
    y = x.clone()
    assert gpu_ctx.orthogonalise(y, out=y) is y and torch.equal(y, got)


@pytest.mark.parametrize("shape", [(3, 20, 30), (2, 128, 128), (1, 200, 150)])
def test_orthogonalise_hard_matrices(gpu_ctx, shape):
    """Zero, rank one, duplicated rows, orthogonal already, extreme scales; each beside ordinary ones."""
    print(f"case hard matrices {shape}", flush=True)
    rng = np.random.default_rng(1)
    n, r, c = shape
    g = rng.standard_normal(shape)
    one = rng.standard_normal((n, r, 1)) @ rng.standard_normal((n, 1, c))
    dup = np.repeat(rng.standard_normal((n, (r + 1) // 2, c)), 2, axis=1)[:, :r]
    q = np.linalg.qr(rng.standard_normal((n, max(r, c), min(r, c))))[0]
    q = np.swapaxes(q, 1, 2) if r < c else q
    all_ = np.concatenate([g, np.zeros(shape), one, dup, q, 1e-18 * g, 1e-30 * g, 1e30 * g]).astype(np.float32)
    got = to_np(gpu_ctx.orthogonalise(torch.tensor(all_, device="cuda:0"), eps=1e-37))
    assert np.all(got[n:2 * n] == 0.0)
    _assert_close(got, oracle.orthogonalise(all_.astype(np.float64), eps=1e-37), False)


def test_orthogonalise_nan_stays_in_its_matrix(gpu_ctx):
    rng = np.random.default_rng(2)
    for r, c in ((30, 40), (200, 180)):
        x = _gradients(rng, (4, r, c)).astype(np.float32)
        x[1, 3, 5] = np.nan
        x[2, 0, 0] = np.inf
        got = to_np(gpu_ctx.orthogonalise(torch.tensor(x, device="cuda:0")))
        assert np.isnan(got[1]).all() and np.isnan(got[2]).all()
        _assert_close(got[[0, 3]], oracle.orthogonalise(x[[0, 3]].astype(np.float64)), False)


def test_orthogonalise_steps_and_coefficients(gpu_ctx):
    rng = np.random.default_rng(3)
    for shape in ((2, 48, 80), (1, 150, 140)):
        x = _gradients(rng, shape).astype(np.float32)
        for steps, coef in ((1, (1.5, -0.5, 0.0)), (3, (2.0, -1.5, 0.5)), (10, (1.875, -1.25, 0.375))):
            got = to_np(gpu_ctx.orthogonalise(torch.tensor(x, device="cuda:0"), steps=steps, coef=coef))
            ref = oracle.orthogonalise(x.astype(np.float64), steps, coef)
            err = np.sqrt(((got - ref) ** 2).sum((1, 2)))
            # slopes of these polynomials are at most coef[0] on [0, 1]
            assert np.all(err <= (coef[0] ** steps + steps * np.sqrt((ref ** 2).sum((1, 2)))) * 8 * 2.0 ** -24)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("nesterov,scale", [(True, "shape"), (False, "rms"), (True, "none")])
def test_muon_step(gpu_ctx, bf16, nesterov, scale):
    """Several steps on tensors of several shapes, two of them alike."""
    print(f"case muon_step bf16={bf16} nesterov={nesterov} scale={scale}", flush=True)
    rng = np.random.default_rng(4)
    shapes = [(128, 128), (3, 128, 6), (128, 128), (2, 6, 128), (200, 150), (3, 64, 100), (1, 1)]
    p = [rng.standard_normal(s).astype(np.float32) for s in shapes]
    m = [np.zeros(s, np.float32) for s in shapes]
    tp, tm = [torch.tensor(a, device="cuda:0") for a in p], [torch.tensor(a, device="cuda:0") for a in m]
    kw = dict(momentum=0.9, nesterov=nesterov, weight_decay=0.1)
    code = {"none": sg.SCALE_NONE, "shape": sg.SCALE_SHAPE, "rms": sg.SCALE_RMS}[scale]
    for step in range(3):
        g = [torch.tensor(_gradients(rng, (1,) * (3 - len(s)) + s).reshape(s), dtype=torch.bfloat16 if bf16 else torch.float32,
                          device="cuda:0") for s in shapes]
        gpu_ctx.muon_step(tp, g, tm, 0.05, scale=code, **kw)
        for i, s in enumerate(shapes):
            want_p, want_m = oracle.muon_step(p[i], to_np(g[i].double()), m[i], 0.05, scale=scale, **kw)
            got_p, got_m = to_np(tp[i]), to_np(tm[i])
            assert np.abs(got_m - want_m).max() <= 2.0 ** -23 * np.abs(want_m).max() * 2
            moved = (1.0 - 0.05 * 0.1) * p[i].astype(np.float64) - want_p
            size = 0.05 * {"none": 1.0, "shape": max(1.0, s[-2] / s[-1]) ** 0.5, "rms": 0.2 * max(s[-2:]) ** 0.5}[scale]
            err = np.sqrt(((got_p - want_p) ** 2).sum((-2, -1)))
            tol = size * _tol(moved / size, False) + 2.0 ** -22 * np.sqrt((want_p ** 2).sum((-2, -1)))
            assert np.all(err <= tol), (step, s, (err / tol).max())
            p[i], m[i] = got_p, got_m          # each step from what the GPU holds


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("shape", [(1, 3, 5), (3, 9, 11), (1, 127, 129), (3, 131, 61), (3, 3, 4), (1, 9, 12), (1, 135, 300)])
def test_muon_step_on_parts_of_a_packed_stack(gpu_ctx, shape, bf16):
    """Arrays that start wherever the one before them ends give what arrays of their own give."""
    print(f"case packed {shape} bf16={bf16}", flush=True)
    rng = np.random.default_rng(shape[1] * 7 + shape[2])
    dtype = torch.bfloat16 if bf16 else torch.float32
    g = torch.tensor(_gradients(rng, (3 * shape[0],) + shape[1:]), dtype=dtype, device="cuda:0").reshape((3,) + shape)
    p, m = (torch.tensor(rng.standard_normal((3,) + shape), dtype=torch.float32, device="cuda:0") for _ in range(2))
    own = [[t[i].clone() for i in range(3)] for t in (p, g, m)]
    gpu_ctx.muon_step(list(p), list(g), list(m), 0.05)
    gpu_ctx.muon_step(*own, 0.05)
    for i in range(3):
        assert torch.equal(p[i], own[0][i]) and torch.equal(m[i], own[2][i])


def test_muon_step_refuses_quads_off_their_alignment(gpu_ctx):
    buf = torch.zeros(3, 4 * 8 + 4, device="cuda:0")
    part = lambda i, off, dtype=torch.float32: buf[i].view(dtype)[off:off + 32].view(4, 8)      # noqa: E731
    gpu_ctx.muon_step([part(0, 4)], [part(1, 0)], [part(2, 4)], 0.1)
    for off in ((1, 0, 0), (0, 2, 0), (0, 0, 3)):
        with pytest.raises(sg.SagipsError, match="aligned to 4 values"):
            gpu_ctx.muon_step(*([part(i, off[i])] for i in range(3)), 0.1)
    gpu_ctx.muon_step([part(0, 0)], [part(1, 4, torch.bfloat16)], [part(2, 0)], 0.1)
    with pytest.raises(sg.SagipsError, match="aligned to 4 values"):
        gpu_ctx.muon_step([part(0, 0)], [part(1, 2, torch.bfloat16)], [part(2, 0)], 0.1)


def test_muon_on_a_stream_of_its_own(gpu_ctx):
    rng = np.random.default_rng(5)
    g = torch.tensor(_gradients(rng, (20, 128, 128)), dtype=torch.float32, device="cuda:0")
    big = torch.tensor(_gradients(rng, (1, 200, 300)), dtype=torch.float32, device="cuda:0")
    a, b = gpu_ctx.orthogonalise(g), gpu_ctx.orthogonalise(big)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    ctx = sg.Context(0, stream=st)
    a2, b2 = ctx.orthogonalise(g), ctx.orthogonalise(big)
    st.synchronize()
    ctx.close()
    assert torch.equal(a, a2) and torch.equal(b, b2)


def test_refusals(gpu_ctx):
    z = lambda *s, **k: torch.zeros(s, device="cuda:0", **k)       # noqa: E731
    x = z(2, 8, 8)
    for kw in (dict(eps=0.0), dict(eps=float("nan")), dict(steps=17), dict(coef=(1.0, float("inf"), 0.0))):
        with pytest.raises(sg.SagipsError):
            gpu_ctx.orthogonalise(x, **kw)
    for bad in (z(8), z(2, 2, 8, 8)):
        with pytest.raises(ValueError):
            gpu_ctx.orthogonalise(bad)
    with pytest.raises(TypeError):
        gpu_ctx.orthogonalise(z(8, 8, dtype=torch.float16))
    with pytest.raises(ValueError):
        gpu_ctx.orthogonalise(x.transpose(1, 2)[:, :4])
    with pytest.raises(ValueError):
        gpu_ctx.orthogonalise(x, steps=0)
    for s in ((1, 0, 4), (1, 16385, 1)):
        with pytest.raises(sg.SagipsError):
            gpu_ctx.orthogonalise(z(*s))
    buf = z(64)
    with pytest.raises(sg.SagipsError):
        gpu_ctx.orthogonalise(buf[:32].view(4, 8), out=buf[16:48].view(4, 8))
    with pytest.raises(sg.SagipsError):
        gpu_ctx.orthogonalise(buf[1:33].view(4, 8))
    p, g, m = z(8, 8), z(8, 8), z(8, 8)
    for kw in (dict(lr=-1.0), dict(lr=0.1, momentum=1.0), dict(lr=0.1, weight_decay=-1.0), dict(lr=0.1, scale=7),
               dict(lr=float("nan"))):
        with pytest.raises(sg.SagipsError):
            gpu_ctx.muon_step([p], [g], [m], **kw)
    with pytest.raises(sg.SagipsError):
        gpu_ctx.muon_step([p], [p], [m], 0.1)
    with pytest.raises(sg.SagipsError):
        gpu_ctx.muon_step([p, p], [g, g], [m, z(8, 8)], 0.1)
    with pytest.raises(ValueError):
        gpu_ctx.muon_step([p], [g], [], 0.1)
    with pytest.raises(ValueError):
        gpu_ctx.muon_step([p], [z(8, 4)], [m], 0.1)
    with pytest.raises(TypeError):
        gpu_ctx.muon_step([p, z(8, 8)], [g, g.bfloat16()], [m, z(8, 8)], 0.1)
    with pytest.raises(ValueError):
        gpu_ctx.muon_step([z(8, 8) for _ in range(17)], [g] * 17, [m] * 17, 0.1)
    assert torch.count_nonzero(p).item() == 0
