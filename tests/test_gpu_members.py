"""GPU parity of the members on rows of their own (forward, backward) against the oracle,
through the C ABI: normwise 1e-4 for fp32, as for every fp32 network of the library; rows within rounding
of a LeakyReLU kink get no gradient, so that both sides take the same slopes."""
import numpy as np
import pytest

from oracle import mixture as mx
from tests.parity import assert_normwise, to_np
from workloads import gen

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2407_00051_amd as sg  # noqa: E402

TOL, KINK = 1e-4, 1e-4
WIDTHS = (6, 128, 128, 128, 128, 6)


def _dev(arrs):
    return [torch.tensor(a, device="cuda:0") for a in arrs]


def _kinks(W, b, x, off, slope=0.2):
    near = np.zeros(x.shape[0], dtype=bool)
    for m in range(len(off) - 1):
        h = x[off[m]:off[m + 1]].astype(np.float64)
        for l in range(len(W) - 1):
            w = W[l][m].astype(np.float64)
            pre = h @ w.T + b[l][m]
            near[off[m]:off[m + 1]] |= (np.abs(pre) <= KINK * (np.abs(h) @ np.abs(w).T + np.abs(b[l][m]))).any(axis=1)
            h = np.where(pre > 0, pre, slope * pre)
    return near


def _offsets(kind, M, n, seed):
    """Rows of the members: alike, at random, all of one, one each, none at the ends, some of no member."""
    r = np.random.default_rng(seed)
    if kind == "even":
        return np.linspace(0, n, M + 1).astype(np.int64)
    if kind == "random":
        return np.concatenate([[0], np.sort(r.integers(0, n + 1, M - 1)), [n]])
    if kind == "one":
        return np.where(np.arange(M + 1) > M // 2, n, 0)
    if kind == "few":
        return np.minimum(np.arange(M + 1), n)
    return np.clip(np.sort(r.integers(3, n - 2, M + 1)), 3, n - 2)       # a hole before and behind


CASES = [(WIDTHS, 1, 1, "even"), (WIDTHS, 1, 64, "even"), (WIDTHS, 5, 65, "random"), (WIDTHS, 8, 2048, "random"), (WIDTHS, 3, 300, "hole"),
         (WIDTHS, 130, 300, "random"), (WIDTHS, 70, 40, "few"), (WIDTHS, 9, 500, "one"), (WIDTHS, 4, 9000, "random"),
         (WIDTHS, 4, 9000, "one"), (WIDTHS, 66, 20011, "random"), (WIDTHS, 2, 40000, "hole"),
         ((4, 128, 128, 2), 3, 700, "random"), ((8, 128, 128, 128, 8), 2, 9001, "random"), ((1, 128, 128, 128, 5), 7, 77, "hole"),
         ((8, 128, 128, 1), 12, 12000, "even")]


@pytest.mark.parametrize("widths,M,n,kind", CASES)
def test_members_match_oracle(gpu_ctx, widths, M, n, kind):
    print(f"case members {widths} M={M} n={n} {kind}", flush=True)
    W, b = gen.generator_stack(widths, M, seed=M + n)
    off = _offsets(kind, M, n, M)
    x = gen.noise(n, widths[0], seed=n)
    xd, od = torch.tensor(x, device="cuda:0"), torch.tensor(off.astype(np.int32), device="cuda:0")
    held = torch.full((n, widths[-1]), 7.0, device="cuda:0")
    got = to_np(gpu_ctx.gen_forward_routed(_dev(W), _dev(b), xd, od, out=held))
    ref = mx.members_forward(W, b, x, off)
    on = ~np.isnan(ref[:, 0])
    assert (got[~on] == 7.0).all()
    if on.any():
        assert np.abs(got[on] - ref[on]).max() / np.abs(ref[on]).max() <= TOL
    g = np.random.default_rng(n).standard_normal((n, widths[-1])).astype(np.float32)
    g[_kinks(W, b, x, off)] = 0.0
    gd = torch.tensor(g, device="cuda:0")
    gd[torch.tensor(~on, device="cuda:0")] = float("nan")              # rows of no member are not looked at
    dx = torch.full((n, widths[0]), 7.0, device="cuda:0")
    dW, db, dx = gpu_ctx.gen_backward_routed(_dev(W), _dev(b), xd, od, gd, dx=dx)
    torch.cuda.synchronize()
    rW, rb, rx = mx.members_backward(W, b, x, off, g)
    for l in range(len(W)):
        assert_normwise(to_np(dW[l]), rW[l], TOL, f"dW[{l}]")
        assert_normwise(to_np(db[l]), rb[l], TOL, f"db[{l}]")
        empty = np.diff(off) == 0
        assert (to_np(dW[l])[empty] == 0).all() and (to_np(db[l])[empty] == 0).all()
        for m in np.flatnonzero(~empty)[:4]:                           # and a member at a time
            assert_normwise(to_np(dW[l])[m], rW[l][m], TOL, f"dW[{l}] member {m}")
    assert (to_np(dx)[~on] == 7.0).all()
    if on.any():
        assert_normwise(to_np(dx)[on], rx[on], TOL, "dx")
    # without dx, and again: the same bits
    dW2, db2, none = gpu_ctx.gen_backward_routed(_dev(W), _dev(b), xd, od, gd)
    assert none is None and all(torch.equal(p, q) for p, q in zip(dW + db, dW2 + db2))


@pytest.mark.parametrize("n", [500, 20000])
def test_offsets_outside_the_rows_are_taken_as_the_nearer_end(gpu_ctx, n):
    W, b = gen.generator_stack(WIDTHS, 3, seed=1)
    x = torch.tensor(gen.noise(n, 6, seed=2), device="cuda:0")
    g = torch.ones((n, 6), device="cuda:0")
    wild = torch.tensor([-9, n // 2, n // 2, 2 ** 31 - 1], dtype=torch.int32, device="cuda:0")
    tame = torch.tensor([0, n // 2, n // 2, n], dtype=torch.int32, device="cuda:0")
    a, c = (gpu_ctx.gen_forward_routed(_dev(W), _dev(b), x, o) for o in (wild, tame))
    p, q = (gpu_ctx.gen_backward_routed(_dev(W), _dev(b), x, o, g, want_dx=True) for o in (wild, tame))
    torch.cuda.synchronize()
    assert torch.equal(a, c) and torch.equal(p[2], q[2]) and all(torch.equal(s, t) for s, t in zip(p[0] + p[1], q[0] + q[1]))


def test_offsets_pass_32_bits(gpu_ctx):
    """370,000,000 rows of 6 (8.9 GB an array): the last member's 1,000 agree with a call of their own."""
    if torch.cuda.get_device_properties(0).total_memory < 96 << 30:
        pytest.skip("needs 96 GB")
    print("case rows 370000000", flush=True)
    n, last = 370_000_000, 1000
    W, b = gen.generator_stack((6, 128, 128, 6), 2, seed=3)
    x, g = torch.zeros((n, 6), device="cuda:0"), torch.zeros((n, 6), device="cuda:0")
    noise = gen.noise(last, 6, seed=4)
    dth = np.random.default_rng(5).standard_normal((last, 6)).astype(np.float32)
    dth[_kinks(W, b, noise, [0, 0, last])] = 0.0
    x[-last:], g[-last:] = torch.tensor(noise, device="cuda:0"), torch.tensor(dth, device="cuda:0")
    W, b = _dev(W), _dev(b)
    off = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda:0")     # noqa: E731
    theta = gpu_ctx.gen_forward_routed(W, b, x, off(0, n - last, n))
    own = gpu_ctx.gen_forward_routed(W, b, x[-last:].clone(), off(0, 0, last))
    dW, db, dx = gpu_ctx.gen_backward_routed(W, b, x, off(0, n - last, n), g, want_dx=True)
    ownW, ownb, owndx = gpu_ctx.gen_backward_routed(W, b, x[-last:].clone(), off(0, 0, last), g[-last:].clone(), want_dx=True)
    torch.cuda.synchronize()
    # either form of the tiles is within the library's normwise bar of the exact result
    near = lambda a, c: ((a - c).abs() <= 2 * TOL * c.abs().max()).all()     # noqa: E731
    assert near(theta[-last:], own) and near(dx[-last:], owndx)
    assert all(near(a[1], c[1]) for a, c in zip(dW + db, ownW + ownb))
    assert all((a[0] == 0).all() for a in dW + db)                           # no gradient, and none of a neighbour's
    assert torch.equal(theta[:64], theta[n - last - 64:n - last])            # equal inputs


def test_agrees_with_the_whole_stack(gpu_ctx):
    """Every member on the same rows, by gen_forward / gen_backward, and on copies of its own."""
    M, k = 4, 1100
    W, b = gen.generator_stack(WIDTHS, M, seed=8)
    n = torch.tensor(gen.noise(k, 6, seed=9), device="cuda:0")
    g = torch.randn((M, k, 6), device="cuda:0")
    off = torch.arange(M + 1, device="cuda:0", dtype=torch.int32) * k
    a = gpu_ctx.gen_forward(_dev(W), _dev(b), n)
    c = gpu_ctx.gen_forward_routed(_dev(W), _dev(b), n.repeat(M, 1), off)
    p = gpu_ctx.gen_backward(_dev(W), _dev(b), n, g)
    q = gpu_ctx.gen_backward_routed(_dev(W), _dev(b), n.repeat(M, 1), off, g.reshape(M * k, 6))
    torch.cuda.synchronize()
    assert (a.reshape(M * k, 6) - c).abs().max().item() <= 1e-5 * a.abs().max().item()
    for s, t in zip(p[0] + p[1], q[0] + q[1]):
        assert_normwise(to_np(t), to_np(s), TOL, "gradient")


def test_refusals(gpu_ctx):
    W, b = gen.generator_stack(WIDTHS, 2, seed=1)
    W, b = _dev(W), _dev(b)
    x, off = torch.zeros((10, 6), device="cuda:0"), torch.tensor([0, 5, 10], dtype=torch.int32, device="cuda:0")
    with pytest.raises(ValueError):
        gpu_ctx.gen_forward_routed(W, b, x, off[:2])
    with pytest.raises(TypeError):
        gpu_ctx.gen_forward_routed(W, b, x, off.long())
    with pytest.raises(sg.SagipsError):
        gpu_ctx.gen_forward_routed(W, b, x[:0], off)
    with pytest.raises(sg.SagipsError):
        gpu_ctx.gen_forward_routed(W, b, x, off, out=x)
    with pytest.raises(ValueError):
        gpu_ctx.gen_backward_routed(W, b, x, off, torch.zeros((9, 6), device="cuda:0"))
    with pytest.raises(sg.SagipsError):
        gpu_ctx.gen_backward_routed(W, b, x, off, torch.zeros((10, 6), device="cuda:0"), dx=x)
