"""Members on rows of their own, to the last bits: stacks of which every feature reads one feature of the layer before
(random permutations with 24-bit weights), so that an output is a chain of products with nothing to add or to cancel, and
an error of one product shows in it.  Every value is positive; u = 2^-24.

A product on the matrix cores is six products of bf16 terms: at most u for the terms left out, five additions onto the
full-size sum of 2 u each (whatever the cores' rounding): 11 u.  The zeros beside it add exactly.  So, relative, with h
hidden-to-hidden layers:
  o       1 (first layer) + 11 h + 1 (last) u; theta = 1 + softplus(o) moves by less, and adds 2 u: (11 h + 4) u,
  dx      sigmoid(o): e^-o <= 0.02 is off by (1 - sigma) o (11 h + 2) u <= 0.08 (11 h + 2) u, a sum and a division
          4 u; one product each of dL/dtheta, the last and the first layer, 11 h for the hidden ones, and at most
          `out` terms a column, whose sum rounds out u: (11.88 h + 8 + out) u,
  dW, db  one row a member: the signal (at most dx's without its sum), the activation (1 + 11 h) u, one product 11 u:
          (22.88 h + 20) u; a feature that is not on a chain has exactly 0.
A product of two terms a value instead of three is off by up to 128 u a factor: test_two_terms_would_show."""
import numpy as np
import pytest

from oracle import mixture as mx
from tests.parity import to_np

torch = pytest.importorskip("torch")

U = 2.0 ** -24
H = 128


def _chains(widths, M, n, seed):
    """Weights of M members, biases of 0, inputs and derivatives of n rows, all in 24 random bits: o lies in [4, 256]."""
    r = np.random.default_rng(seed)
    value = lambda lo, *s: (lo * (1.0 + r.random(s))).astype(np.float32)     # noqa: E731
    W = []
    for l, (a, b) in enumerate(zip(widths, widths[1:])):
        w = np.zeros((M, b, a), np.float32)
        for m in range(M):
            at = np.arange(b) % a if l == 0 else r.permutation(a)[:b]
            w[m, np.arange(b), at] = value(4.0 if l == len(widths) - 2 else 1.0, b)
        W.append(w)
    return W, [np.zeros((M, b), np.float32) for b in widths[1:]], value(1.0, n, widths[0]), value(1.0, n, widths[-1])


def _near(got, want, bar, what):
    assert (got[want == 0] == 0).all(), what
    on = want != 0
    worst = float((np.abs(got[on] - want[on]) / want[on]).max()) / U
    print(f"  {what}: {worst:.1f} u (bar {bar:.1f} u)", flush=True)
    assert worst <= bar, (what, worst, bar)


# one row a member: tiles of 16 rows, and of 64; rows enough for the forward pass's tiles of 64
@pytest.mark.gpu
@pytest.mark.parametrize("widths", [(6, H, H, H, H, 6), (4, H, H, H, 3), (8, H, H, 8)])
@pytest.mark.parametrize("M,n", [(40, 40), (300, 300), (8, 9000), (3, 70)])
def test_every_product_to_fp32(gpu_ctx, widths, M, n):
    print(f"case chains {widths} M={M} n={n}", flush=True)
    h, out = len(widths) - 3, widths[-1]
    W, b, x, g = _chains(widths, M, n, M + n + h)
    off = np.arange(M + 1) * n // M
    dev = lambda a: torch.tensor(a, device="cuda:0")                        # noqa: E731
    Wd, bd, xd, od = [dev(w) for w in W], [dev(v) for v in b], dev(x), dev(off.astype(np.int32))
    theta = to_np(gpu_ctx.gen_forward_routed(Wd, bd, xd, od)).astype(np.float64)
    dW, db, dx = gpu_ctx.gen_backward_routed(Wd, bd, xd, od, dev(g), want_dx=True)
    torch.cuda.synchronize()
    _near(theta, mx.members_forward(W, b, x, off), 11 * h + 4, "theta")
    rW, rb, rx = mx.members_backward(W, b, x, off, g)
    _near(to_np(dx).astype(np.float64), rx, 11.88 * h + 8 + out, "dx")
    if n == M:
        for l in range(len(W)):
            _near(to_np(dW[l]).astype(np.float64), rW[l], 22.88 * h + 20, f"dW[{l}]")
            _near(to_np(db[l]).astype(np.float64), rb[l], 22.88 * h + 20, f"db[{l}]")


@pytest.mark.gpu
@pytest.mark.parametrize("n,at", [(50, 0), (50, 50), (300, 7), (20000, 0), (20000, 20000)])
def test_no_member_has_rows(gpu_ctx, n, at):
    """Offsets that are all the same: no row is looked at or written, and every gradient of a parameter is 0."""
    print(f"case empty n={n} at={at}", flush=True)
    W, b, x, g = _chains((6, H, H, H, H, 6), 70, n, 1)
    dev = lambda a: torch.tensor(a, device="cuda:0")                        # noqa: E731
    Wd, bd = [dev(w) for w in W], [dev(v) for v in b]
    off = torch.full((71,), at, dtype=torch.int32, device="cuda:0")
    held = torch.full((n, 6), 7.0, device="cuda:0")
    x, g = torch.full_like(held, float("nan")), torch.full_like(held, float("nan"))
    theta = gpu_ctx.gen_forward_routed(Wd, bd, x, off, out=held.clone())
    dW, db, dx = gpu_ctx.gen_backward_routed(Wd, bd, x, off, g, dx=held.clone())
    torch.cuda.synchronize()
    assert torch.equal(theta, held) and torch.equal(dx, held) and all((t == 0).all() for t in dW + db)


def _bf16(x):
    return torch.tensor(np.asarray(x, dtype=np.float64)).float().bfloat16().double().numpy()



def _two(x):
    """x without its third term."""
    x = np.asarray(x, dtype=np.float32).astype(np.float64)
    hi = _bf16(x)
    return hi + _bf16(x - hi)


def test_two_terms_would_show():
    """The bars lie below what chains of two-term products are off by: forward and the gradient of a hidden layer."""
    widths, M, h = (6, H, H, H, H, 6), 40, 3
    W, b, x, g = _chains(widths, M, M, 2)
    off = np.arange(M + 1)
    cut = [W[0]] + [_two(w) for w in W[1:-1]] + [W[-1]]
    ref, got = mx.members_forward(W, b, x, off), mx.members_forward(cut, b, x, off)
    assert (np.abs(got - ref) / ref).max() > 1.5 * (11 * h + 4) * U
    rW, _, rx = mx.members_backward(W, b, x, off, g)
    _, _, gx = mx.members_backward(cut, b, x, off, g)
    on = rx != 0
    assert (np.abs(gx[on] - rx[on]) / rx[on]).max() > 1.5 * (11.88 * h + 14) * U
    # an outer product of which either side is cut
    d, A = np.float32(1.0) + np.random.default_rng(1).random((2, 4000), dtype=np.float32)
    exact = d.astype(np.float64) * A
    assert (np.abs(_two(d) * _two(A) - exact) / exact).max() > 1.5 * (22.88 * h + 20) * U
