"""The operators of a mixture of generators run together, as paper_2407_00051_amd/mixture.py and gan.py call them:
against a float64 composition of the oracle, in HIP graphs, on other streams and contexts, and in the
GAN loop."""
import numpy as np
import pytest

from oracle import mixture as mx
from tests.parity import assert_normwise, to_np
from workloads import gen

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2407_00051_amd as sg  # noqa: E402
from paper_2407_00051_amd import gan  # noqa: E402
from paper_2407_00051_amd.mixture import Mixture  # noqa: E402

TOL, KINK = 1e-4, 1e-4        # fp32 networks: the library's normwise bar
WIDTHS = (6, 128, 128, 128, 128, 6)


def _setup(M, k, seed, dev="cuda:0"):
    W, b = gen.generator_stack(WIDTHS, M, seed=seed)
    r = np.random.default_rng(seed)
    Wr, br = r.standard_normal((M, 6)).astype(np.float32), 0.3 * r.standard_normal(M).astype(np.float32)
    n = gen.noise(k, 6, seed=seed + 1)
    t = lambda a: torch.tensor(a, device=dev)      # noqa: E731
    return (W, b, Wr, br, n), ([t(w) for w in W], [t(v) for v in b], t(Wr), t(br), t(n))


def _oracle(W, b, Wr, br, n, g, top, entropy_coef):
    """theta, and the gradients of <g, theta> - entropy_coef mean H, in float64."""
    k, M = n.shape[0], Wr.shape[0]
    logits = n.astype(np.float64) @ Wr.astype(np.float64).T + br
    f = mx.choice_logprob(logits, None, top)
    own = mx.choice_logprob(f["top_logp"], None, top)
    w = np.exp(own["top_logp"])
    p = mx.route(f["top_choice"], M)
    item = p["order"]
    x = n[item // top]
    th = mx.members_forward(W, b, x, p["offsets"])
    theta, _ = mx.combine(th, p["place"], w)
    if g is None:
        return theta, logits, (x, p["offsets"])
    dth, dw, _ = mx.combine_backward(g, th, p["place"], w)
    dW, db, _ = mx.members_backward(W, b, x, p["offsets"], dth)
    d_top = mx.choice_backward(f["top_logp"], None, None, None, dw * w)
    d_logits = mx.choice_backward(logits, None, None, np.full(k, -entropy_coef / k), d_top)
    return theta, dW, db, d_logits.T @ n.astype(np.float64), d_logits.sum(0)


def _definite(W, b, Wr, br, n, top):
    """Rows whose choice or LeakyReLU slopes are not within rounding of another one."""
    theta, logits, (x, off) = _oracle(W, b, Wr, br, n, None, top, 0.0)
    s = np.sort(logits, axis=1)[:, ::-1]
    ok = (s[:, :-1] - s[:, 1:])[:, :top].min(axis=1) > 1e-4 if logits.shape[1] > 1 else np.ones(len(n), bool)
    for m in range(Wr.shape[0]):
        h = n.astype(np.float64)
        for l in range(len(W) - 1):
            w = W[l][m].astype(np.float64)
            pre = h @ w.T + b[l][m]
            ok &= (np.abs(pre) > KINK * (np.abs(h) @ np.abs(w).T + np.abs(b[l][m]))).all(axis=1)
            h = np.where(pre > 0, pre, 0.2 * pre)
    return ok


@pytest.mark.parametrize("M,k,top", [(1, 70, 1), (3, 500, 2), (8, 1024, 2), (5, 300, 5), (8, 4200, 3)])
def test_mixture_matches_oracle(gpu_ctx, M, k, top):
    print(f"case mixture M={M} k={k} top={top}", flush=True)
    (W, b, Wr, br, n), _ = _setup(M, k, M + k)
    n = n[_definite(W, b, Wr, br, n, top)]
    dev = lambda a: torch.tensor(a, device="cuda:0")                  # noqa: E731
    mix = Mixture(gpu_ctx, [dev(w) for w in W], [dev(v) for v in b], dev(Wr), dev(br), top=top, entropy_coef=0.5)
    g = np.random.default_rng(k).standard_normal((len(n), 6)).astype(np.float32)
    theta = mix.forward(dev(n))
    mix.backward(dev(g))
    torch.cuda.synchronize()
    rt, rW, rb, rWr, rbr = _oracle(W, b, Wr, br, n, g, top, 0.5)
    assert_normwise(to_np(theta), rt, TOL, "theta")
    for l in range(len(W)):
        assert_normwise(to_np(mix.dW[l]), rW[l], TOL, f"dW[{l}]")
        assert_normwise(to_np(mix.db[l]), rb[l], TOL, f"db[{l}]")
    assert_normwise(to_np(mix.dWr), rWr, TOL, "dWr")
    assert_normwise(to_np(mix.dbr), rbr, TOL, "dbr")


def test_router_gradient_against_differences(gpu_ctx):
    """d<g, theta> / d br by central differences of the whole pass (h = 2^-6: truncation below
    h^2 / 6 of the third derivative, of order |g theta|; rounding 2^-24 |theta| sqrt(k) / h): 2e-3 of the gradient's
    norm, for rows whose choice stays."""
    (W, b, Wr, br, n), _ = _setup(4, 800, 3)
    logits = np.sort(n @ Wr.T + br, axis=1)[:, ::-1]
    n = n[np.abs(np.diff(logits, axis=1))[:, :2].min(axis=1) > 0.1]
    dev = lambda a: torch.tensor(a, device="cuda:0")                  # noqa: E731
    g = torch.randn((len(n), 6), generator=torch.Generator(device="cuda:0").manual_seed(1), device="cuda:0")
    Wd, bd, nd = [dev(w) for w in W], [dev(v) for v in b], dev(n)
    value = lambda br_: (Mixture(gpu_ctx, Wd, bd, dev(Wr), br_, top=2).forward(nd).double() * g.double()).sum().item()   # noqa: E731
    mix = Mixture(gpu_ctx, Wd, bd, dev(Wr), dev(br), top=2)
    mix.forward(nd)
    mix.backward(g)
    h, num = 2.0 ** -6, []
    for m in range(4):
        e = torch.zeros(4, device="cuda:0")
        e[m] = h
        num.append((value(dev(br) + e) - value(dev(br) - e)) / (2 * h))
    got = to_np(mix.dbr)
    assert np.linalg.norm(got - num) <= 2e-3 * np.linalg.norm(num), (got, num)


def _pass(mix, n, g):
    theta = mix.forward(n)
    mix.backward(g)
    return [theta] + [t for t in mix.gradients()]


@pytest.mark.parametrize("M,k,top", [(3, 40, 2), (8, 1024, 2), (6, 5000, 3)])
def test_replays_equal_eager_calls(M, k, top):
    """The whole pass in one HIP graph: every replay gives bit for bit what eager calls give on the same
    inputs, with eager work and synchronisations between the replays."""
    print(f"case graph M={M} k={k} top={top}", flush=True)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        ctx, eager = sg.Context(0, stream=st), sg.Context(0, stream=st)
        _, (W, b, Wr, br, n) = _setup(M, k, 1)
        g = torch.randn((k, 6), device="cuda:0")
        mix, other = Mixture(ctx, W, b, Wr, br, top=top), Mixture(eager, W, b, Wr, br, top=top)
        _pass(mix, n, g)                                   # workspaces grow here, not in the capture
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            out = _pass(mix, n, g)
        for replay in range(4):
            new = _setup(M, k, 10 + replay)[1]
            for a, c in zip([*W, *b, Wr, br, n], [*new[0], *new[1], *new[2:]]):
                a.copy_(c)
            g.normal_()
            graph.replay()
            st.synchronize()
            got = [t.clone() for t in out]
            want = _pass(other, n, g)
            st.synchronize()
            # positions and sums of the library are deterministic; dWr and dbr are torch's own products
            assert all(torch.equal(a, c) for a, c in zip(got[:-2], want[:-2]))
            assert all(torch.allclose(a, c, rtol=1e-4, atol=1e-4 * c.abs().max().item()) for a, c in zip(got[-2:], want[-2:]))
        st.synchronize()
        ctx.close()
        eager.close()


def test_contexts_on_streams_of_their_own():
    """Two contexts at work at once, each on a stream, neither torch's current one; outputs allocated by the
    binding, inputs dropped at once."""
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    ctxs = [sg.Context(0, stream=s) for s in streams]
    held = [_setup(4, 6000, 20 + i)[1] for i in range(2)]
    g = torch.randn((6000, 6), device="cuda:0")
    torch.cuda.synchronize()
    # the router's products are torch's and run on its stream: members and weights given here
    outs = []
    for i in range(2):
        W, b, Wr, br, n = held[i]
        logits = (n @ Wr.t() + br)
        torch.cuda.synchronize()
        outs.append([])
        for _ in range(3):
            f = ctxs[i].choice_logprob(logits, top=2)
            p = ctxs[i].route(f["top_choice"], 4)
            th = ctxs[i].gen_forward_routed(W, b, ctxs[i].dispatch(n, p), p["offsets"])
            outs[i] = [f["top_logp"], ctxs[i].combine(th, p, f["top_logp"]),
                       *ctxs[i].gen_backward_routed(W, b, ctxs[i].dispatch(n, p), p["offsets"],
                                                    ctxs[i].combine_backward(g, th, p, f["top_logp"])[0])[0]]
    torch.cuda.synchronize()
    one = sg.Context(0)
    for i in range(2):
        W, b, Wr, br, n = held[i]
        f = one.choice_logprob(n @ Wr.t() + br, top=2)
        p = one.route(f["top_choice"], 4)
        th = one.gen_forward_routed(W, b, one.dispatch(n, p), p["offsets"])
        want = [f["top_logp"], one.combine(th, p, f["top_logp"]),
                *one.gen_backward_routed(W, b, one.dispatch(n, p), p["offsets"], one.combine_backward(g, th, p, f["top_logp"])[0])[0]]
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(outs[i], want))
    for c in ctxs + [one]:
        c.close()


def test_mixture_on_a_stream_that_is_not_the_current_one(gpu_ctx):
    """A context on a stream of its own with work queued on it: torch's part of a step runs there too, between
    the library's calls that it depends on, and inputs and results may be dropped at once."""
    print("case mixture on its own stream", flush=True)
    busy = torch.randn((2048, 65536), device="cuda:0")
    results = []
    for own in (False, True):
        _, (W, b, Wr, br, n) = _setup(4, 3000, 30)
        g = torch.ones((3000, 6), device="cuda:0")
        ctx = sg.Context(0, stream=torch.cuda.Stream()) if own else sg.Context(0)
        mix = Mixture(ctx, W, b, Wr, br, entropy_coef=0.1)
        m, v = ([torch.zeros_like(p) for p in mix.parameters()] for _ in range(2))
        torch.cuda.synchronize()
        thetas = []
        for t in range(3):
            ctx.choice_logprob(busy)
            theta = mix.forward(n)
            mix.backward(g)
            ctx.adam_step(mix.parameters(), mix.gradients(), m, v, t + 1, 1e-3)
            with mix.on_stream():
                thetas.append(theta.clone())
            del theta
        torch.cuda.synchronize()
        results.append(thetas + mix.parameters())
        ctx.close()
    # Adam's first steps are lr g / |g|: a gradient's rounding (the library's product may sum in another order) shows
    # only where it is near eps = 1e-8 of the step
    assert all(torch.allclose(a, c, rtol=1e-4, atol=1e-4) for a, c in zip(*results))
    assert not torch.equal(results[0][0], results[0][1])


def test_a_router_that_leaves_a_row_without_members(gpu_ctx):
    """Members masked by -inf take no rows; a row whose members are all masked gives theta 0 and no gradient."""
    x = torch.zeros((3, 4), device="cuda:0")
    x[0, 1:] = float("-inf")
    x[1] = float("-inf")
    f = gpu_ctx.choice_logprob(x, top=2)
    own = gpu_ctx.choice_logprob(f["top_logp"], top=2)
    w = own["top_logp"].exp()
    p = gpu_ctx.route(f["top_choice"], 4)
    W, b = gen.generator_stack(WIDTHS, 4, seed=2)
    W, b = [torch.tensor(v, device="cuda:0") for v in W], [torch.tensor(v, device="cuda:0") for v in b]
    n = torch.randn((3, 6), device="cuda:0")
    th = gpu_ctx.gen_forward_routed(W, b, gpu_ctx.dispatch(n, p), p["offsets"])
    theta = gpu_ctx.combine(th, p, w)
    dth, dw = gpu_ctx.combine_backward(torch.ones_like(theta), th, p, w)
    d = gpu_ctx.choice_backward(f["top_logp"], own, d_top=dw * w)
    torch.cuda.synchronize()
    assert f["top_choice"].tolist() == [[0, -1], [-1, -1], [0, 1]] and w.tolist() == [[1.0, 0.0], [0.0, 0.0], [0.5, 0.5]]
    assert (theta[1] == 0).all() and (theta[0] > 1).all() and torch.isfinite(d).all() and (d[1] == 0).all()


def test_nan_in_the_router_shows(gpu_ctx):
    """A row whose logits are NaN or +inf has theta NaN; the others are those of the router without them."""
    _, (W, b, Wr, br, n) = _setup(4, 10, 8)
    mix = Mixture(gpu_ctx, W, b, Wr, br)
    good = mix.forward(n).clone()
    n[3, 2], n[6] = float("nan"), float("inf")
    theta = mix.forward(n)
    mix.backward(torch.ones_like(theta))
    torch.cuda.synchronize()
    rest = [i for i in range(10) if i not in (3, 6)]
    # the router's product is the library's: its bits need not be the same, and a weight moves by 2 u |logit| at most
    assert torch.isnan(theta[[3, 6]]).all() and torch.allclose(theta[rest], good[rest], rtol=1e-5)
    assert torch.isnan(mix.dWr).any() and all(torch.isfinite(t).all() for t in mix.dW)


def test_gan_loop_with_a_mixture(gpu_ctx):
    """Runs, moves every parameter that has a gradient, and keeps them finite."""
    (_, _, _, _, _), (W, b, Wr, br, n) = _setup(4, 128, 7)
    ts = torch.tensor([[2.0, 5.0, 1.5, 3.0, 3.0, 2.0]], device="cuda:0")
    pool = gpu_ctx.sample_events(ts, 4000, 1)
    DW, Db = gen.xavier_mlp((2, 128, 128, 128, 128, 1), 2)
    t = lambda arrs: [torch.tensor(a, device="cuda:0") for a in arrs]      # noqa: E731
    loop = gan.GanLoop(gpu_ctx, W, b, t(DW), t(Db), pool, 128, 20, router=(Wr, br), top=2, entropy_coef=0.01)
    before = [p.clone() for p in loop.mixture.parameters()]
    for _ in range(3):
        loop.step(n)
    r = loop.residual(n, ts[0])
    torch.cuda.synchronize()
    after = loop.mixture.parameters()
    assert all(torch.isfinite(p).all() for p in after) and all(not torch.equal(p, q) for p, q in zip(before, after))
    assert torch.isfinite(r["r_hat"]).all()


def test_mixture_refuses(gpu_ctx):
    _, (W, b, Wr, br, n) = _setup(4, 10, 7)
    for bad in (dict(top=0), dict(top=5)):
        with pytest.raises(ValueError):
            Mixture(gpu_ctx, W, b, Wr, br, **bad)
    with pytest.raises(ValueError):
        Mixture(gpu_ctx, W, b, Wr[:3], br[:3])
