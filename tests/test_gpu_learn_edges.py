"""Ends of the ranges that the losses accept, against the float64 oracle.

Tolerances are those of test_gpu_learn, whose derivation holds here too unless a test says otherwise."""
import numpy as np
import pytest

import oracle
from tests.parity import to_np
from tests.test_gpu_learn import ADV_TOL, KW, TOL, _check_policy, _events, _mask, _policy_case, _pref_case, _t

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2407_00051_amd as sg  # noqa: E402


# ---- advantages

@pytest.mark.parametrize("eps", [0.0, 1e-60])
@pytest.mark.parametrize("rows,E", [(4, 1), (6, 5), (5, 300), (3, 1500), (3, 20000), (3000, 200)])
def test_group_advantage_without_eps(gpu_ctx, rows, E, eps):
    """Rows of equal rewards, rows with one valid event and rows of rewards among the smallest numbers."""
    print(f"case advantage rows={rows} E={E} eps={eps}", flush=True)
    rng = np.random.default_rng(E)
    r = rng.standard_normal((rows, E)).astype(np.float32)
    r[0] = -3.3
    m = np.ones((rows, E), bool)
    m[1] = False
    m[1, E // 2] = True
    r[2] = (r[2] * 1e-42).astype(np.float32)
    if rows > 4:
        m[4] = False
    given = np.where(m, r, np.float32(np.nan))
    got = to_np(gpu_ctx.group_advantage(_t(given), mask=_t(m), eps=eps)).astype(np.float64)
    assert np.all(got[0] == 0.0) and np.all(got[1] == 0.0) and np.all(got[~m] == 0.0)
    if E == 1:
        assert np.all(got == 0.0)
        return
    some = [i for i in range(rows) if i > 1 and m[i].any()]
    ref = oracle.group_advantage(r[some], m[some], True, eps)
    assert np.all(np.abs(got[some] - ref) <= ADV_TOL * np.abs(ref).max(1, keepdims=True))


# ---- rows far apart

def _difference_terms(theta, ref, x):
    """Of the log ratio of events x [n][d]: the sum of the absolute values of its terms, and of the
    factors of its logarithms ln(1 - x^a)."""
    a, b, a2, b2 = (np.float64(v) for v in (theta[0::2], theta[1::2], ref[0::2], ref[1::2]))
    lx = np.log(np.clip(np.float64(x), oracle.learn.X_LO, oracle.learn.X_HI))
    g, g2 = np.log(-np.expm1(a * lx)), np.log(-np.expm1(a2 * lx))
    terms = (np.abs(np.log(a / a2)) + np.abs(np.log(b / b2)) + np.abs((a - a2) * lx) + np.abs(b - 1.0) * (np.abs(g) + np.abs(g2))
             + np.abs((b - b2) * g2))
    return terms.sum(1), np.sum(np.abs(b - 1.0) * 2.0 + np.abs(b - b2)) * np.ones(len(x))


@pytest.mark.parametrize("factor", [1e-2, 1e-3, 1e-6, 1e-9, 1e3])
@pytest.mark.parametrize("d", [2, 3])
def test_log_ratio_of_rows_far_apart(gpu_ctx, d, factor):
    """Sets of unequal size, so that the rows' own logarithms stay in the margin.  Tolerance: of an
    event's terms 8 units in the last place of fp32 (a logarithm, its factor, six sums), and 6e-7 for
    each ln(1 - x^a) times its factor."""
    print(f"case far rows d={d} factor={factor}", flush=True)
    rng = np.random.default_rng(int(1e4 * d) + int(-np.log10(factor)) + 20)
    rows, T, T2 = 9, 5, 2
    ref = rng.uniform(1.0, 5.0, (rows, 2 * d)).astype(np.float32)
    theta = ref.copy()
    which = rng.integers(0, 2 * d, rows)
    theta[np.arange(rows), which] *= np.float32(factor)
    theta[0] = ref[0] * np.float32(factor)
    c = dict(theta=theta, theta_ref=ref, chosen=_events(rng, ref, T), rejected=_events(rng, ref, T2))
    beta = 0.01
    want = oracle.preference_loss(**c, len_chosen=None, len_rejected=None, beta=beta)
    got = gpu_ctx.preference_loss(**{k: _t(v) for k, v in c.items()}, beta=beta)
    tol = np.zeros(rows)
    for i in range(rows):
        for k in ("chosen", "rejected"):
            terms, logs = _difference_terms(theta[i], ref[i], c[k][i])
            tol[i] += beta * np.sum(8 * 2.0 ** -24 * terms + 6e-7 * logs)
    err = np.abs(to_np(got["margin"]).astype(np.float64) - want["margin"])
    print(f"  worst of error / tolerance {np.max(err / tol):.3f}", flush=True)
    assert np.all(err <= tol), (err / tol)
    assert abs(got["loss"].item() - want["loss"]) <= tol.mean() + 1e-6 * want["loss"]
    assert np.all(np.abs(to_np(got["dtheta"]) - want["dtheta"]) <= (TOL + tol[:, None]) * want["abs_dtheta"])


# ---- ratios beyond fp32

def _far_event(rng, E):
    """Rows (a = 1 and 2.2) between which the first event, near 0, has e^103 to one of density."""
    near, far = np.array([[1.0, 2.0, 1.5, 2.0]], np.float32), np.array([[2.2, 2.0, 1.5, 2.0]], np.float32)
    x = _events(rng, far, E)
    x[0, 0, 0] = 2e-38
    return near, far, x


@pytest.mark.parametrize("zero", [0.0, -0.0])
def test_event_without_advantage_beyond_the_ratios_range(gpu_ctx, zero):
    """rho A of A = 0 is 0 however large the ratio; a NaN event stays NaN."""
    rng = np.random.default_rng(21)
    near, far, x = _far_event(rng, 50)
    adv = rng.standard_normal((1, 50)).astype(np.float32)
    adv[0, 0] = zero
    c = dict(theta=near, theta_old=far, x=x, adv=adv)
    want = oracle.policy_loss(**c, clip_low=1.0, clip_high=50.0)
    t = {k: _t(v) for k, v in c.items()}
    _check_policy(gpu_ctx.policy_loss(**t, clip_low=1.0, clip_high=50.0), want)
    t["x"][0, 0, 0] = float("nan")
    o = gpu_ctx.policy_loss(**t, clip_low=1.0, clip_high=50.0)
    assert torch.isnan(o["loss"]).item() and torch.isnan(o["dtheta"][0, :2]).all().item()


def test_no_weight_on_a_divergence_beyond_fp32(gpu_ctx):
    """kl_coef = 0 leaves the loss and its gradient to the ratios, whatever the divergence that is reported."""
    rng = np.random.default_rng(22)
    near, far, x = _far_event(rng, 50)
    c = dict(theta=far, theta_old=far, theta_ref=near, x=x, adv=rng.standard_normal((1, 50)).astype(np.float32))
    want = oracle.policy_loss(**c, kl_coef=0.0)
    got = gpu_ctx.policy_loss(**{k: _t(v) for k, v in c.items()}, kl_coef=0.0)
    assert abs(got["loss"].item() - want["loss"]) <= TOL * max(1.0, abs(want["loss"]))
    assert np.all(np.abs(to_np(got["dtheta"]) - want["dtheta"]) <= TOL * want["abs_dtheta"])
    assert got["kl"].item() == np.inf and want["kl"] > 1e40


# ---- contexts and graphs

def _both(ctx, c, p):
    a, b = ctx.policy_loss(**c, **KW, average="rows"), ctx.preference_loss(**p)
    return [a["loss"], a["kl"], a["clip_frac"], a["dtheta"], b["loss"], b["margin"], b["dtheta"]]


def test_first_losses_of_a_context_in_a_graph(gpu_ctx):
    """A context whose first losses are captured: eager calls before the first replay, replays and eager
    calls between them all give the same bits."""
    print("case first call captured", flush=True)
    rng = np.random.default_rng(30)
    c = {k: _t(v) for k, v in _policy_case(rng, 50, 70, 3, "some", True).items()}
    p = {k: _t(v) for k, v in _pref_case(rng, 50, 3, 9, 9, 3, True).items()}
    want = _both(gpu_ctx, c, p)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        ctx = sg.Context(0, stream=st)
        ctx.group_advantage(torch.zeros((1, 20000), device="cuda:0"))      # makes the workspace, outside the capture
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st, capture_error_mode="relaxed"):
            out = _both(ctx, c, p)
        for _ in range(3):
            eager = _both(ctx, c, p)
            graph.replay()
            st.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(eager, want))
            assert all(torch.equal(a, b) for a, b in zip(out, want))
        ctx.close()


def test_more_contexts_than_counters(gpu_ctx):
    """Contexts beyond the 64 that have counters end in a second launch, with the same bits."""
    print("case 70 contexts", flush=True)
    rng = np.random.default_rng(31)
    c = {k: _t(v) for k, v in _policy_case(rng, 50, 70, 3, "some", True).items()}
    p = {k: _t(v) for k, v in _pref_case(rng, 50, 3, 9, 9, 3, True).items()}
    want = _both(gpu_ctx, c, p)
    for _ in range(2):
        many = [sg.Context(0) for _ in range(70)]
        for ctx in many:
            assert all(torch.equal(a, b) for a, b in zip(_both(ctx, c, p), want))
        for ctx in many:
            ctx.close()


# ---- every way in which sums are joined

def _launches(ctx, call):
    """The call's result and the names of the kernels that it launched."""
    ctx.set_timing(True)
    ctx.kernel_times()
    out = call()
    names = set(ctx.kernel_times())
    ctx.set_timing(False)
    return out, names


def _sum_of_terms(c, kl_coef, average):
    """As the oracle's abs_dtheta, but with the slope dL/dl = -rho A [not clipped] - kl_coef (e^r - 1) by
    its terms too: over thousands of short rows it comes near 0 in some row, and there its own
    rounding, 1e-5 of rho A and of e^r, is what is left."""
    x, m = c["x"].astype(np.float64), np.ones(c["adv"].shape, bool) if c["mask"] is None else c["mask"]
    rows, E, d = x.shape
    each = lambda t: oracle.event_logp(np.repeat(t, E, 0), x.reshape(-1, d))     # noqa: E731
    l, _, terms = each(c["theta"])
    rho, r = np.exp(l - each(c["theta_old"])[0]), each(c["theta_ref"])[0] - l
    A = np.where(m, c["adv"], 0.0).reshape(-1).astype(np.float64)
    cut = np.clip(rho, 1.0 - KW["clip_low"], 1.0 + KW["clip_high"]) * A < rho * A
    n = m.sum(1)
    w = np.where(m, 1.0 / n.sum() if average == "events" else (1.0 / np.maximum(n, 1) / (n > 0).sum())[:, None], 0.0).reshape(-1)
    size = w * (np.where(cut, 0.0, np.abs(rho * A)) + kl_coef * (np.exp(r) + 1.0))
    return (size[:, None] * terms).reshape(rows, E, -1).sum(1)


@pytest.mark.parametrize("average", ["events", "rows"])
@pytest.mark.parametrize("mask", ["none", "holes"])
@pytest.mark.parametrize("rows,E,two", [(60, 257, False), (60, 600, False), (60, 1000, False),         # 2, 3, 4 slices a row
                                        (1400, 257, True), (1400, 600, True), (1400, 1000, True),
                                        (9000, 17, True), (1300, 90, True), (1370, 3, True)])
def test_policy_joins(gpu_ctx, rows, E, two, mask, average):
    print(f"case policy join {rows} x {E} mask={mask} {average}", flush=True)
    rng = np.random.default_rng(rows + E)
    c = _policy_case(rng, rows, E, 3, mask, True)
    want = oracle.policy_loss(**c, **KW, average=average)
    want["abs_dtheta"] = _sum_of_terms(c, KW["kl_coef"], average)
    if c["mask"] is not None:
        c["adv"][~c["mask"]] = np.nan
    got, names = _launches(gpu_ctx, lambda: gpu_ctx.policy_loss(**{k: _t(v) for k, v in c.items()}, **KW, average=average))
    assert ("policy_finish" in names) == two, names
    _check_policy(got, want)


@pytest.mark.parametrize("rows,pairs,T,d,two", [(40, 64, 70, 2, True), (40, 64, 70, 3, True), (3000, 1, 5, 3, True), (3000, 1, 5, 2, True),
                                                (1400, 7, 9, 3, True), (1, 6000, 3, 2, False), (1, 1200, 90, 3, True),
                                                (2, 3, 4096, 2, False)])
def test_preference_joins(gpu_ctx, rows, pairs, T, d, two):
    print(f"case preference join {rows} x {pairs} x {T} d={d}", flush=True)
    rng = np.random.default_rng(rows + pairs)
    c = _pref_case(rng, rows, pairs, T, T, d, True)
    want = oracle.preference_loss(**c, beta=0.1, label_smoothing=0.05)
    got, names = _launches(gpu_ctx, lambda: gpu_ctx.preference_loss(**{k: _t(v) for k, v in c.items()}, beta=0.1, label_smoothing=0.05))
    assert ("preference_finish" in names) == two, names
    assert np.all(np.abs(to_np(got["margin"]) - want["margin"]) <= 0.1 * TOL * 2 * T)
    assert abs(got["loss"].item() - want["loss"]) <= 0.1 * TOL * 2 * T + 1e-6 * want["loss"]
    assert np.all(np.abs(to_np(got["dtheta"]) - want["dtheta"]) <= (TOL + 0.1 * TOL * 2 * T) * want["abs_dtheta"])


@pytest.mark.parametrize("mask", ["none", "holes"])
@pytest.mark.parametrize("rows,E", [(40000, 17), (3000, 200), (600, 1000), (9000, 60)])
def test_advantages_of_many_rows(gpu_ctx, rows, E, mask):
    print(f"case advantage {rows} x {E} mask={mask}", flush=True)
    rng = np.random.default_rng(rows)
    r = (rng.standard_normal((rows, E)) + 10.0 * rng.standard_normal((rows, 1))).astype(np.float32)
    m = _mask(rng, mask, r.shape)
    ref = oracle.group_advantage(r, m, True, 1e-6)
    got = to_np(gpu_ctx.group_advantage(_t(r if m is None else np.where(m, r, np.float32(np.inf))), mask=_t(m))).astype(np.float64)
    assert np.all(np.abs(got - ref) <= ADV_TOL * np.abs(ref).max(1, keepdims=True))
