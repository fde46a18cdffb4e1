"""Advantages, policy loss and preference loss on the GPU against the float64
oracle: lengths from one event, odd sizes, masks that leave a row (or all) empty,
NaN and infinities in masked places, events at the interval's ends, refusals.

Tolerances, derived from the arithmetic.  A coordinate's log2(1 - x^a) is off by at
most 6e-7 (1 - x^a by 4e-7 of itself where x^a is near 3/4, a rounding of the log),
times b - 1 < 5 in each of two densities, so that a log ratio is off by at most 1e-5
in all and rho by 1e-5 of itself; a derivative's terms by less.  Sums are compared
against the sum of their terms' absolute values."""
import numpy as np
import pytest

import oracle
from tests.parity import to_np

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2407_00051_amd as sg  # noqa: E402

TOL = 1e-5
ADV_TOL = 1e-6      # of the row's largest: a subtraction in 64 bits, a rounding, an fp32 deviation and a product


def _t(a, **kw):
    return None if a is None else torch.tensor(a, device="cuda:0", **kw)


def _rows(rng, n, d, spread):
    old = rng.uniform(1.0, 5.0, (n, 2 * d)).astype(np.float32)
    return (old * np.exp(spread * rng.standard_normal(old.shape))).astype(np.float32), old


def _events(rng, rows, n):
    """n events of each row by the inverse CDF."""
    a, b = rows[:, None, 0::2].astype(np.float64), rows[:, None, 1::2].astype(np.float64)
    u = rng.random((rows.shape[0], n, rows.shape[1] // 2))
    return np.clip((-np.expm1(np.log1p(-u) / b)) ** (1.0 / a), 1e-30, 1.0).astype(np.float32)


def _mask(rng, kind, shape):
    if kind == "none":
        return None
    m = rng.random(shape) < 0.8
    if kind == "holes":
        m[::3] = False
    if kind == "empty":
        m[:] = False
    return m


# ---- advantages

@pytest.mark.parametrize("mask", ["none", "some", "holes", "empty"])
@pytest.mark.parametrize("rows,E", [(1, 1), (7, 1), (5, 3), (130, 33), (9, 64), (1024, 100), (3, 1024), (2, 1025), (5, 4099),
                                    (2, 16384), (3, 16385), (2, 70001)])
def test_group_advantage(gpu_ctx, rows, E, mask):
    print(f"case group_advantage rows={rows} E={E} mask={mask}", flush=True)
    rng = np.random.default_rng(rows * 7 + E)
    r = (rng.standard_normal((rows, E)) * 1.5 + 40.0 * rng.standard_normal((rows, 1))).astype(np.float32)
    m = _mask(rng, mask, r.shape)
    given = r.copy()
    if m is not None:
        given[~m] = rng.choice(np.array([np.nan, np.inf, -np.inf], np.float32), int((~m).sum()))
    for normalise in (True, False):
        got = to_np(gpu_ctx.group_advantage(_t(given), mask=_t(m), normalise=normalise, eps=1e-6)).astype(np.float64)
        ref = oracle.group_advantage(r, m, normalise, 1e-6)
        scale = np.abs(ref).max(1, keepdims=True)
        assert np.all(np.abs(got - ref) <= ADV_TOL * scale), np.abs(got - ref).max()
        if m is not None:
            assert np.all(got[~m] == 0.0)


@pytest.mark.parametrize("E", [1, 5, 100, 3000, 40000])
def test_group_advantage_of_equal_rewards_is_zero(gpu_ctx, E):
    r = torch.full((3, E), 0.1, device="cuda:0") * torch.tensor([[1.0], [3.3], [-777.7]], device="cuda:0")
    assert torch.count_nonzero(gpu_ctx.group_advantage(r)).item() == 0
    r2 = r.clone()
    assert gpu_ctx.group_advantage(r2, out=r2) is r2          # in place
    assert torch.count_nonzero(r2).item() == 0


# ---- policy loss

def _policy_case(rng, rows, E, d, mask, ref, spread=0.05):
    th, old = _rows(rng, rows, d, spread)
    c = dict(theta=th, theta_old=old, x=_events(rng, old, E), adv=rng.standard_normal((rows, E)).astype(np.float32),
             theta_ref=(old * 1.07).astype(np.float32) if ref else None, mask=_mask(rng, mask, (rows, E)))
    # within rounding of the clip's edges either side is right: such events get no advantage
    l = [oracle.event_logp(np.repeat(r, E, 0), c["x"].reshape(-1, d))[0] for r in (th, old)]
    rho = np.exp(l[0] - l[1]).reshape(rows, E)
    c["adv"][(np.abs(rho - 0.8) < 1e-4) | (np.abs(rho - 1.25) < 1e-4)] = 0.0
    return c


KW = dict(clip_low=0.2, clip_high=0.25, kl_coef=0.05)


def _check_policy(got, ref):
    for k in ("loss", "kl", "clip_frac"):
        assert abs(got[k].item() - ref[k]) <= TOL * max(1.0, abs(ref[k])), (k, got[k].item(), ref[k])
    err = np.abs(to_np(got["dtheta"]).astype(np.float64) - ref["dtheta"])
    assert np.all(err <= TOL * ref["abs_dtheta"]), (err / np.maximum(ref["abs_dtheta"], 1e-300)).max()


@pytest.mark.parametrize("average", ["events", "rows"])
@pytest.mark.parametrize("ref", [False, True])
@pytest.mark.parametrize("mask", ["none", "some", "holes", "empty"])
@pytest.mark.parametrize("rows,E,d", [(1, 1, 2), (67, 1, 3), (3, 2, 2), (33, 31, 3), (5, 64, 2), (4, 65, 3), (40, 100, 3),
                                      (1, 5001, 2), (3, 1999, 3)])
def test_policy_loss(gpu_ctx, rows, E, d, mask, ref, average):
    print(f"case policy rows={rows} E={E} d={d} mask={mask} ref={ref} {average}", flush=True)
    rng = np.random.default_rng(rows + 10 * E + d)
    c = _policy_case(rng, rows, E, d, mask, ref)
    want = oracle.policy_loss(**c, **KW, average=average)
    m = c["mask"]
    if m is not None:                                   # what is masked is not looked at
        c["adv"][~m] = np.nan
        c["x"][~m] = rng.choice(np.array([np.nan, np.inf, -1.0], np.float32), (int((~m).sum()), d))
    got = gpu_ctx.policy_loss(**{k: _t(v) for k, v in c.items()}, **KW, average=average)
    _check_policy(got, want)
    if mask == "empty":
        assert got["loss"].item() == 0.0 and torch.count_nonzero(got["dtheta"]).item() == 0


def test_policy_loss_many_rows_and_a_row_over_many_slices(gpu_ctx):
    for rows, E, d in ((5000, 17, 2), (2, 300001, 2)):
        print(f"case policy rows={rows} E={E}", flush=True)
        rng = np.random.default_rng(rows)
        c = _policy_case(rng, rows, E, d, "some", True)
        want = oracle.policy_loss(**c, **KW, average="rows")
        _check_policy(gpu_ctx.policy_loss(**{k: _t(v) for k, v in c.items()}, **KW, average="rows"), want)


def test_policy_gradient_against_differences(gpu_ctx):
    """dtheta against central differences of the GPU's own loss: steps of 2^-7 of a value move the
    loss by its slope with a relative error of the step's square times a third derivative of order 1."""
    rng = np.random.default_rng(3)
    rows, E, d = 2, 4000, 2
    c = _policy_case(rng, rows, E, d, "some", True, spread=0.02)
    kw = dict(clip_low=1.0, clip_high=50.0, kl_coef=0.5)        # nothing clipped: the loss is smooth
    t = {k: _t(v) for k, v in c.items()}
    g = to_np(gpu_ctx.policy_loss(**t, **kw)["dtheta"])
    for i in range(rows):
        for j in range(2 * d):
            h = float(c["theta"][i, j]) * 2.0 ** -7
            val = []
            for s in (1.0, -1.0):
                th = c["theta"].copy()
                th[i, j] += s * h
                val.append((gpu_ctx.policy_loss(**{**t, "theta": _t(th)}, **kw)["loss"].item(), float(th[i, j])))
            num = (val[0][0] - val[1][0]) / (val[0][1] - val[1][1])
            assert abs(num - g[i, j]) <= 1e-3 * np.abs(g).max() + 2e-5, (num, g[i, j])


def test_policy_events_at_the_ends(gpu_ctx):
    """Events rounded to 0 or 1 are read at the nearest number inside; a NaN event makes NaN."""
    rng = np.random.default_rng(4)
    c = _policy_case(rng, 2, 70, 2, "none", True, spread=0.001)
    c["x"][0, 3] = [0.0, 1.0]
    c["x"][1, 5] = [1.0, 0.5]
    c["adv"][0, 3] = c["adv"][1, 5] = 0.0
    want = oracle.policy_loss(**c, clip_low=1.0, clip_high=50.0, kl_coef=0.05)
    t = {k: _t(v) for k, v in c.items()}
    _check_policy(gpu_ctx.policy_loss(**t, clip_low=1.0, clip_high=50.0, kl_coef=0.05), want)
    t["x"][1, 6, 0] = float("nan")
    o = gpu_ctx.policy_loss(**t, **KW)
    assert torch.isnan(o["loss"]).item() and torch.isnan(o["dtheta"][1]).all().item()
    assert not torch.isnan(o["dtheta"][0]).any().item()


# ---- preference loss

def _pref_case(rng, rows, pairs, T, T2, d, ragged):
    th, ref = _rows(rng, rows, d, 0.05)
    P = rows * pairs
    c = dict(theta=th, theta_ref=ref, chosen=_events(rng, ref, pairs * T).reshape(P, T, d),
             rejected=_events(rng, ref, pairs * T2).reshape(P, T2, d), len_chosen=None, len_rejected=None)
    if ragged:
        c["len_chosen"] = rng.integers(-1, T + 2, P).astype(np.int32)
        c["len_rejected"] = rng.integers(0, T2 + 1, P).astype(np.int32)
    return c


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("rows,pairs,T,T2,d", [(1, 1, 1, 1, 2), (5, 3, 1, 1, 3), (1, 333, 1, 2, 2), (64, 5, 7, 3, 3),
                                              (2, 9, 64, 65, 2), (3, 4, 700, 650, 2), (1, 1, 5000, 4999, 3),
                                              (2, 3, 9001, 10, 2)])
def test_preference_loss(gpu_ctx, rows, pairs, T, T2, d, ragged):
    print(f"case preference rows={rows} pairs={pairs} T={T},{T2} d={d} ragged={ragged}", flush=True)
    rng = np.random.default_rng(rows * 1000 + pairs * 10 + T)
    c = _pref_case(rng, rows, pairs, T, T2, d, ragged)
    want = oracle.preference_loss(**c, beta=0.1, label_smoothing=0.05)
    if ragged:                                          # what lies past a set's length is not looked at
        for k in ("chosen", "rejected"):
            for p in range(rows * pairs):
                c[k][p, max(0, c["len_" + k][p]):] = np.nan
    got = gpu_ctx.preference_loss(**{k: _t(v) for k, v in c.items()}, beta=0.1, label_smoothing=0.05)
    err = np.abs(to_np(got["margin"]) - want["margin"])
    assert np.all(err <= 0.1 * TOL * (T + T2)), err.max()
    assert abs(got["loss"].item() - want["loss"]) <= 0.1 * TOL * (T + T2) + 1e-6 * want["loss"]
    # the slope of a pair is off by at most the margin's error times its own size
    tol = (TOL + 0.1 * TOL * (T + T2)) * want["abs_dtheta"]
    assert np.all(np.abs(to_np(got["dtheta"]) - want["dtheta"]) <= tol)


def test_preference_of_far_margins(gpu_ctx):
    """Margins of either sign far from 0: the loss tends to |h| or to 0, nothing overflows."""
    rng = np.random.default_rng(11)
    c = _pref_case(rng, 2, 8, 40, 40, 2, False)
    c["theta"] = (c["theta_ref"] * 3.0).astype(np.float32)
    want = oracle.preference_loss(**c, beta=20.0)
    assert want["margin"].max() > 100 and want["margin"].min() < -100
    got = gpu_ctx.preference_loss(**{k: _t(v) for k, v in c.items()}, beta=20.0)
    assert np.isfinite(to_np(got["dtheta"])).all()
    assert np.all(np.abs(to_np(got["margin"]) - want["margin"]) <= 20.0 * 3 * TOL * 80)
    assert abs(got["loss"].item() - want["loss"]) <= 20.0 * 3 * TOL * 80


def test_optional_outputs_streams_and_repeats(gpu_ctx):
    """No gradient asked for; the same bits again; on a stream of its own."""
    rng = np.random.default_rng(12)
    c = {k: _t(v) for k, v in _policy_case(rng, 50, 70, 3, "some", True).items()}
    p = {k: _t(v) for k, v in _pref_case(rng, 50, 3, 9, 9, 3, True).items()}
    a, b = gpu_ctx.policy_loss(**c, **KW), gpu_ctx.preference_loss(**p)
    assert gpu_ctx.policy_loss(**c, **KW, want_grad=False)["dtheta"] is None
    assert torch.equal(gpu_ctx.policy_loss(**c, **KW, want_grad=False)["loss"], a["loss"])
    assert torch.equal(gpu_ctx.preference_loss(**p, want_grad=False)["margin"], b["margin"])
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    ctx = sg.Context(0, stream=st)
    a2, b2 = ctx.policy_loss(**c, **KW), ctx.preference_loss(**p)
    adv = ctx.group_advantage(c["adv"], mask=c["mask"])
    st.synchronize()
    ctx.close()
    for k in ("loss", "kl", "clip_frac", "dtheta"):
        assert torch.equal(a[k], a2[k]), k
    for k in ("loss", "margin", "dtheta"):
        assert torch.equal(b[k], b2[k]), k
    assert torch.equal(adv, gpu_ctx.group_advantage(c["adv"], mask=c["mask"]))


def test_refusals(gpu_ctx):
    rng = np.random.default_rng(13)
    c = {k: _t(v) for k, v in _policy_case(rng, 4, 10, 2, "some", True).items()}
    p = {k: _t(v) for k, v in _pref_case(rng, 4, 2, 5, 5, 2, True).items()}

    def bad(err, f, base, **kw):
        with pytest.raises(err):
            f(**{**base, **kw})

    for kw in (dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_high=float("nan")), dict(kl_coef=-1.0),
               dict(kl_coef=float("inf"))):
        bad(sg.SagipsError, gpu_ctx.policy_loss, c, **kw)
    bad(ValueError, gpu_ctx.policy_loss, c, average="all")
    bad(ValueError, gpu_ctx.policy_loss, c, theta_old=c["theta_old"][:3])
    bad(ValueError, gpu_ctx.policy_loss, c, x=c["x"][:, :9])
    bad(ValueError, gpu_ctx.policy_loss, c, x=c["x"].transpose(0, 1))
    bad(ValueError, gpu_ctx.policy_loss, c, adv=c["adv"].t())
    bad(TypeError, gpu_ctx.policy_loss, c, mask=c["mask"].float())
    bad(TypeError, gpu_ctx.policy_loss, c, x=c["x"].double())
    bad(ValueError, gpu_ctx.policy_loss, c, x=c["x"].cpu())
    bad(sg.SagipsError, gpu_ctx.policy_loss, c, x=torch.zeros(1 + c["x"].numel(), device="cuda:0")[1:].view_as(c["x"]))
    bad(sg.SagipsError, gpu_ctx.policy_loss, c, adv=c["adv"][:, :0].contiguous(), x=c["x"][:, :0].contiguous(), mask=None)
    for kw in (dict(beta=0.0), dict(beta=float("nan")), dict(label_smoothing=1.5), dict(label_smoothing=-0.5)):
        bad(sg.SagipsError, gpu_ctx.preference_loss, p, **kw)
    bad(ValueError, gpu_ctx.preference_loss, p, rejected=p["rejected"][:7].contiguous())
    bad(ValueError, gpu_ctx.preference_loss, p, theta=c["theta"][:3].contiguous(), theta_ref=c["theta"][:3].contiguous())
    bad(TypeError, gpu_ctx.preference_loss, p, len_chosen=p["len_chosen"].long())
    r = torch.zeros((4, 8), device="cuda:0")
    bad(sg.SagipsError, gpu_ctx.group_advantage, dict(reward=r), eps=-1.0)
    bad(ValueError, gpu_ctx.group_advantage, dict(reward=r), mask=torch.ones((4, 7), dtype=torch.bool, device="cuda:0"))
    bad(ValueError, gpu_ctx.group_advantage, dict(reward=r[0]))
    buf = torch.zeros(64, device="cuda:0")
    bad(sg.SagipsError, gpu_ctx.group_advantage, dict(reward=buf[:32].view(4, 8)), out=buf[16:48].view(4, 8))
    assert gpu_ctx.lib.sagips_group_advantage(None, None, None, 1, 1, 1, 0.0, None) == sg.E_INVAL
