"""The loop that trains from scores alone (paper_2407_00051_amd/score.py): each part of
one step against the float64 oracle applied to the tensors that the loop holds, the
refusals, and a run in which the observables approach the reference data's."""
import numpy as np
import pytest

import oracle
from tests.parity import assert_normwise, to_np
from workloads import gen

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2407_00051_amd.score import ScoreLoop, score_closure  # noqa: E402

GW_, DW_ = (6, 128, 128, 128, 128, 6), (2, 128, 128, 128, 128, 1)
TS = np.array([[2.0, 5.0, 1.5, 3.0, 3.0, 2.0]], dtype=np.float32)
TOL = 1e-4       # the library's fp32 bound


def _loop(ctx, k, E, **kw):
    GW, Gb = gen.generator_stack(GW_, 1, 21)
    DW, Db = gen.xavier_mlp(DW_, 2)
    d = lambda xs: [torch.tensor(x, device="cuda:0") for x in xs]     # noqa: E731
    pool = ctx.sample_events(torch.tensor(TS, device="cuda:0"), 2 * k * E, 1)
    return ScoreLoop(ctx, d(w[0] for w in GW), d(v[0] for v in Gb), d(DW), d(Db), pool, k, E, **kw)


def _np64(ts):
    return [to_np(t).astype(np.float64) for t in ts]


def _accept(x):
    return x[:, :, 0] > 0.2


@pytest.mark.parametrize("objective,cuts", [("policy", False), ("policy", True), ("preference", False)])
def test_step_against_the_oracle(gpu_ctx, objective, cuts):
    print(f"case score step {objective} cuts={cuts}", flush=True)
    k, E = 48, 60
    loop = _loop(gpu_ctx, k, E, objective=objective, epochs=2, set_size=7, accept=_accept if cuts else None)
    noise = torch.tensor(np.random.default_rng(3).standard_normal((k, 6)).astype(np.float32), device="cuda:0")
    held = {key: [t.clone() for t in getattr(loop, key)] for key in ("G_W", "G_b", "D_W", "D_b")}
    # one epoch at a time, to see the state between them
    loop.epochs = 1
    loop.step(noise)
    torch.cuda.synchronize()
    old = to_np(loop.theta_old[0]).astype(np.float64)
    assert_normwise(old, oracle.generator_forward(_np64(held["G_W"]), _np64(held["G_b"]), to_np(noise).astype(np.float64)), TOL, "theta")
    x = to_np(loop.x).astype(np.float64)
    assert_normwise(x, oracle.sample(to_np(loop.theta_old[0]), E, 0), TOL, "events")
    logits = oracle.mlp_forward(_np64(held["D_W"]), _np64(held["D_b"]), oracle.features_proxy2(x))
    logits = np.asarray(logits[0] if isinstance(logits, tuple) else logits).reshape(-1)
    assert_normwise(to_np(loop.outs["logits_fake"]), logits, TOL, "logits")
    scores = to_np(loop.outs["logits_fake"]).reshape(k, E).astype(np.float64)
    x3 = x.reshape(k, E, 3)
    if objective == "policy":
        mask = x3[:, :, 0].astype(np.float32) > np.float32(0.2) if cuts else None
        adv = oracle.group_advantage(scores, mask)
        want = oracle.policy_loss(old, old, x3, adv, theta_ref=old, mask=mask, kl_coef=0.05, average="rows")
        # theta is theta_old: every ratio is one, the gradient that of the mean of -A l
        assert abs(loop.last["loss"].item() - want["loss"]) <= 1e-5 and loop.last["kl"].item() <= 1e-10
    else:
        S = E // 7
        order = np.argsort(-scores[:, :S * 7].reshape(k, S, 7).mean(2), axis=1)
        sets = x3[:, :S * 7].reshape(k, S, 7, 3)
        pick = lambda o: np.stack([sets[i, o[i]] for i in range(k)]).reshape(-1, 7, 3)     # noqa: E731
        want = oracle.preference_loss(old, old, pick(order[:, :S // 2]), pick(order[:, ::-1][:, :S // 2]), beta=0.1)
        assert abs(loop.last["loss"].item() - np.log(2.0)) <= 1e-6
    err = np.abs(to_np(loop.last["dtheta"]) - want["dtheta"])
    assert np.all(err <= TOL * want["abs_dtheta"])
    gW, gb = oracle.generator_backward(_np64(held["G_W"]), _np64(held["G_b"]), to_np(noise).astype(np.float64),
                                       to_np(loop.last["dtheta"]).astype(np.float64))
    # hidden matrices move along the orthogonalised gradient, the rest as Adam's first step does
    for name, nets, grads, lr_m, lr_a in (("G", held["G_W"], loop.gW, 1e-4, 1e-5), ("D", held["D_W"], loop.outs["dW"], 5e-3, 1e-4)):
        now = loop.G_W if name == "G" else loop.D_W
        for l in range(1, 4):
            g = to_np(grads[l]).astype(np.float64)
            p, _ = oracle.muon_step(to_np(nets[l]), g, np.zeros_like(g), lr_m)
            assert_normwise(to_np(now[l]) - to_np(nets[l]), p - to_np(nets[l]), 1e-3, f"{name} W[{l}] moved")
        for l in (0, 4):
            g = to_np(grads[l]).astype(np.float64)
            p, _, _ = oracle.adam_step(to_np(nets[l]), g, np.zeros_like(g), np.zeros_like(g), 1, lr_a)
            assert np.abs(to_np(now[l]) - p).max() <= 1e-2 * lr_a
    assert_normwise(to_np(loop.gW[4]), gW[4], 1e-3, "dW_G[4]")


def test_second_epoch_sees_the_moved_rows(gpu_ctx):
    """With two epochs theta has left theta_old when the last loss is formed."""
    k, E = 40, 80
    loop = _loop(gpu_ctx, k, E, epochs=2, lr_muon_g=5e-3)
    loop.step(torch.tensor(np.random.default_rng(4).standard_normal((k, 6)).astype(np.float32), device="cuda:0"))
    old, th = to_np(loop.theta_old[0]).astype(np.float64), to_np(loop.theta[0]).astype(np.float64)
    x = to_np(loop.x).reshape(k, E, 3)
    adv = oracle.group_advantage(to_np(loop.outs["logits_fake"]).reshape(k, E))
    want = oracle.policy_loss(th, old, x, adv, theta_ref=old, kl_coef=0.05, average="rows")
    assert np.abs(th - old).max() > 1e-3 and want["kl"] > 0.0
    assert abs(loop.last["loss"].item() - want["loss"]) <= 1e-4
    assert abs(loop.last["kl"].item() - want["kl"]) <= 1e-3 * want["kl"] + 1e-7


@pytest.mark.parametrize("objective", ["policy", "preference"])
def test_observables_approach_the_reference(gpu_ctx, objective):
    """After 500 steps at the default rates the distribution of the two observables (quantiles along
    eight directions) is at less than half of its first distance from the reference data's."""
    obs = lambda t: torch.stack([t[:, 0] + t[:, 2], t[:, 1] + t[:, 2]], 1)      # noqa: E731
    q = torch.linspace(0.02, 0.98, 49, device="cuda:0")

    def distance(a, b):
        d = []
        for phi in np.linspace(0.0, np.pi, 8, endpoint=False):
            v = torch.tensor([np.cos(phi), np.sin(phi)], dtype=torch.float32, device="cuda:0")
            d.append((torch.quantile(a @ v, q) - torch.quantile(b @ v, q)).abs().mean().item())
        return float(np.mean(d))

    far = []
    k, E = 256, 50
    loop = _loop(gpu_ctx, k, E, objective=objective)
    rng = np.random.default_rng(5)
    for s in range(500):
        loop.step(torch.tensor(rng.standard_normal((k, 6)).astype(np.float32), device="cuda:0"))
        if s in (0, 499):
            far.append(distance(obs(loop.x), obs(loop.pool)))
    print(f"  {objective}: distance of the observables {far[0]:.4f} -> {far[1]:.4f}", flush=True)
    assert far[1] < 0.5 * far[0]


def test_closure_runs_and_refusals(gpu_ctx):
    hist = score_closure(gpu_ctx, steps=4, report_every=2, k=32, events_per_theta=40)
    assert [h["step"] for h in hist] == [2, 4] and all(np.isfinite(h["loss"]) for h in hist)
    for kw in (dict(objective="else"), dict(objective="preference", set_size=31), dict(objective="preference", accept=_accept),
               dict(objective="preference", set_size=0)):
        with pytest.raises(ValueError):
            _loop(gpu_ctx, 8, 60, **kw)
