"""Training the generator against a pipeline that only scores its events, on one
GPU, sequenced from the library's calls (no host synchronisation).

The GAN loop (gan.py) needs every module between the parameters and the
discriminator's response to be differentiable.  Here nothing behind the sampler
is: the discriminator's logits of the events, after any cuts, are rewards, and
the generator learns from the density with which its parameters produce the
events.  Step t (counting from 1):
  1. theta_old = 1 + softplus(G(noise_t))                       sagips_gen_forward
  2. events x at theta_old (counter base (t-1) N)               sagips_sample_events
  3. reference batch = bootstrap step t of the data pool        sagips_bootstrap
  4. discriminator, BCE, dL_D/dW_D; the logits of x             sagips_disc_fwd_bwd
  5. `epochs` times: theta = 1 + softplus(G(noise_t)),          sagips_gen_forward
     dL/dtheta by one of
       policy      advantages of the logits within each row     sagips_group_advantage
                   and the clipped policy loss, its KL term
                   against theta_old                            sagips_policy_loss
       preference  each row's sets of events ranked by their
                   mean logit, the better half against the
                   worse                                        sagips_preference_loss
     dL/dW_G                                                    sagips_gen_backward
     hidden matrices by their orthogonalised momentum, the
     other parameters by Adam                                   sagips_muon_step, sagips_adam_step
  6. the discriminator likewise, from the gradients of 4.
"""
from __future__ import annotations

from typing import Callable, List, Optional, Sequence

from . import FEAT_PROXY2, Context


class Split:
    """The parameters of one network: matrices between hidden layers, which take
    orthogonalised updates, and the rest, which Adam moves."""

    def __init__(self, Ws: Sequence, bs: Sequence, dWs: Sequence, dbs: Sequence):
        import torch
        hidden = range(1, len(Ws) - 1)
        self.mat, self.d_mat = [Ws[l] for l in hidden], [dWs[l] for l in hidden]
        self.rest, self.d_rest = [Ws[0], Ws[-1], *bs], [dWs[0], dWs[-1], *dbs]
        self.momenta = [torch.zeros_like(w) for w in self.mat]
        self.m = [torch.zeros_like(p) for p in self.rest]
        self.v = [torch.zeros_like(p) for p in self.rest]
        self.t = 0

    def step(self, ctx: Context, lr_muon: float, lr_adam: float) -> None:
        self.t += 1
        if self.mat:
            ctx.muon_step(self.mat, self.d_mat, self.momenta, lr_muon)
        ctx.adam_step(self.rest, self.d_rest, self.m, self.v, self.t, lr_adam)


class ScoreLoop:
    """Generator and discriminator (parameters updated in place) and the reference
    data pool, all device tensors owned by the caller.  `accept(x)` may return a
    bool mask [k][E] of the events [k][E][3] that pass the cuts."""

    def __init__(self, ctx: Context, G_W: Sequence, G_b: Sequence, D_W: Sequence, D_b: Sequence, pool, k: int,
                 events_per_theta: int, objective: str = "policy", epochs: int = 2, set_size: int = 10,
                 accept: Optional[Callable] = None, fake_seed: int = 0, boot_seed: int = 5, lr_g: float = 1e-5,
                 lr_d: float = 1e-4, lr_muon_g: float = 1e-4, lr_muon_d: float = 5e-3, slope: float = 0.2,
                 features: int = FEAT_PROXY2, clip: float = 0.2, kl_coef: float = 0.05, beta: float = 0.1):
        import torch
        if objective not in ("policy", "preference"):
            raise ValueError("objective must be 'policy' or 'preference'")
        if objective == "preference" and (accept is not None or events_per_theta < 2 * set_size or set_size < 1):
            raise ValueError("preferences need two sets of events a row and take no cuts")
        self.ctx = ctx
        self.G_W, self.G_b, self.D_W, self.D_b = list(G_W), list(G_b), list(D_W), list(D_b)
        self.pool, self.objective, self.epochs, self.T, self.accept = pool, objective, epochs, set_size, accept
        self.k, self.E = int(k), int(events_per_theta)
        self.N = self.k * self.E
        self.fake_seed, self.boot_seed, self.slope, self.features = fake_seed, boot_seed, slope, features
        self.lr_g, self.lr_d, self.lr_muon_g, self.lr_muon_d = lr_g, lr_d, lr_muon_g, lr_muon_d
        self.clip, self.kl_coef, self.beta = clip, kl_coef, beta
        self.t = 0
        n_out = self.G_W[-1].shape[0]
        f32 = dict(dtype=torch.float32, device=pool.device)
        self.theta_old = torch.empty((1, self.k, n_out), **f32)
        self.theta = torch.empty((1, self.k, n_out), **f32)
        self.x = torch.empty((self.N, n_out // 2), **f32)
        self.real = torch.empty((self.N, pool.shape[1]), **f32)
        self.outs = {"loss_d": torch.empty(1, **f32), "loss_g": torch.empty(1, **f32),
                     "logits_fake": torch.empty(self.N, **f32), "logits_real": torch.empty(self.N, **f32),
                     "dW": [torch.empty_like(w) for w in self.D_W], "db": [torch.empty_like(v) for v in self.D_b]}
        self.gW, self.gb = [torch.empty_like(w) for w in self.G_W], [torch.empty_like(v) for v in self.G_b]
        self.D = Split(self.D_W, self.D_b, self.outs["dW"], self.outs["db"])
        self.G = Split(self.G_W, self.G_b, self.gW, self.gb)
        self.last: dict = {}

    def _pairs(self, x, scores):
        """Sets of a row ranked by their mean score, best against worst, second best against second
        worst, ...: chosen and rejected [k * pairs][T][3]."""
        S, T, d = self.E // self.T, self.T, x.shape[2]
        mean = scores[:, :S * T].reshape(self.k, S, T).mean(2)
        order = mean.argsort(dim=1, descending=True)
        sets = x[:, :S * T].reshape(self.k, S, T * d)
        half = S // 2
        best, worst = order[:, :half], order.flip(1)[:, :half]
        take = lambda i: sets.gather(1, i[:, :, None].expand(-1, -1, T * d)).reshape(self.k * half, T, d)   # noqa: E731
        return take(best), take(worst)

    def step(self, noise) -> None:
        """One training step on the noise batch [k][in] (a device tensor)."""
        self.t += 1
        c = self.ctx
        c.gen_forward(self.G_W, self.G_b, noise, slope=self.slope, out=self.theta_old)
        old = self.theta_old[0]
        c.sample_events(old, self.E, self.fake_seed, counter_base=(self.t - 1) * self.N, out=self.x)
        c.bootstrap(self.pool, self.N, self.boot_seed, self.t, out=self.real)
        c.disc_fwd_bwd(self.D_W, self.D_b, self.real, fake_x=self.x, features=self.features, slope=self.slope,
                       want_dx=False, outputs=self.outs)
        x, scores = self.x.view(self.k, self.E, -1), self.outs["logits_fake"].view(self.k, self.E)
        if self.objective == "policy":
            mask = self.accept(x) if self.accept is not None else None
            adv = c.group_advantage(scores, mask=mask)
        else:
            chosen, rejected = self._pairs(x, scores)
        for _ in range(self.epochs):
            c.gen_forward(self.G_W, self.G_b, noise, slope=self.slope, out=self.theta)
            if self.objective == "policy":
                self.last = c.policy_loss(self.theta[0], old, x, adv, theta_ref=old, mask=mask, clip_low=self.clip,
                                          clip_high=self.clip, kl_coef=self.kl_coef, average="rows")
            else:
                self.last = c.preference_loss(self.theta[0], old, chosen, rejected, beta=self.beta)
            c.gen_backward(self.G_W, self.G_b, noise, self.last["dtheta"], slope=self.slope, dW=self.gW, db=self.gb)
            self.G.step(c, self.lr_muon_g, self.lr_g)
        self.D.step(c, self.lr_muon_d, self.lr_d)

    def residual(self, noise, theta_star) -> dict:
        """p_hat (mean prediction over the noise batch) and r_hat = (theta* - p_hat) / theta*."""
        return self.ctx.ensemble_response(self.G_W, self.G_b, noise, p_true=theta_star, slope=self.slope)


def score_closure(ctx: Context, steps: int, report_every: int = 100, k: int = 1024, events_per_theta: int = 100,
                  objective: str = "policy", seed: int = 0, log: Optional[Callable] = None, **kw) -> List[dict]:
    """The loop-closure test (generator 6-128-128-128-128-6, discriminator 2-128-128-128-128-1,
    reference data at theta* = (2, 5, 1.5, 3, 3, 2)) without a gradient through the pipeline."""
    import numpy as np
    import torch

    from workloads import gen

    dev = "cuda:%d" % ctx.device
    ts = torch.tensor([[2.0, 5.0, 1.5, 3.0, 3.0, 2.0]], device=dev)
    pool = ctx.sample_events(ts, 2 * k * events_per_theta, seed + 1)
    GW, Gb = gen.generator_stack((6, 128, 128, 128, 128, 6), 1, seed + 21)
    DW, Db = gen.xavier_mlp((2, 128, 128, 128, 128, 1), seed + 2)
    to = lambda arrs: [torch.tensor(a, device=dev) for a in arrs]      # noqa: E731
    loop = ScoreLoop(ctx, to(w[0] for w in GW), to(v[0] for v in Gb), to(DW), to(Db), pool, k, events_per_theta,
                     objective=objective, fake_seed=seed, boot_seed=seed + 5, **kw)
    rng = np.random.default_rng(seed + 22)
    draw = lambda: torch.tensor(rng.standard_normal((k, 6)).astype(np.float32), device=dev)   # noqa: E731
    eval_noise = draw()
    history = []
    for s in range(1, steps + 1):
        loop.step(draw())
        if s % report_every == 0 or s == steps:
            r = loop.residual(eval_noise, ts[0])
            rec = {"step": s, "loss": loop.last["loss"].item(), "loss_d": loop.outs["loss_d"].item(),
                   "p_hat": r["p_hat"].tolist(), "r_hat": r["r_hat"].tolist()}
            history.append(rec)
            if log:
                log(rec)
    return history


if __name__ == "__main__":
    import argparse
    import json

    ap = argparse.ArgumentParser(description="loop-closure run that learns from scores alone, on one GPU")
    ap.add_argument("--steps", type=int, default=1000)
    ap.add_argument("--report-every", type=int, default=100)
    ap.add_argument("--objective", choices=("policy", "preference"), default="policy")
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    ctx = Context(0)
    score_closure(ctx, a.steps, a.report_every, objective=a.objective, seed=a.seed, log=lambda r: print(json.dumps(r), flush=True))
    ctx.close()
