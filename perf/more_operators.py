"""The operators of a mixture of generators, as cases that can be timed and compared:
the choice of members (log probabilities of given choices, entropy and the most likely
alternatives, and the gradient), rows sorted by member and back with weights applied (and
the gradient), and the members' networks on the rows that each was given.

  listed()   twelve cases, from one noise batch's router to the largest batches
  draw(rng)  one more case of the same kinds and ranges
  prepare, run, work, exact: see each function

run() computes an operator in elementary fp32 torch operations, or, where `own`
is set, through the library's entry points.  exact() states the results in
float64, from the definitions, without either.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SLOPE = 0.2
HIDDEN = 128


# ---------------------------------------------------------------------------
# The cases

def listed():
    return [
        # the router of the paper's noise batch: 1,024 rows choose 2 of 8 members (latency)
        dict(name="choice_router", kind="choice", rows=1024, choices=8, top=2, dtype="f32", scale=1.0, masked=0.0, pad=0),
        # one row over many choices with twenty alternatives, as a discrete policy is asked step by step
        dict(name="choice_one_row", kind="choice", rows=1, choices=131072, top=20, dtype="bf16", scale=0.7, masked=0.0, pad=0),
        # a training batch of a policy over many choices, and one of odd sizes with masked choices in strided rows
        dict(name="choice_large", kind="choice", rows=4096, choices=65536, top=8, dtype="bf16", scale=1.0, masked=0.0, pad=0),
        dict(name="choice_ragged", kind="choice", rows=3001, choices=1543, top=5, dtype="f32", scale=1.3, masked=0.3, pad=7),
        # the router's gradient, and a policy's over an odd number of choices
        dict(name="choice_grad_router", kind="choice_grad", rows=1024, choices=8, top=2, dtype="f32", scale=1.0, masked=0.1, pad=0),
        dict(name="choice_grad_large", kind="choice_grad", rows=4096, choices=50001, top=1, dtype="bf16", scale=1.0, masked=0.0,
             pad=0),
        # the paper's noise batch sorted by member, and a large batch of wide hidden rows over many
        # experts; a few choices are dropped
        dict(name="dispatch_paper", kind="dispatch", rows=1024, slots=2, members=8, width=6, dtype="f32", skew=1.0, dropped=0.0),
        dict(name="dispatch_large", kind="dispatch", rows=16384, slots=8, members=256, width=2048, dtype="bf16", skew=0.5,
             dropped=0.05),
        # theta of the paper's batch put back in order with its weights, forward and gradient, and wide rows
        dict(name="combine_paper", kind="combine", rows=1024, slots=2, members=8, width=6, dtype="f32", skew=1.0, dropped=0.0),
        dict(name="combine_large", kind="combine", rows=16384, slots=8, members=256, width=2048, dtype="bf16", skew=0.5,
             dropped=0.05),
        # the paper's generator, 100 members on an unevenly shared batch of noise rows, and the gradients of a
        # mixture of 8 members in a training step
        dict(name="members_forward", kind="members", items=131072, members=100, layers=3, inputs=6, outputs=6, skew=0.7),
        dict(name="members_grad", kind="members_grad", items=16384, members=8, layers=3, inputs=6, outputs=6, skew=0.7),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["choice", "choice", "choice_grad", "choice_grad", "dispatch", "combine", "members", "members_grad"])
    if kind.startswith("choice"):
        dtype = rng.choice(["f32", "bf16"])
        choices = _log_int(rng, 2, 200000)
        most = (1 << 27) // (2 if dtype == "f32" else 1)
        rows = _log_int(rng, max(1, 1024 // choices), max(1, min(65536, most // choices)))
        return dict(kind=kind, rows=rows, choices=choices, top=min(choices, rng.choice([0, 1, 2, 4, 8, 20, 32])), dtype=dtype,
                    scale=rng.choice([1.0, 0.7, 1.3]), masked=rng.choice([0.0, 0.3]), pad=rng.choice([0, 0, 5, 16]))
    if kind in ("dispatch", "combine"):
        dtype = rng.choice(["f32", "bf16"])
        rows, slots = _log_int(rng, 1, 65536), rng.randint(1, 8)
        most = (1 << 27) // (2 if dtype == "f32" else 1)
        return dict(kind=kind, rows=rows, slots=slots, members=_log_int(rng, 1, 512),
                    width=_log_int(rng, 1, max(1, min(8192, most // (rows * slots)))), dtype=dtype,
                    skew=rng.choice([0.0, 0.5, 1.0]), dropped=rng.choice([0.0, 0.05]))
    return dict(kind=kind, items=_log_int(rng, 16, 131072 if kind == "members" else 16384), members=_log_int(rng, 1, 100),
                layers=rng.randint(1, 3), inputs=rng.randint(1, 8), outputs=rng.randint(1, 8), skew=rng.choice([0.0, 0.7, 1.0]))


# ---------------------------------------------------------------------------
# Inputs

def _dev():
    return torch.device("cuda:0")


def _rng(seed, salt):
    return torch.Generator(device=_dev()).manual_seed(int(seed) * 1000003 + salt)


def _rand(g, *shape):
    return torch.rand(shape, generator=g, device=_dev())


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=_dev())


def _chosen_members(g, n, members, skew):
    """Members of n items [n] int64: member m is taken with a weight that falls as (m + 1)^-skew."""
    share = torch.arange(1, members + 1, device=_dev(), dtype=torch.float64) ** -skew
    edges = torch.cumsum(share / share.sum(), 0)
    u = torch.rand(n, generator=g, device=_dev(), dtype=torch.float64)
    return torch.searchsorted(edges, u).clamp_(max=members - 1)


def _inputs(case, seed):
    """The tensors of a case, from the seed alone."""
    kind, g = case["kind"], _rng(seed, 23)
    t = {}
    if kind.startswith("choice"):
        n, V, K = case["rows"], case["choices"], case["top"]
        # logits with a few likely choices a row; where choices are masked every 61st row loses all
        x = torch.empty((n, V + case["pad"]), dtype=DTYPES[case["dtype"]], device=_dev())
        step = max(1, (1 << 26) // x.shape[1])
        for i in range(0, n, step):
            v = x[i:i + step]
            z = _randn(g, *v.shape)
            v.copy_(z * (1.0 + z.abs()))
        t["logits"] = x[:, :V]
        t["choice"] = (_rand(g, n) ** 2 * V).floor().clamp_(max=V - 1).to(torch.int32)
        if case["masked"]:
            for i in range(0, n, step):
                cut = _rand(g, *x[i:i + step].shape) < case["masked"]
                x[i:i + step].masked_fill_(cut, float("-inf"))
            t["logits"][60::61] = float("-inf")
            t["choice"][_rand(g, n) < 0.02] = -1           # rows without a choice of their own (padding)
        if kind == "choice_grad":
            t["d_logp"], t["d_entropy"] = _randn(g, n), 0.1 * _randn(g, n)
            t["d_top"] = _randn(g, n, K) if K else None
        return t
    if kind in ("dispatch", "combine"):
        n, K, w = case["rows"], case["slots"], case["width"]
        m = _chosen_members(g, n * K, case["members"], case["skew"])
        if case["dropped"]:
            m = torch.where(_rand(g, n * K) < case["dropped"], -1, m)
        t["member"] = m.reshape(n, K).to(torch.int32)
        dt = DTYPES[case["dtype"]]
        if kind == "dispatch":
            t["x"] = _randn(g, n, w).to(dt)
            t["sorted"] = torch.zeros((n * K, w), dtype=dt, device=_dev())
        else:
            t["y"] = _randn(g, n * K, w).to(dt)
            t["dout"] = _randn(g, n, w).to(dt)
            t["weight"] = torch.softmax(_randn(g, n, K), 1)
            t["dy"] = torch.zeros((n * K, w), dtype=dt, device=_dev())
            # the sorting of an earlier call of the same step
            key = torch.where(m < 0, case["members"], m)
            order = torch.sort(key, stable=True)[1]
            total = int((m >= 0).sum())
            place = torch.empty_like(order)
            place[order] = torch.arange(n * K, device=_dev())
            edge = torch.searchsorted(key[order], torch.arange(case["members"] + 1, device=_dev()))
            order[total:] = -1
            t["plan"] = {"offsets": edge.to(torch.int32), "order": order.to(torch.int32),
                         "place": torch.where(place < total, place, -1).reshape(n, K).to(torch.int32)}
        return t
    # networks as the framework initialises them: Kaiming-normal weights, uniform biases
    n, M = case["items"], case["members"]
    widths = [case["inputs"]] + [HIDDEN] * (case["layers"] + 1) + [case["outputs"]]
    t["W"] = [_randn(g, M, b, a) * math.sqrt(2.0 / ((1.0 + SLOPE * SLOPE) * a)) for a, b in zip(widths, widths[1:])]
    t["b"] = [(2.0 * _rand(g, M, b) - 1.0) / math.sqrt(a) for a, b in zip(widths, widths[1:])]
    t["x"] = _randn(g, n, case["inputs"])
    m = _chosen_members(g, n, M, case["skew"])
    t["counts"] = torch.bincount(m, minlength=M)
    t["offsets"] = torch.cat([t["counts"].new_zeros(1), torch.cumsum(t["counts"], 0)]).to(torch.int32)
    if kind == "members_grad":
        t["dtheta"] = _randn(g, n, case["outputs"])
        t["dtheta"][_near_kink(t)] = 0.0
    return t


def _spans(t):
    """(member, first row, row after the last) of every member that has rows."""
    edge = t["offsets"].tolist()
    return [(m, lo, hi) for m, (lo, hi) in enumerate(zip(edge, edge[1:])) if hi > lo]


def _near_kink(t):
    """Rows with a hidden unit within rounding of LeakyReLU's kink, where 32 bits may decide either
    way: they get no gradient, so that every result is a definite one."""
    near = torch.zeros(t["x"].shape[0], dtype=torch.bool, device=_dev())
    for m, lo, hi in _spans(t):
        h = t["x"][lo:hi].double()
        for W, b in list(zip(t["W"], t["b"]))[:-1]:
            W, b = W[m].double(), b[m].double()
            pre = h @ W.T + b
            size = h.abs() @ W.abs().T + b.abs()
            near[lo:hi] |= (pre.abs() <= 1e-5 * size).any(1)
            h = torch.where(pre > 0, pre, SLOPE * pre)
    return near


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if "counts" in s:
        s["longest"] = int(s["counts"].max())              # known to a program that has sorted its rows
    if own:
        import paper_2407_00051_amd as sg
        s["ctx"] = sg.default_context(0)
    if case["kind"] == "choice_grad":                      # what the forward call of the same step left
        if own:
            s["fwd"] = s["ctx"].choice_logprob(s["logits"], s["choice"], top=case["top"], scale=case["scale"])
        else:
            s["fwd"] = _choice_plain(s)
    return s


# ---------------------------------------------------------------------------
# One pass

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    ctx, case = s["ctx"], s["case"]
    kind = case["kind"]
    if kind == "choice":
        o = ctx.choice_logprob(s["logits"], s["choice"], top=case["top"], scale=case["scale"])
        return {k: o[k] for k in ("logp", "entropy", "top_choice", "top_logp")}
    if kind == "choice_grad":
        return ctx.choice_backward(s["logits"], s["fwd"], s["choice"], d_logp=s["d_logp"], d_entropy=s["d_entropy"],
                                   d_top=s["d_top"], scale=case["scale"])
    if kind == "dispatch":
        plan = ctx.route(s["member"], case["members"])
        xs = ctx.dispatch(s["x"], plan, out=s["sorted"])
        return {**{k: plan[k] for k in ("offsets", "order", "place")}, "sorted": xs}
    if kind == "combine":
        out = ctx.combine(s["y"], s["plan"], s["weight"])
        dy, dweight = ctx.combine_backward(s["dout"], s["y"], s["plan"], s["weight"], dy=s["dy"])
        return {"out": out, "dy": dy, "dweight": dweight}
    if kind == "members":
        return ctx.gen_forward_routed(s["W"], s["b"], s["x"], s["offsets"], slope=SLOPE)
    dW, db, dx = ctx.gen_backward_routed(s["W"], s["b"], s["x"], s["offsets"], s["dtheta"], slope=SLOPE, want_dx=True)
    return {"dW": dW, "db": db, "dx": dx}


def _choice_plain(s):
    case = s["case"]
    x, K = s["logits"].float(), case["top"]
    V = x.shape[1]
    z = case["scale"] * x
    m = z.amax(1, keepdim=True)
    empty = m[:, 0] == float("-inf")
    d = z - torch.where(empty[:, None], 0.0, m)
    e = torch.exp(d)
    total = e.sum(1)
    log_total = torch.log(total)
    entropy = torch.where(empty, 0.0, log_total - torch.where(e > 0, e * d, 0.0).sum(1) / total)
    choice = s["choice"].long()
    given = (choice >= 0) & (choice < V)
    logp = torch.where(given, d.gather(1, choice.clamp(0, V - 1)[:, None])[:, 0] - log_total, 0.0)
    logp = torch.where(given & empty, float("-inf"), logp)
    o = {"logp": logp, "entropy": entropy}
    # alternatives by logit, the lower index first where they are equal: one 64-bit key each
    if K:
        bits = (x + 0.0).view(torch.int32).long()
        key = ((bits ^ ((bits >> 31) & 0x7FFFFFFF)) << 32) + (V - 1 - torch.arange(V, device=x.device))
        top = V - 1 - (torch.topk(key, K, dim=1)[0] & 0xFFFFFFFF)
        lp = d.gather(1, top) - log_total[:, None]
        none = x.gather(1, top) == float("-inf")
        o["top_choice"] = torch.where(none, -1, top).to(torch.int32)
        o["top_logp"] = torch.where(none, float("-inf"), lp)
    else:
        o["top_choice"] = torch.empty((x.shape[0], 0), dtype=torch.int32, device=x.device)
        o["top_logp"] = torch.empty((x.shape[0], 0), device=x.device)
    return {**o, "shift": torch.where(empty[:, None], 0.0, m), "log_total": log_total[:, None]}


def _choice_grad_plain(s):
    case, f = s["case"], s["fwd"]
    x, V = s["logits"].float(), s["logits"].shape[1]
    lp = case["scale"] * x - f["shift"] - f["log_total"]
    p = torch.where(x == float("-inf"), 0.0, torch.exp(lp))
    choice = s["choice"].long()
    hit = (choice >= 0) & (choice < V) & (f["logp"] > float("-inf"))
    gl = torch.where(hit, s["d_logp"], 0.0)
    total = gl
    if case["top"]:
        on = f["top_choice"] >= 0
        gt = torch.where(on, s["d_top"], 0.0)
        total = gl + gt.sum(1)
    dz = -p * total[:, None] - s["d_entropy"][:, None] * torch.where(p > 0, p * (lp + f["entropy"][:, None]), 0.0)
    dz.scatter_add_(1, choice.clamp(0, V - 1)[:, None], gl[:, None])
    if case["top"]:
        dz.scatter_add_(1, f["top_choice"].long().clamp(min=0), gt)
    return (case["scale"] * dz).to(s["logits"].dtype)


def _members_plain(s, backward):
    """Every member's rows padded to the longest member's."""
    n, L = s["x"].shape[0], s["longest"]
    lo, count = s["offsets"][:-1].long()[:, None], s["counts"][:, None]
    at = torch.arange(L, device=_dev())[None, :]
    on = at < count
    row = torch.where(on, lo + at, n)                                  # n: a row of zeros
    take = lambda v: torch.cat([v, v.new_zeros(1, v.shape[1])])[row]   # noqa: E731
    hs = [take(s["x"])]
    for l, (W, b) in enumerate(zip(s["W"], s["b"])):
        pre = torch.bmm(hs[-1], W.transpose(1, 2).contiguous()) + b[:, None, :]
        hs.append(pre if l == len(s["W"]) - 1 else torch.where(pre > 0, pre, SLOPE * pre))
    o = hs.pop()
    back = (torch.repeat_interleave(torch.arange(row.shape[0], device=_dev()), s["counts"], output_size=n) * L
            + torch.arange(n, device=_dev()) - torch.repeat_interleave(lo[:, 0], s["counts"], output_size=n))
    if not backward:
        theta = 1.0 + o.clamp(min=0.0) + torch.log1p(torch.exp(-o.abs()))
        return theta.flatten(0, 1)[back]
    g = take(s["dtheta"]) * torch.sigmoid(o)
    dW, db = [], []
    for l in range(len(s["W"]) - 1, -1, -1):
        dW.append(torch.bmm(g.transpose(1, 2).contiguous(), hs[l]))
        db.append(g.sum(1))
        g = torch.bmm(g, s["W"][l])
        if l:
            g = torch.where(hs[l] > 0, g, SLOPE * g)
    return {"dW": dW[::-1], "db": db[::-1], "dx": g.flatten(0, 1)[back]}


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "choice":
        o = _choice_plain(s)
        return {k: o[k] for k in ("logp", "entropy", "top_choice", "top_logp")}
    if kind == "choice_grad":
        return _choice_grad_plain(s)
    if kind == "dispatch":
        n, K, M = case["rows"], case["slots"], case["members"]
        m = s["member"].reshape(-1).long()
        key = torch.where((m >= 0) & (m < M), m, M)
        by, order = torch.sort(key, stable=True)
        at = torch.arange(n * K, device=m.device)
        place = torch.empty_like(order)
        place[order] = at
        on = by < M
        xs = s["sorted"]
        xs.copy_(torch.where(on[:, None], s["x"][torch.div(order, K, rounding_mode="floor")], xs))
        return {"offsets": torch.searchsorted(by, torch.arange(M + 1, device=m.device)).to(torch.int32),
                "order": torch.where(on, order, -1).to(torch.int32),
                "place": torch.where(key < M, place, -1).reshape(n, K).to(torch.int32), "sorted": xs}
    if kind == "combine":
        n, K, w = case["rows"], case["slots"], case["width"]
        place = s["plan"]["place"].long()
        on = place >= 0
        y = s["y"][place.clamp(min=0)].float()                                      # [n][K][w]
        weight = torch.where(on, s["weight"], 0.0)
        out = (weight[:, :, None] * y).sum(1).to(s["y"].dtype)
        dout = s["dout"].float()
        dweight = torch.where(on, (dout[:, None, :] * y).sum(2), 0.0)
        dy, order = s["dy"], s["plan"]["order"].long()
        at = order.clamp(min=0)
        g = (s["weight"].flatten()[at][:, None] * dout[torch.div(at, K, rounding_mode="floor")]).to(dy.dtype)
        dy.copy_(torch.where((order >= 0)[:, None], g, dy))
        return {"out": out, "dy": dy, "dweight": dweight}
    return _members_plain(s, kind == "members_grad")


# ---------------------------------------------------------------------------
# What one pass cannot do without

def work(case):
    """Bytes: inputs once and outputs once.  Flops: eight operations a logit for the choices; of the
    networks two a weight and row in each product."""
    kind = case["kind"]
    if kind.startswith("choice"):
        n, V, K, size = case["rows"], case["choices"], case["top"], 2.0 if case["dtype"] == "bf16" else 4.0
        grad = kind == "choice_grad"
        return {"bytes": n * V * size * (2 if grad else 1) + n * (12.0 + 8.0 * K + (16.0 if grad else 0.0)), "flops": 8.0 * n * V}
    if kind in ("dispatch", "combine"):
        n, K, w, size = case["rows"], case["slots"], case["width"], 2.0 if case["dtype"] == "bf16" else 4.0
        items = n * K * (1.0 - case["dropped"])
        if kind == "dispatch":
            return {"bytes": size * w * (n + items) + 12.0 * n * K + 4.0 * case["members"], "flops": 1.0 * n * K}
        # y read once for both directions would need them together: two passes are two reads
        return {"bytes": size * w * (2 * n + 3 * items) + 16.0 * n * K, "flops": 5.0 * items * w}
    n, M = case["items"], case["members"]
    widths = [case["inputs"]] + [HIDDEN] * (case["layers"] + 1) + [case["outputs"]]
    weights = sum(a * b for a, b in zip(widths, widths[1:]))
    params = 4.0 * M * (weights + sum(widths[1:]))
    if kind == "members":
        return {"bytes": 4.0 * n * (case["inputs"] + case["outputs"]) + params, "flops": 2.0 * n * weights}
    return {"bytes": 4.0 * n * (2 * case["inputs"] + case["outputs"]) + 2.0 * params, "flops": 6.0 * n * weights}


# ---------------------------------------------------------------------------
# The results in float64

def _choice64(t, case, backward):
    n, V, K = case["rows"], case["choices"], case["top"]
    inf = float("inf")
    out = {"logp": [], "entropy": [], "top_choice": [], "top_logp": []}
    grads = []
    step = max(1, (1 << 24) // V)
    for i in range(0, n, step):
        x = t["logits"][i:i + step].double()
        c = t["choice"][i:i + step].long()
        lp = torch.log_softmax(case["scale"] * x, 1)
        none = (x == -inf).all(1)
        lp = torch.where(x == -inf, -inf, lp)                        # rows without any choice: all of them
        p = torch.exp(lp)
        H = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
        given = (c >= 0) & (c < V)
        mine = lp[torch.arange(len(c), device=c.device), c.clamp(0, V - 1)]
        out["logp"].append(torch.where(given, mine, 0.0))
        out["entropy"].append(torch.where(none, 0.0, H))
        idx = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :K]
        tl = torch.gather(lp, 1, idx)
        idx = torch.where(tl == -inf, -1, idx)
        out["top_choice"].append(idx.to(torch.int32))
        out["top_logp"].append(tl)
        if backward:
            gH = t["d_entropy"][i:i + step].double()[:, None]
            gl = torch.where(given & (mine > -inf), t["d_logp"][i:i + step].double(), 0.0)
            u = torch.zeros_like(x)                                  # dL / d lp
            u[torch.arange(len(c), device=c.device), c.clamp(0, V - 1)] += gl
            if K:
                gt = torch.where(idx >= 0, t["d_top"][i:i + step].double(), 0.0)
                u = u.scatter_add(1, idx.long().clamp(min=0), gt)
            # H = -sum p lp: dH / dz_v = -p_v (lp_v + H)
            dz = u - p * u.sum(1, keepdim=True) - gH * torch.where(p > 0, p * (lp + H[:, None]), torch.zeros_like(p))
            grads.append(case["scale"] * dz)
    return torch.cat(grads) if backward else {k: torch.cat(v) for k, v in out.items()}


def _members64(t, case, backward):
    n = case["items"]
    f64 = dict(dtype=torch.float64, device=_dev())
    theta, dx = torch.zeros((n, case["outputs"]), **f64), torch.zeros((n, case["inputs"]), **f64)
    dW, db = [torch.zeros(w.shape, **f64) for w in t["W"]], [torch.zeros(v.shape, **f64) for v in t["b"]]
    for m, lo, hi in _spans(t):
        W, b = [w[m].double() for w in t["W"]], [v[m].double() for v in t["b"]]
        act, pres = [t["x"][lo:hi].double()], []
        for l in range(len(W)):
            pres.append(act[-1] @ W[l].T + b[l])
            act.append(torch.nn.functional.leaky_relu(pres[-1], SLOPE))
        theta[lo:hi] = 1.0 + torch.nn.functional.softplus(pres[-1], threshold=1000.0)
        if backward:
            delta = t["dtheta"][lo:hi].double() / (1.0 + torch.exp(-pres[-1]))
            for l in reversed(range(len(W))):
                dW[l][m], db[l][m] = delta.T @ act[l], delta.sum(0)
                delta = delta @ W[l]
                if l:
                    delta = delta * torch.where(pres[l - 1] > 0, 1.0, SLOPE)
            dx[lo:hi] = delta
    return {"dW": dW, "db": db, "dx": dx} if backward else theta


def exact(case, seed):
    t, kind = _inputs(case, seed), case["kind"]
    if kind.startswith("choice"):
        return _choice64(t, case, kind == "choice_grad")
    if kind in ("dispatch", "combine"):
        n, K, M = case["rows"], case["slots"], case["members"]
        member = t["member"].cpu().numpy().ravel()
        items = np.flatnonzero((member >= 0) & (member < M))
        order = items[np.argsort(member[items], kind="stable")]
        place = np.full(n * K, -1, dtype=np.int64)
        place[order] = np.arange(len(order))
        if kind == "dispatch":
            xs = torch.zeros((n * K, case["width"]), dtype=torch.float64, device=_dev())
            xs[:len(order)] = t["x"][torch.from_numpy(order // K).to(_dev())].double()
            return {"offsets": np.concatenate([[0], np.cumsum(np.bincount(member[items], minlength=M))]).astype(np.int32),
                    "order": np.concatenate([order, np.full(n * K - len(order), -1)]).astype(np.int32),
                    "place": place.reshape(n, K).astype(np.int32), "sorted": xs}
        out = torch.zeros((n, case["width"]), dtype=torch.float64, device=_dev())
        dy = torch.zeros((n * K, case["width"]), dtype=torch.float64, device=_dev())
        dweight = torch.zeros((n, K), dtype=torch.float64, device=_dev())
        place = torch.from_numpy(place.reshape(n, K)).to(_dev())
        for k in range(K):
            rows = torch.nonzero(place[:, k] >= 0)[:, 0]
            p, w = place[rows, k], t["weight"][rows, k].double()[:, None]
            yk, dk = t["y"][p].double(), t["dout"][rows].double()
            out[rows] += w * yk
            dy[p] = w * dk
            dweight[rows, k] = (dk * yk).sum(1)
        return {"out": out, "dy": dy, "dweight": dweight}
    return _members64(t, case, kind == "members_grad")
