"""The losses and the matrix update recorded in one HIP graph on a context's own stream: every
replay gives bit for bit what eager calls give on the same inputs, with eager work of the program
and synchronisations between the replays.  (Results are deterministic: no tolerance.)"""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2407_00051_amd as sg  # noqa: E402

# rows, events, matrices: one row that ends in its last workgroup, many rows, long sets and large matrices
CASES = [(1, 3000, (2, 40, 60)), (300, 100, (3, 128, 128)), (4, 20000, (1, 200, 300))]


def _inputs(rows, events, shape, seed):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    rand = lambda *s: torch.rand(s, generator=g, device="cuda:0")          # noqa: E731
    theta = 1.0 + 4.0 * rand(rows, 6)
    return dict(theta=theta, old=theta * (1.0 + 0.1 * rand(rows, 6)), x=rand(rows, events, 3), reward=rand(rows, events),
                other=rand(rows, events, 3), p=rand(*shape), grad=rand(*shape) - 0.5, m=torch.zeros(shape, device="cuda:0"))


def _calls(ctx, t):
    adv = ctx.group_advantage(t["reward"])
    a = ctx.policy_loss(t["theta"], t["old"], t["x"], adv, theta_ref=t["old"], kl_coef=0.1, average="rows")
    b = ctx.preference_loss(t["theta"], t["old"], t["x"], t["other"])
    ctx.muon_step([t["p"]], [t["grad"]], [t["m"]], 0.05)
    return [adv, a["loss"], a["kl"], a["clip_frac"], a["dtheta"], b["loss"], b["margin"], b["dtheta"], t["p"], t["m"]]


@pytest.mark.parametrize("rows,events,shape", CASES)
def test_replays_equal_eager_calls(gpu_ctx, rows, events, shape):
    print(f"case graph {rows} x {events}, {shape}", flush=True)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        ctx = sg.Context(0, stream=st)
        held = _inputs(rows, events, shape, 0)
        _calls(ctx, held)                                  # workspaces grow here, not in the capture
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            out = _calls(ctx, held)
        for replay in range(4):
            new = _inputs(rows, events, shape, 10 + replay)
            for k in held:
                held[k].copy_(new[k])
            graph.replay()
            st.synchronize()
            got = [v.clone() for v in out]
            want = _calls(ctx, new)                        # eager, same context, between the replays
            st.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), [torch.equal(a, b) for a, b in zip(got, want)]
        st.synchronize()
        ctx.close()
