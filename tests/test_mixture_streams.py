"""Which stream a mixture's tensors are marked for, on the CPU: a context on a stream of its own, whose calls are
stood in for by plain torch, with torch's streams and record_stream replaced by a record of what they were given."""
from contextlib import contextmanager

import pytest

torch = pytest.importorskip("torch")
import paper_2407_00051_amd as sg  # noqa: E402
from paper_2407_00051_amd import gan  # noqa: E402
from paper_2407_00051_amd.mixture import Mixture  # noqa: E402

K, M, TOP, IN, OUT = 12, 3, 2, 4, 5


class _Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


class _Record:
    """(tensor, stream) of every record_stream call; tensors are held, so that none takes another's place."""

    def __init__(self):
        self.caller, self.own = _Stream(1), _Stream(2)
        self.current, self.calls = self.caller, []

    def streams(self, t):
        return [s for a, s in self.calls if a is t]


@pytest.fixture
def record(monkeypatch):
    r = _Record()

    @contextmanager
    def stream(s):
        before, r.current = r.current, s
        yield
        r.current = before

    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: r.current)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: r.calls.append((t, s)))
    return r


class _Context(sg.Context):
    """The library's calls of a mixture, of the right shapes; the first `top` members take every row."""

    def __init__(self, record, follow=False):
        self.device, self._follow, self._stream, self.h = 0, follow, record.caller if follow else record.own, None

    def choice_logprob(self, logits, choice=None, top=0, scale=1.0):
        n = logits.shape[0]
        lp = torch.log_softmax(logits, 1)[:, :top]
        return {"entropy": torch.zeros(n), "top_logp": lp, "top_choice": torch.arange(top, dtype=torch.int32).repeat(n, 1)}

    def choice_backward(self, logits, fwd, choice=None, d_logp=None, d_entropy=None, d_top=None, scale=1.0, out=None):
        return torch.zeros_like(logits)

    def route(self, member, n_members):
        return {"offsets": torch.zeros(n_members + 1, dtype=torch.int32), "place": torch.arange(member.numel()).view(member.shape)}

    def dispatch(self, x, plan, out=None):
        return x.repeat_interleave(TOP, 0)

    def gen_forward_routed(self, W, b, x, offsets, slope=0.2, out=None):
        return torch.ones(x.shape[0], W[-1].shape[1])

    def gen_backward_routed(self, W, b, x, offsets, dL_dtheta, slope=0.2, dW=None, db=None, want_dx=False, dx=None):
        return dW, db, None

    def combine(self, y, plan, weight=None, out=None):
        return (y.view(K, TOP, -1) * weight[..., None]).sum(1)

    def combine_backward(self, dout, y, plan, weight=None, want_dweight=True, dy=None):
        return torch.zeros_like(y), torch.zeros_like(weight)


def _stack():
    widths = (IN, 8, OUT)
    return ([torch.zeros(M, widths[l + 1], widths[l]) for l in range(2)], [torch.zeros(M, widths[l + 1]) for l in range(2)],
            torch.zeros(M, IN), torch.zeros(M))


def _loop(ctx):
    W, b, Wr, br = _stack()
    return gan.GanLoop(ctx, W, b, [torch.zeros(1, 2)], [torch.zeros(1)], torch.zeros(6, 2), K, 1, router=(Wr, br), top=TOP)


def test_residual_marks_what_it_takes_and_gives(record):
    """What a caller hands in and may drop is marked for the context's stream, what it gets for the caller's."""
    loop = _loop(_Context(record))
    noise, star = torch.randn(K, IN), torch.ones(OUT)
    r = loop.residual(noise, star)
    assert record.current is record.caller
    for name, t in (("noise", noise), ("theta_star", star)):
        assert record.own in record.streams(t), name
    for name in ("p_hat", "r_hat"):
        assert record.caller in record.streams(r[name]), name


def test_a_following_context_marks_nothing(record):
    loop = _loop(_Context(record, follow=True))
    loop.residual(torch.randn(K, IN), torch.ones(OUT))
    loop.mixture.backward(torch.zeros(K, OUT))
    assert record.calls == []


def test_a_pass_marks_its_inputs_and_theta(record):
    W, b, Wr, br = _stack()
    mix = Mixture(_Context(record), W, b, Wr, br, top=TOP)
    noise, d = torch.randn(K, IN), torch.zeros(K, OUT)
    theta = mix.forward(noise)
    mix.backward(d)
    assert record.streams(noise) == [record.own] and record.streams(d) == [record.own]
    assert record.streams(theta) == [record.caller]


def test_residual_has_what_a_single_generator_gives(record):
    """p_hat, sigma and r_hat, as ensemble_response: one generator has no spread, and without theta* there is no r_hat."""
    loop = _loop(_Context(record))
    r = loop.residual(torch.randn(K, IN), torch.full((OUT,), 2.0))
    assert set(r) == {"p_hat", "sigma", "r_hat"} and r["sigma"].tolist() == [0.0] * OUT
    assert record.caller in record.streams(r["sigma"])
    assert torch.allclose(r["r_hat"], (2.0 - r["p_hat"]) / 2.0)
    none = loop.residual(torch.randn(K, IN), None)
    assert none["r_hat"] is None and none["p_hat"].shape == (OUT,)


def test_parameters_and_gradients_are_marked(record):
    """A mixture may be dropped, parameters and gradients with it, while the context's stream works on them; a
    stream set later is marked too."""
    W, b, Wr, br = _stack()
    ctx = _Context(record)
    mix = Mixture(ctx, W, b, Wr, br, top=TOP)
    with mix.on_stream():                                  # a caller who is on that stream already
        mix.forward(torch.randn(K, IN))
    mix.forward(torch.randn(K, IN))
    mix.backward(torch.zeros(K, OUT))
    for t in mix.parameters() + mix.gradients():
        assert record.streams(t) == [record.own]
    mix.forward(torch.randn(K, IN))
    other = ctx._stream = _Stream(3)
    mix.forward(torch.randn(K, IN))
    for t in mix.parameters() + mix.gradients():
        assert record.streams(t) == [record.own, other]
