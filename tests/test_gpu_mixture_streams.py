"""A mixture in the GAN loop on a context with a stream of its own: inputs and results that are dropped while their
stream still works on them keep their values."""
import numpy as np
import pytest

from workloads import gen

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2407_00051_amd as sg  # noqa: E402
from paper_2407_00051_amd import gan  # noqa: E402

M, K = 4, 2000


def _loop(ctx):
    W, b = gen.generator_stack((6, 128, 128, 128, 128, 6), M, seed=40)
    DW, Db = gen.xavier_mlp((2, 128, 128, 128, 128, 1), 2)
    to = lambda arrs: [torch.tensor(a, device="cuda:0") for a in arrs]      # noqa: E731
    r = np.random.default_rng(41)
    router = to([r.standard_normal((M, 6)).astype(np.float32), np.zeros(M, np.float32)])
    return gan.GanLoop(ctx, to(W), to(b), to(DW), to(Db), torch.zeros((100, 2), device="cuda:0"), K, 1, router=router, top=2)


def _inputs():
    return (torch.tensor(gen.noise(K, 6, seed=42), device="cuda:0"),
            torch.tensor([2.0, 5.0, 1.5, 3.0, 3.0, 2.0], device="cuda:0"))


def _fill(like, count=8):
    """Memory of these shapes, taken from the current stream's free blocks and overwritten."""
    for shape in like:
        for _ in range(count):
            torch.full(shape, float("nan"), device="cuda:0")
        held = [torch.full(shape, float("nan"), device="cuda:0") for _ in range(count)]
        del held


def test_residual_keeps_dropped_inputs_and_results(gpu_ctx):
    print("case residual on its own stream", flush=True)
    busy = torch.randn((2048, 65536), device="cuda:0")
    noise, star = _inputs()
    want = _loop(gpu_ctx).residual(noise, star)
    want = [want[k].clone() for k in ("p_hat", "r_hat")]
    own = torch.cuda.Stream()
    ctx = sg.Context(0, stream=own)
    loop = _loop(ctx)
    loop.residual(noise, star)                             # the library's workspaces and torch's
    del noise, star
    torch.cuda.synchronize()
    for _ in range(3):
        noise, star = _inputs()
        torch.cuda.synchronize()
        for _ in range(4):
            ctx.choice_logprob(busy)                       # the context's stream has work before the call's
        r = loop.residual(noise, star)
        shapes = [noise.shape, star.shape]
        del noise, star
        _fill(shapes)                                      # on the caller's stream, which is free
        torch.cuda.current_stream().wait_stream(own)
        for _ in range(4):
            gpu_ctx.choice_logprob(busy)                   # and the caller's before it reads the results
        got = [r[k].clone() for k in ("p_hat", "r_hat")]
        shapes = [r["p_hat"].shape]
        del r
        with torch.cuda.stream(own):
            _fill(shapes)
        torch.cuda.synchronize()
        # the router's product is the library's, whose bits need not be the same from call to call
        assert all(torch.allclose(a, c, rtol=1e-4, atol=1e-5) for a, c in zip(got, want)), (got, want)
    ctx.close()
