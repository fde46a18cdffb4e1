"""The choices at the ends of what they accept, against the float64 oracle: finite logits near the type's
lowest and largest values, masked choices of NaN rows, padding of in-place gradients, sizes beyond 32 bits.

Tolerances are those of test_gpu_choice.py; an ln p below fp32's lowest number is that number."""
import numpy as np
import pytest

from oracle import mixture as mx
from tests.test_gpu_choice import DT, U, _chain, _check_grad, _logits, _np

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2407_00051_amd as sg  # noqa: E402

LOWEST = float(np.finfo(np.float32).min)


def _check_low(f, x, choice, top, scale, what):
    """As test_gpu_choice's forward check.  ln p adds to its roundings that of x - m, of the scale and of their product: 3 u of
    |ln p|, within the 4 counted there."""
    ref = mx.choice_logprob(_np(x), choice, top, scale)
    H, more = ref["entropy"], _chain(*x.shape, "") - 128
    np.testing.assert_array_equal(f["top_choice"].cpu().numpy(), ref["top_choice"], err_msg=what)
    for k, h in (("logp", H), ("top_logp", H[:, None])):
        masked = np.isneginf(ref[k])
        want = np.where(masked, 0.0, np.maximum(ref[k], LOWEST))
        got = _np(f[k])
        np.testing.assert_array_equal(np.isneginf(got), masked, err_msg=f"{what} {k}")
        tol = U * (170 + more + 4 * h + 4 * np.abs(want))
        err = np.abs(np.where(masked, 0.0, got) - want)
        assert (err <= tol).all(), (what, k, float((err / tol).max()))
    err, tol = np.abs(_np(f["entropy"]) - H), U * (170 + more + 8 * H) * (1 + H)
    assert (err <= tol).all(), (what, "entropy", float((err / tol).max()))


def _low_rows(n, V, dtype, seed):
    """Rows that mix ordinary logits with the type's lowest and largest values, and choices on the lowest.  By turns:
    ordinary ones and a few lowest; two ordinary, two lowest, the others masked; two ordinary, the others lowest; as
    the first with one of the largest value."""
    x = _logits(n, V, dtype, seed)
    low, big = torch.finfo(DT[dtype]).min, torch.finfo(DT[dtype]).max
    at = [0, V // 2, V - 1, V // 3]
    for r in range(n):
        kind = r % 4
        if kind in (1, 2):
            keep = x[r, [1, V - 2]].clone()
            x[r] = float("-inf") if kind == 1 else low
            x[r, [1, V - 2]] = keep
        x[r, at[:3]] = low
        if kind == 3:
            x[r, at[3]] = big
    return x, np.array([at[r // 4 % 3] for r in range(n)])


# every form that a row takes: lanes of a wave, a wave, 256 and 1,024 threads, read twice, and in parts, joined by the last
# of them or by a second launch
LOW = [(8, 7, "f32"), (8, 40, "bf16"), (8, 300, "f32"), (12, 500, "bf16"), (8, 1500, "f32"), (8, 6000, "bf16"), (8, 7000, "f32"),
       (128, 30001, "f32"), (128, 140001, "bf16"), (4, 30001, "f32"), (4, 70001, "bf16"), (24, 70001, "f32")]


@pytest.mark.parametrize("n,V,dtype", LOW)
@pytest.mark.parametrize("scale", [1.0, 0.7, 3.0, 2.0 ** -100])
def test_lowest_values_are_not_masked(gpu_ctx, n, V, dtype, scale):
    """A finite logit, however low, has a finite ln p and takes part in the gradient."""
    top = 5
    print(f"case lowest {n} x {V} {dtype} scale {scale}", flush=True)
    x, choice = _low_rows(n, V, dtype, V)
    c = torch.tensor(choice.astype(np.int32), device="cuda:0")
    f = gpu_ctx.choice_logprob(x, c, top=top, scale=scale)
    gl, gH, gt = torch.ones(n, device="cuda:0"), torch.full((n,), 0.5, device="cuda:0"), torch.full((n, top), 0.25, device="cuda:0")
    d = gpu_ctx.choice_backward(x, f, c, gl, gH, gt, scale=scale)
    torch.cuda.synchronize()
    _check_low(f, x, choice, top, scale, f"lowest {n} x {V}")
    _check_grad(d, x, choice, gl, gH, gt, scale, f"lowest {n} x {V}")
    # no masked value has a gradient, and every choice has its own
    at = torch.tensor(choice, device="cuda:0")
    own = d[torch.arange(n, device="cuda:0"), at].float()
    assert (own >= 0.9 * scale).all() and (d[torch.isneginf(x)] == 0).all()


def test_a_lowest_choice_by_hand(gpu_ctx):
    """Logits (1.5, 0, lowest), choice 2 and a derivative of 1: ln p = the lowest value's, dL/dx = (-p_0, -p_1, 1)."""
    for dtype in ("f32", "bf16"):
        low = torch.finfo(DT[dtype]).min
        x = torch.tensor([[1.5, 0.0, low]], dtype=DT[dtype], device="cuda:0")
        c = torch.tensor([2], dtype=torch.int32, device="cuda:0")
        f = gpu_ctx.choice_logprob(x, c, top=3)
        d = gpu_ctx.choice_backward(x, f, c, torch.ones(1, device="cuda:0"))
        torch.cuda.synchronize()
        p0 = 1 / (1 + np.exp(-1.5))
        assert f["top_choice"].tolist() == [[0, 1, 2]] and abs(f["logp"].item() - low) <= 4 * U * -low
        np.testing.assert_allclose(_np(d)[0], [-p0, p0 - 1, 1.0], rtol=torch.finfo(DT[dtype]).eps / 2 + 200 * U)


@pytest.mark.parametrize("n,V,dtype", [(6, 9, "f32"), (6, 300, "bf16"), (6, 5000, "f32"), (6, 40001, "bf16")])
def test_masked_choice_of_a_nan_row_has_no_gradient(gpu_ctx, n, V, dtype):
    """A row whose results are NaN has a NaN gradient but for its masked choices, whose gradient is 0, the given
    choice among them."""
    print(f"case nan {n} x {V} {dtype}", flush=True)
    x = _logits(n, V, dtype, 5)
    x[:, V // 2] = float("-inf")
    x[1, 0], x[3, V - 1] = float("nan"), float("inf")
    choice = np.array([V // 2, V // 2, 1, V // 2, V - 2, V // 2])
    c = torch.tensor(choice.astype(np.int32), device="cuda:0")
    one = torch.ones(n, device="cuda:0")
    f = gpu_ctx.choice_logprob(x, c, top=2)
    d = gpu_ctx.choice_backward(x, f, c, one, one, torch.ones((n, 2), device="cuda:0"))
    torch.cuda.synchronize()
    nan = torch.tensor([False, True, False, True, False, False], device="cuda:0")
    assert torch.equal(torch.isnan(f["logp"]), nan) and (d[:, V // 2] == 0).all()
    rest = torch.arange(V, device="cuda:0") != V // 2
    assert torch.isnan(d[nan][:, rest]).all() and torch.isfinite(d[~nan]).all()


def test_sizes_beyond_32_bits_are_refused(gpu_ctx):
    """Sizes that the C ABI's 32-bit fields cannot hold are refused, not taken modulo 2^32."""
    if torch.cuda.get_device_properties(0).total_memory < 96 << 30:
        pytest.skip("needs 96 GB")
    over = 1 << 32
    wide = torch.empty((1, over + 8), dtype=torch.bfloat16, device="cuda:0")
    few = torch.zeros((4, 2), dtype=torch.int32, device="cuda:0")
    with pytest.raises(sg.SagipsError):
        gpu_ctx.choice_logprob(wide)
    with pytest.raises(ValueError):
        gpu_ctx.dispatch(wide, {"place": few[:1]})
    with pytest.raises(ValueError):
        gpu_ctx.route(few, over + 8)
    del wide
    many = torch.empty((1, over + 2), dtype=torch.int32, device="cuda:0")
    with pytest.raises(ValueError):
        gpu_ctx.route(many, 4)
    with pytest.raises(ValueError):
        gpu_ctx.combine(torch.empty((over + 2, 1), dtype=torch.bfloat16, device="cuda:0"), {"place": many})
    del many
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,pad", [(37, 3), (37, 8), (1500, 1), (1500, 4), (5000, 5), (40, 24), (20001, 7)])
def test_in_place_gradient_leaves_what_is_between_the_rows(gpu_ctx, V, pad, dtype):
    """Columns behind the choices of a strided buffer keep their bits, also where the gradient is written over the logits."""
    print(f"case in place {V} {dtype} pad {pad}", flush=True)
    x = _logits(6, V, dtype, V, 0.1, pad)
    held = x._base                                         # [6][V + pad]
    assert held.shape == (6, V + pad) and held.data_ptr() == x.data_ptr()
    held[:, V:] = torch.randn((6, pad), device="cuda:0").to(DT[dtype])
    before = held.clone()
    c = torch.arange(6, device="cuda:0", dtype=torch.int32)
    f = gpu_ctx.choice_logprob(x, c, top=2)
    d = gpu_ctx.choice_backward(x, f, c, torch.ones(6, device="cuda:0"), d_top=torch.ones((6, 2), device="cuda:0"))
    gpu_ctx.choice_backward(x, f, c, torch.ones(6, device="cuda:0"), d_top=torch.ones((6, 2), device="cuda:0"), out=x)
    torch.cuda.synchronize()
    assert torch.equal(x, d) and torch.equal(held[:, V:], before[:, V:])
