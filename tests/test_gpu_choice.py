"""GPU parity of the choices (log probabilities, entropy, alternatives) and of their gradient
against the float64 oracle, through the C ABI.

Tolerances count roundings in units of u = 2^-24.  A row's sum s is formed by a thread's
chain of at most 128 additions (of more for rows beyond 256 KiB, whose chains are counted below),
six exchanges in the wave and 16 across waves: at most 160 u of s, plus the exponents' own
roundings, 4 u |d| each, weighted by p: 4 u H at most, plus 4 u for exp and log themselves.  So
  ln p:  u (170 + 4 H + 4 |ln p|) absolute,
  H:     the same for ln s, and 170 u of T = sum p |d| <= H: u (170 + 8 H) (1 + H),
  the gradient: 4 more than ln p's relative error on every p, u (180 + 4 H + 4 |ln p|) of the
         sum of its absolute terms (|ln p| is at most 60 where p matters), and half a step of the
         output's type."""
import numpy as np
import pytest

from oracle import mixture as mx

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2407_00051_amd as sg  # noqa: E402

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _logits(n, V, dtype, seed, masked=0.0, pad=0, spread=3.0):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    x = (spread * torch.randn((n, V + pad), generator=g, device="cuda:0")).to(DT[dtype])
    if masked:
        x[torch.rand((n, V + pad), generator=g, device="cuda:0") < masked] = float("-inf")
    return x[:, :V]


def _np(t):
    return t.detach().cpu().double().numpy()


def _chain(n, V, dtype):
    """Additions in a thread's chain (see above)."""
    return 128 + max(0, V - 65536) // 1024


def _check_forward(f, x, choice, top, scale, what):
    ref = mx.choice_logprob(_np(x), choice, top, scale)
    H, more = ref["entropy"], _chain(*x.shape, "") - 128
    np.testing.assert_array_equal(f["top_choice"].cpu().numpy(), ref["top_choice"], err_msg=what)
    for k, rows in (("logp", H), ("top_logp", H[:, None])):
        if ref[k] is None:
            continue
        got, on = _np(f[k]), np.isfinite(ref[k])
        np.testing.assert_array_equal(got[~on], ref[k][~on], err_msg=what)
        tol = U * (170 + more + 4 * rows + 4 * np.where(on, np.abs(np.where(on, ref[k], 0.0)), 0.0))
        err = np.abs(np.where(on, got, 0.0) - np.where(on, ref[k], 0.0))
        assert (err <= tol).all(), (what, k, float((err / tol).max()))
    err, tol = np.abs(_np(f["entropy"]) - H), U * (170 + more + 8 * H) * (1 + H)
    assert (err <= tol).all(), (what, "entropy", float((err / tol).max()))


def _check_grad(got, x, choice, gl, gH, gt, scale, what):
    f64 = lambda t: None if t is None else _np(t)     # noqa: E731
    ref, terms = mx.choice_backward(_np(x), choice, f64(gl), f64(gH), f64(gt), scale, with_terms=True)
    H = mx.choice_logprob(_np(x), None, 0, scale)["entropy"][:, None]
    half = torch.finfo(got.dtype).eps / 2
    tol = half * np.abs(ref) + (1 + half) * U * (180 + 240 + 4 * H) * terms + 2.0 ** -126
    err = np.abs(_np(got) - ref)
    assert (err <= tol).all(), (what, float((err / tol).max()))


# one choice, and both ends of every form that a row takes: 1 to 64 units of 16 bytes, a wave, 256 and
# 1,024 threads, and rows that are read twice; rows that begin on any value
SIZES = [1, 2, 3, 4, 5, 8, 9, 15, 17, 33, 64, 65, 127, 129, 255, 257, 500, 513, 1000, 1025, 2049, 4097, 8191, 16385, 32769,
         65537, 131073, 140001]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", SIZES)
def test_forward_and_gradient_match_oracle(gpu_ctx, V, dtype):
    n = 1 if V > 100000 else 2 if V > 20000 else 5
    for pad, top, scale, masked in ((0, min(V, 3), 1.0, 0.0), (3, min(V, 32), 0.7, 0.4)):
        what = f"choice {n} x {V} {dtype} pad {pad} top {top}"
        print("case", what, flush=True)
        x = _logits(n, V, dtype, V + pad, masked, pad)
        choice = (np.arange(n) * 7 + 1) % V
        choice[n // 2] = -1 if n > 2 else choice[n // 2]
        c = torch.tensor(choice.astype(np.int32), device="cuda:0")
        f = gpu_ctx.choice_logprob(x, c, top=top, scale=scale)
        torch.cuda.synchronize()
        _check_forward(f, x, choice, top, scale, what)
        g = torch.Generator(device="cuda:0").manual_seed(V)
        gl, gH = (torch.randn(n, generator=g, device="cuda:0") for _ in range(2))
        gt = torch.randn((n, top), generator=g, device="cuda:0")
        d = gpu_ctx.choice_backward(x, f, c, gl, gH, gt, scale=scale)
        torch.cuda.synchronize()
        assert d.dtype == x.dtype and d.shape == x.shape
        _check_grad(d, x, choice, gl, gH, gt, scale, what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,V", [(4099, 8), (70001, 3), (1025, 300), (300, 5000)])
def test_many_rows(gpu_ctx, n, V, dtype):
    print(f"case choice rows {n} x {V} {dtype}", flush=True)
    x = _logits(n, V, dtype, n)
    choice = np.arange(n) % V
    c = torch.tensor(choice.astype(np.int32), device="cuda:0")
    f = gpu_ctx.choice_logprob(x, c, top=2)
    d = gpu_ctx.choice_backward(x, f, c, d_logp=torch.ones(n, device="cuda:0"))
    torch.cuda.synchronize()
    _check_forward(f, x, choice, 2, 1.0, f"{n} x {V}")
    some = np.random.default_rng(0).choice(n, 64, replace=False)
    _check_grad(d[some], x[some], choice[some], torch.ones(64), None, None, 1.0, f"{n} x {V}")


@pytest.mark.parametrize("V", [1, 7, 64, 700, 20000, 150000])
def test_masked_rows(gpu_ctx, V):
    """Rows of nothing, of one choice, of the type's lowest value, of equal values, and masked choices."""
    inf, low = float("-inf"), torch.finfo(torch.float32).min
    x = torch.full((5, V), inf, device="cuda:0")
    x[1, V // 2] = -3.0
    x[2] = low
    x[3] = 1.5
    x[4, 0] = low
    choice = np.array([0, V // 2, V - 1, V // 3, V - 1])
    c = torch.tensor(choice.astype(np.int32), device="cuda:0")
    top = 4
    f = gpu_ctx.choice_logprob(x, c, top=top)
    one = torch.ones(5, device="cuda:0")
    d = gpu_ctx.choice_backward(x, f, c, one, one, torch.ones((5, top), device="cuda:0"))
    torch.cuda.synchronize()
    _check_forward(f, x, choice, top, 1.0, f"masked {V}")
    _check_grad(d, x, choice, one, one, torch.ones((5, top)), 1.0, f"masked {V}")
    assert torch.equal(d[0], torch.zeros_like(d[0])) and (f["top_choice"][0] == -1).all()
    assert f["logp"][1].item() == 0.0 and f["entropy"][:2].tolist() == [0.0, 0.0]


@pytest.mark.parametrize("V", [5, 300, 9000, 140000])
def test_nan_stays_in_its_row(gpu_ctx, V):
    x = _logits(4, V, "f32", 3)
    x[1, V - 1] = float("nan")
    x[2, 0] = float("inf")
    c = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    f = gpu_ctx.choice_logprob(x, c, top=2)
    one = torch.ones(4, device="cuda:0")
    d = gpu_ctx.choice_backward(x, f, c, one, one)
    torch.cuda.synchronize()
    for k in ("logp", "entropy", "top_logp"):
        assert torch.isnan(f[k][1:3]).all() and not torch.isnan(f[k][[0, 3]]).any(), k
    assert (f["top_choice"][1:3] == -1).all() and (f["top_choice"][[0, 3]] >= 0).all()
    assert torch.isnan(d[1:3]).all() and not torch.isnan(d[[0, 3]]).any()


@pytest.mark.parametrize("n,V", [(3, 4000), (2, 33000), (1, 300000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_alternatives_that_one_thread_holds(gpu_ctx, n, V, dtype):
    """Rows whose largest values recur with the period of a thread's reads, and falling and rising rows."""
    i = torch.arange(V, device="cuda:0")
    N = 4 if dtype == "f32" else 8
    rows = [torch.where(i % (N * 1024) < N, 5.0, 0.0), torch.where(i % (N * 64) < N, 5.0, 0.0), -i / V, i / V]
    for k, row in enumerate(rows):
        x = row.to(DT[dtype])[None].repeat(n, 1)
        print(f"case held {n} x {V} {dtype} pattern {k}", flush=True)
        f = gpu_ctx.choice_logprob(x, top=32)
        torch.cuda.synchronize()
        _check_forward(f, x, None, 32, 1.0, f"pattern {k}")


@pytest.mark.parametrize("n,V,dtype", [(16, 9001, "f32"), (17, 9001, "f32"), (40, 20011, "bf16"), (127, 17001, "bf16"),
                                       (128, 17001, "bf16"), (20, 70001, "f32"), (1, 600011, "bf16")])
def test_few_long_rows(gpu_ctx, n, V, dtype):
    """Rows in parts, joined by the last part or by a second launch, and the first number of rows that are not."""
    print(f"case parts {n} x {V} {dtype}", flush=True)
    x = _logits(n, V, dtype, V, 0.2, 1)
    x[n // 2] = 1.5                                       # equal alternatives in every part
    x[n // 2, 5] = float("-inf")
    x[n - 1, 70:] = float("-inf") if n > 1 else 0.25      # parts of nothing
    choice = (np.arange(n) * 11 + 3) % V
    c = torch.tensor(choice.astype(np.int32), device="cuda:0")
    f = gpu_ctx.choice_logprob(x, c, top=32, scale=0.9)
    again = gpu_ctx.choice_logprob(x, c, top=32, scale=0.9)
    torch.cuda.synchronize()
    _check_forward(f, x, choice, 32, 0.9, f"parts {n} x {V}")
    assert all(torch.equal(f[k], again[k]) for k in f)


def test_more_contexts_than_counters(gpu_ctx):
    """Contexts beyond the 64 that have counters join the parts in a second launch, with the same bits."""
    print("case 70 contexts", flush=True)
    x = _logits(2, 30001, "f32", 5)
    c = torch.tensor([1, 30000], dtype=torch.int32, device="cuda:0")
    want = gpu_ctx.choice_logprob(x, c, top=20)
    many = [sg.Context(0) for _ in range(70)]
    for ctx in many:
        f = ctx.choice_logprob(x, c, top=20)
        assert all(torch.equal(f[k], want[k]) for k in f)
    for ctx in many:
        ctx.close()


def test_parts_in_a_graph(gpu_ctx):
    """Rows in parts captured and replayed, with eager calls of the context between: the counters are left as found."""
    print("case parts captured", flush=True)
    x = _logits(3, 40001, "bf16", 6)
    c = torch.tensor([7, 0, 40000], dtype=torch.int32, device="cuda:0")
    want = gpu_ctx.choice_logprob(x, c, top=9)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        ctx = sg.Context(0, stream=st)
        ctx.choice_logprob(x, c, top=9)                   # makes the workspace, outside the capture
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st, capture_error_mode="relaxed"):
            out = ctx.choice_logprob(x, c, top=9)
        for _ in range(3):
            for t in out.values():
                t.fill_(-2)
            eager = ctx.choice_logprob(x, c, top=9)
            graph.replay()
            st.synchronize()
            assert all(torch.equal(out[k], want[k]) and torch.equal(eager[k], want[k]) for k in want)
        ctx.close()


@pytest.mark.parametrize("n,V,dtype,top,opad", [(40003, 525, "bf16", 4, 0), (40003, 200, "f32", 5, 0), (5000, 2300, "f32", 7, 1),
                                                (4300000, 300, "bf16", 2, 1)])
def test_more_rows_than_a_launch_has_groups(gpu_ctx, n, V, dtype, top, opad):
    """Workgroups that take several rows, forward, and several chunks of rows in the gradient (the last case)."""
    if n > 10 ** 6 and torch.cuda.get_device_properties(0).total_memory < 64 << 30:
        pytest.skip("needs 64 GB")
    print(f"case {n} x {V} {dtype}", flush=True)
    x = _logits(n, V, dtype, n, 0.1)
    c = torch.randint(0, V, (n,), device="cuda:0", dtype=torch.int32)
    gl, gH, gt = torch.ones(n, device="cuda:0"), torch.full((n,), 0.3, device="cuda:0"), torch.ones((n, top), device="cuda:0")
    f = gpu_ctx.choice_logprob(x, c, top=top)
    out = torch.empty((n, V + opad), dtype=x.dtype, device="cuda:0")[:, :V]
    d = gpu_ctx.choice_backward(x, f, c, gl, gH, gt, out=out)
    torch.cuda.synchronize()
    some = np.unique(np.concatenate([np.arange(40), np.random.default_rng(1).choice(n, 60), np.arange(n - 40, n)]))
    part = {k: v[torch.tensor(some, device="cuda:0")] for k, v in f.items()}
    choice = c.cpu().numpy()[some]
    _check_forward(part, x[some], choice, top, 1.0, f"{n} x {V}")
    _check_grad(d[some], x[some], choice, gl[some], gH[some], gt[some], 1.0, f"{n} x {V}")


def test_gradient_in_place_strided_and_of_other_alignment(gpu_ctx):
    for dtype in ("f32", "bf16"):
        for V, pad, opad in ((37, 3, 0), (37, 0, 5), (1500, 4, 4), (5000, 1, 2), (40, 24, 8)):
            print(f"case grad {V} {dtype} {pad} {opad}", flush=True)
            x = _logits(6, V, dtype, V, 0.1, pad)
            choice = np.array([0, V - 1, 3, -5, V, 2])
            c = torch.tensor(choice.astype(np.int32), device="cuda:0")
            gl, gt = torch.randn(6, device="cuda:0"), torch.randn((6, 2), device="cuda:0")
            f = gpu_ctx.choice_logprob(x, c, top=2, scale=1.3)
            held = torch.full((6, V + opad), 7.0, dtype=DT[dtype], device="cuda:0")
            d = gpu_ctx.choice_backward(x, f, c, gl, None, gt, scale=1.3, out=held[:, :V])
            torch.cuda.synchronize()
            _check_grad(d, x, choice, gl, None, gt, 1.3, f"{V} {dtype}")
            assert (held[:, V:] == 7.0).all()                      # what lies between the rows stays
            before = _np(x)
            same = gpu_ctx.choice_backward(x, f, c, gl, None, gt, scale=1.3, out=x)
            torch.cuda.synchronize()
            assert same.data_ptr() == x.data_ptr() and torch.equal(same, d)
            assert np.isfinite(before[0, 0]) or np.isneginf(before[0, 0])


def test_choice_that_is_also_an_alternative(gpu_ctx):
    """The same index twice: both parts of the gradient arrive."""
    for V in (6, 900, 30000):
        x = _logits(3, V, "f32", V)
        best = x.argmax(1).to(torch.int32)
        gl, gt = torch.tensor([1.0, -2.0, 0.5], device="cuda:0"), torch.randn((3, 3), device="cuda:0")
        f = gpu_ctx.choice_logprob(x, best, top=3)
        d = gpu_ctx.choice_backward(x, f, best, gl, None, gt)
        torch.cuda.synchronize()
        _check_grad(d, x, best.cpu().numpy(), gl, None, gt, 1.0, f"twice {V}")


def test_gradient_against_differences(gpu_ctx):
    """A small distribution's whole gradient against central differences of the kernel's own
    results: step h = 2^-6 gives (h^2 / 6) |f'''| <= 5e-5 |g| of truncation and 2 u (1 + |f|) / h of rounding."""
    x = torch.tensor([[0.5, -1.0, 0.25, 1.5]], device="cuda:0")
    c, h = torch.tensor([2], dtype=torch.int32, device="cuda:0"), 2.0 ** -6
    f = gpu_ctx.choice_logprob(x, c, top=1)
    d = gpu_ctx.choice_backward(x, f, c, torch.tensor([1.0], device="cuda:0"), torch.tensor([0.5], device="cuda:0"),
                                torch.tensor([[2.0]], device="cuda:0"))
    value = lambda y: (lambda o: o["logp"][0].double() + 0.5 * o["entropy"][0].double() + 2.0 * o["top_logp"][0, 0].double())(  # noqa: E731
        gpu_ctx.choice_logprob(y, c, top=1))
    for v in range(4):
        e = torch.zeros_like(x)
        e[0, v] = h
        num = (value(x + e) - value(x - e)) / (2 * h)
        assert abs(num.item() - d[0, v].item()) < 3.5 * 5e-5 + 170 * 2 * U * 4 / h, v


def test_long_strides_pass_32_bits(gpu_ctx):
    """Rows more than 2^31 values apart in all: 3 rows of stride 2^30 + 8 bf16 values (6.4 GB)."""
    if torch.cuda.get_device_properties(0).total_memory < 32 << 30:
        pytest.skip("needs 32 GB")
    stride, V = (1 << 30) + 8, 100
    held = torch.empty(2 * stride + V, dtype=torch.bfloat16, device="cuda:0")
    x = held.as_strided((3, V), (stride, 1))
    x.copy_(_logits(3, V, "bf16", 9))
    c = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda:0")
    f = gpu_ctx.choice_logprob(x, c, top=2)
    d = gpu_ctx.choice_backward(x, f, c, torch.ones(3, device="cuda:0"), out=x.clone())
    torch.cuda.synchronize()
    _check_forward(f, x, np.array([1, 2, 3]), 2, 1.0, "strides")
    _check_grad(d, x, np.array([1, 2, 3]), torch.ones(3), None, None, 1.0, "strides")


def test_refusals(gpu_ctx):
    x = _logits(3, 10, "f32", 1)
    c = torch.zeros(3, dtype=torch.int32, device="cuda:0")
    f = gpu_ctx.choice_logprob(x, c, top=2)
    one = torch.ones(3, device="cuda:0")
    with pytest.raises(ValueError):
        gpu_ctx.choice_logprob(x, c, top=33)
    with pytest.raises(sg.SagipsError):
        gpu_ctx.choice_logprob(x, c, scale=0.0)
    with pytest.raises(TypeError):
        gpu_ctx.choice_logprob(x.half(), c)
    with pytest.raises(TypeError):
        gpu_ctx.choice_logprob(x, c.long())
    with pytest.raises(ValueError):
        gpu_ctx.choice_logprob(x.t(), c)
    with pytest.raises(ValueError):
        gpu_ctx.choice_logprob(x.cpu(), None)
    with pytest.raises(ValueError):
        gpu_ctx.choice_logprob(x[:, :0], None)
    with pytest.raises(sg.SagipsError):
        gpu_ctx.choice_backward(x, f, c)                            # nothing to differentiate
    with pytest.raises(ValueError):
        gpu_ctx.choice_backward(x, gpu_ctx.choice_logprob(x), None, one)
    with pytest.raises(ValueError):
        gpu_ctx.choice_backward(x, f, c, one, out=x[:, :5])
    held = torch.zeros(40, device="cuda:0")
    y = held[:30].view(3, 10)
    with pytest.raises(sg.SagipsError):
        gpu_ctx.choice_backward(y, f, c, one, out=held[1:31].view(3, 10))
