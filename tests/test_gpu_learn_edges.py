"""Ends of the ranges that the losses accept, against the float64 oracle.

Tolerances are those of test_gpu_learn, whose derivation holds here too unless a test says otherwise."""
import numpy as np
import pytest

import oracle
from tests.parity import to_np
from tests.test_gpu_learn import ADV_TOL, _t

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


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
