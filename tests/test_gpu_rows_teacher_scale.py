"""Teachers' logits that are large in units of the temperature: t / T and the log-sum-exp next to it are taken apart in 64 bits, so q
is as good as for small ones.  Tolerances: the module's next door (1e-5 on q, EXP on sums)."""
import numpy as np
import pytest

from oracle import specs_rows as R
from paper_2506_15733_b200 import binding
from tests import test_gpu_rows as base

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("how", ["two", "one"])
@pytest.mark.parametrize("tail", [False, True], ids=["list", "tail"])
@pytest.mark.parametrize("T", [0.03, 0.07, 0.3, 1.7])
@pytest.mark.parametrize("rows,V,dtype", [(6, 300, "f32"), (6, 40003, "f32"), (155, 49301, "f32"), (6, 700, "bf16")])
def test_teachers_far_from_zero(rows, V, dtype, T, tail, how):
    ctx = binding.Context(0)
    g, K = base.rng(97), 30
    T = float(np.float32(T))
    x = g.normal(size=(rows, V)) * T
    ids, _, _ = base.make_teacher(g, rows, V, K, T, False, ragged=False)
    t = (g.normal(size=(rows, K)) * 2 * T + np.linspace(-3000, 3000, rows)[:, None] * T).astype(np.float32)
    lse = None
    if tail:
        s = t.astype(np.float64) / T
        lse = (s.max(1) + np.log(np.exp(s - s.max(1, keepdims=True)).sum(1)) + g.uniform(0.05, 0.5, rows)).astype(np.float32)
    logits, x = base.device_rows(x, dtype)
    want = R.distill(x, ids, t, T, lse)
    base.check_distill(base.distill(ctx, logits, ids, t, T, lse, None, None, how), want, dtype, T, None, None)
    assert ctx.device_status() == 0
    ctx.close()
