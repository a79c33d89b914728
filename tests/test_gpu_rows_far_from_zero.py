"""Rows whose logits lie far from 0 in units of the temperature, in an order that raises every thread's running maximum again and
again: sums of exponentials are as good there as anywhere.

Tolerance: EXP of the module next door (its exponents' arguments are products less an offset, rounded once, and the offset's own
rounding is put right at the end); each raise multiplies what was summed before by one exponential and a quotient, 2^-21 together,
and a thread of the longest row here has at most 20 units: 20 * 2^-21 = 1e-5 more."""
import math

import numpy as np
import pytest

from oracle import specs_rows as R
from paper_2506_15733_b200 import binding
from tests import test_gpu_rows as base

pytestmark = pytest.mark.gpu
TOL = base.EXP + 20 * 2.0**-21


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    assert c.device_status() == 0, "device status word not clean at the end of the module"
    c.close()


def climbing(g, rows, V, offset, spread):
    """Ascending, descending and shuffled rows around +-offset; row by row a little off it, so that no rounding is favoured."""
    sign = np.where(np.arange(rows) % 2, 1, -1)[:, None]
    x = np.sort(g.uniform(0, spread, (rows, V)), axis=1) + (offset * g.uniform(0.97, 1.0, (rows, 1)) * sign)
    x[2::3] = g.permuted(x[2::3], axis=1)
    x[1::6] = x[1::6, ::-1]
    return x


CASES = [("f32", 45000.0, 1.0), ("f32", 20000.0, 1.0), ("f32", 3000.0, 0.1), ("f32", 300.0, 1.0), ("f32", 50000.0, 1.0),
         ("f16", 2000.0, 1.0), ("f16", 2000.0, 0.25), ("bf16", 250.0, 0.5), ("bf16", 1000.0, 0.03)]


@pytest.mark.parametrize("dtype,offset,T", CASES)
@pytest.mark.parametrize("tail", [False, True], ids=["list", "tail"])
@pytest.mark.parametrize("rows,V", [(6, 700), (6, 20011), (155, 49301)])
def test_distillation_sums_far_from_zero(ctx, dtype, offset, T, tail, rows, V):
    if rows > 100 and dtype != "f32":
        V *= 2
    g = base.rng(int(offset) + V)
    logits, x = base.device_rows(climbing(g, rows, V, offset, 6 * T), dtype)
    ids, t, lse = base.make_teacher(g, rows, V, 20, T, tail)
    T32 = float(np.float32(T))
    loss, stats, grad, parts = R.distill(x, ids, t, T32, lse)
    for how in ("two", "one"):
        got = base.distill(ctx, logits, ids, t, T32, lse, None, None, how)
        if got[1] is not None:
            assert (np.abs(got[1] - stats) <= TOL * np.abs(stats)).all(), np.abs(got[1] / np.maximum(stats, 1e-30) - 1).max(0)
        q_sum = parts["q"].sum(1)
        tol = 2 * TOL * (1 + q_sum + (parts["ratio"] > 0)) + 2.0**-22 * np.abs(loss)
        assert (np.abs(got[0] - loss) <= tol).all(), np.abs(got[0] - loss).max()
        bits, least = base.BITS[dtype]
        half = 0.5 * np.exp2(np.maximum(np.frexp(grad)[1] - bits, least))
        p, q, ratio = parts["p"], parts["q"], parts["ratio"][:, None]
        tol = (TOL * p * np.maximum(q_sum[:, None], 1.0) + 2 * TOL * p * ratio + 1e-5 * q) / T32 * 1.01 + half
        assert (np.abs(got[2] - grad) <= tol).all(), (np.abs(got[2] - grad) / tol).max()


@pytest.mark.parametrize("dtype,offset", [("f32", 45000.0), ("f32", 20000.0), ("f32", 300.0), ("f16", 2000.0), ("bf16", 250.0)])
@pytest.mark.parametrize("rows,V", [(6, 700), (6, 20011), (200, 9001)])
def test_log_probabilities_far_from_zero(ctx, dtype, offset, rows, V):
    g = base.rng(int(offset) + V + 1)
    logits, x = base.device_rows(climbing(g, rows, V, offset, 6.0), dtype)
    u = g.uniform(0, 1, rows).astype(np.float32)
    tok, lp, _ = base.run_sample(ctx, logits, u)
    for r in range(rows):
        want = x[r, tok[r]] - x[r].max() - math.log(np.exp(x[r] - x[r].max()).sum())
        assert abs(lp[r] - want) <= TOL + 2.0**-23 * abs(want), (r, lp[r], want)


@pytest.mark.parametrize("rows,V", [(6, 20011), (155, 33001)])
def test_log_sum_exps_far_from_zero(ctx, rows, V):
    # as far as a float of that size can show it: the largest logit itself is 0, the others climb towards it from far below
    g = base.rng(V)
    x = climbing(g, rows, V, 300.0, 6.0)
    logits, x = base.device_rows(x, "f32")
    base.check_top(ctx, logits, x, 30, 1.0)
