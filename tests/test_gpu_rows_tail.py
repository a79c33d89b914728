"""The remaining mass of a teacher's list (q_r) against a student that gives what is not listed very little: probabilities
p_r far below the range of a float, in the loss, its gradient and the statistics between the two passes.

Tolerances, from the arithmetic and not from a run.  EXP is the module's next door: a sum of exponentials to 3e-5.
  * loss: 2 EXP on the listed terms; ln p_r is a gap of |ln p_r| whose factor 1 / T is rounded to a float (2^-24), plus the
    EXP of a sum each in rest and total; the loss itself is a float.
  * gradient of an unlisted entry: p S to EXP, and q_r p / p_r to 2 EXP plus, between the two passes, the rounding of ln rest to
    a float (2^-24 |ln rest|, and as much again where the backward pass takes it apart).  Powers below 2^-126 are 0.
  * gradient of a listed entry: EXP on p S, 1e-5 on q.
  * stats: EXP on a sum; where a logarithm stands for it, EXP and 2^-23 of itself.
"""
import math

import numpy as np
import pytest
import torch

from oracle import specs_rows as R
from paper_2506_15733_b200 import binding
from tests import test_gpu_rows as base

pytestmark = pytest.mark.gpu
EXP, TYPES, INF = base.EXP, base.TYPES, math.inf
FLT_MIN = 2.0**-126


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    assert c.device_status() == 0, "device status word not clean at the end of the module"
    c.close()


def sure_rows(g, rows, V, K, gap, T):
    """Rows whose listed logits lie ``gap`` T above all the others, in several forms; lists without repeats but for one row."""
    half = gap * T / 2
    x = g.normal(size=(rows, V)) * 0.5 * T - half
    ids = np.stack([g.permutation(V)[:K] for _ in range(rows)]).astype(np.int32)
    for r in range(rows):
        x[r, ids[r]] = half + g.normal(size=K) * 0.5 * T
        if r % 5 == 1:                                     # as many largest ones as there can be, all alike
            x[r, ids[r]] = half
        if r % 5 == 2:                                     # one unlisted entry nearly alone, the others much further down
            x[r] = np.where(x[r] > 0, x[r], -half - 20 * T)
            x[r, (ids[r, 0] + 1) % V if (ids[r, 0] + 1) % V not in ids[r] else np.setdiff1d(np.arange(V), ids[r])[0]] = -half
        if r % 5 == 3:                                     # an ordinary row among them
            x[r] = g.normal(size=V) * 2
        if r % 5 == 4:                                     # an id that is listed twice
            ids[r, 1] = ids[r, 0]
            x[r] = np.where(np.isin(np.arange(V), ids[r]), x[r], -half - np.abs(g.normal(size=V)))
    t = (g.normal(size=(rows, K)) * T).astype(np.float32)
    s = t / T
    lse = (np.log(np.exp(s).sum(1)) + g.uniform(0.1, 0.6, rows)).astype(np.float32)
    return x, ids, t, lse


def check(ctx, logits, x, ids, t, T, lse, how, dtype):
    rows, V = x.shape
    T32 = float(np.float32(T))
    w = np.linspace(0.5, 2, rows).astype(np.float32)
    loss, stats, grad, parts = R.distill(x, ids, t, T, lse, w)
    got = base.distill(ctx, logits, ids, t, T, lse, w, None, how)
    p, q, ratio = parts["p"], parts["q"], parts["ratio"]
    on = np.zeros((rows, V), dtype=bool)
    for r in range(rows):
        on[r, ids[r][ids[r] >= 0]] = True
    q_sum = q.sum(1)
    q_r = np.maximum(0, 1 - q_sum) if lse is not None else np.zeros(rows)
    # the gap by the definition, without an exponential that could underflow
    hidden = np.where(on, -INF, x).max(1)
    gap = np.where(hidden > -INF, (x.max(1) - hidden) / T32, 0.0)
    assert np.isfinite(loss).all() and np.isfinite(grad).all()
    tol = w * (2 * EXP * (1 + q_sum) + q_r * (2 * EXP + 2.0**-23 * gap)) + 2.0**-22 * np.abs(loss)
    bad = ~(np.abs(got[0] - loss) <= tol)
    assert not bad.any(), ("loss", np.nonzero(bad)[0][:5], loss[bad][:5], got[0][bad][:5])
    if got[1] is not None and lse is not None:
        rest, third = stats[:, 2], got[1][:, 2].astype(np.float64)
        with np.errstate(divide="ignore", invalid="ignore"):
            fine = np.where(rest >= FLT_MIN, np.abs(third - rest) <= EXP * rest,
                            (third < 0) & (np.abs(third - np.log(rest)) <= EXP + 2.0**-23 * np.abs(np.log(rest))))
        assert fine.all(), ("stats", rest[~fine][:5], third[~fine][:5])
    scale = (w / T32)[:, None]
    S = np.maximum(q_sum + q_r, 1.0)[:, None]
    bits, least = base.BITS[dtype]
    half = 0.5 * np.exp2(np.maximum(np.frexp(grad)[1] - bits, least))
    tail = np.where(on, 0.0, p * ratio[:, None])           # q_r p_v / p_r
    tol = scale * (EXP * p * S + tail * (2 * EXP + 2.0**-22 * gap[:, None]) + 1e-5 * q + FLT_MIN * (S + 1)) * 1.01 + half
    bad = ~(np.abs(got[2] - grad) <= tol)
    at = np.argwhere(bad)
    assert not bad.any(), ("grad", len(at), at[:5], grad[bad][:5], got[2][bad][:5])


GAPS = [60.0, 80.0, 86.5, 87.2, 88.0, 95.0, 110.0, 400.0, 680.0]


@pytest.mark.parametrize("how", ["two", "one", "one_in_place"])
@pytest.mark.parametrize("tail", [False, True], ids=["list", "tail"])
@pytest.mark.parametrize("T", [1.0, 0.2])
@pytest.mark.parametrize("shape", [(5, 200, 12, 0, 0), (10, 1500, 64, 3, 1), (5, 20011, 64, 5, 2)], ids=str)
@pytest.mark.parametrize("dtype", TYPES)
def test_the_remaining_mass_of_a_sure_student(ctx, dtype, shape, T, tail, how):
    rows, V, K, pad, shift = shape
    for i, gap in enumerate(GAPS):
        x, ids, t, lse = sure_rows(base.rng(7000 + 10 * V + i), rows, V, K, gap, T)
        logits, x = base.device_rows(x, dtype, pad, shift)
        check(ctx, logits, x, ids, t, T, lse if tail else None, how, dtype)


@pytest.mark.parametrize("how", ["two", "one", "one_in_place"])
@pytest.mark.parametrize("dtype,pad,shift", [("f32", 3, 1), ("bf16", 0, 0), ("f16", 1, 2)])
def test_the_remaining_mass_of_a_sure_student_among_long_rows(ctx, dtype, pad, shift, how):
    # the kernel that keeps one CTA on an SM; every row has another gap
    rows, V, K = (155, 49301, 64) if dtype == "f32" else (155, 98403, 64)
    for T in (1.0, 0.2):
        g = base.rng(7100)
        x, ids, t, lse = sure_rows(g, rows, V, K, 1.0, T)
        for r in range(rows):
            if r % 5 != 3:
                gap = (GAPS + [87.0, 500.0])[r % 11]
                on = np.isin(np.arange(V), ids[r])
                x[r] = np.where(on, x[r] + (gap - 1) * T / 2, x[r] - (gap - 1) * T / 2)
        ids[7, :4], ids[8, :3] = [0, 1, V - 1, V - 2], [V - 3, 2, 3]      # entries of the row's partial units
        for r in (7, 8):
            ids[r, 4:] = 50 + np.arange(60) * 7
            x[r] = -20.0 * T
            x[r, ids[r]] = 75.0 * T
        logits, x = base.device_rows(x, dtype, pad, shift)
        check(ctx, logits, x, ids, t, T, lse, how, dtype)


@pytest.mark.parametrize("how", ["two", "one"])
def test_the_worked_examples(ctx, how):
    # 12 listed at 60, 188 at -28: the loss has a tail of about 88 q_r; 12 at 60, one at -27.2 and the others at -100: finite
    ids = np.arange(12, dtype=np.int32)[None].repeat(2, 0)
    x = np.full((2, 200), -28.0)
    x[1, 12], x[1, 13:] = -27.2, -100.0
    x[:, :12] = 60.0
    t = np.zeros((2, 12), np.float32)
    lse = np.full(2, math.log(12) + 0.3, np.float32)
    for dtype in TYPES:
        logits, y = base.device_rows(x, dtype)
        check(ctx, logits, y, ids, t, 1.0, lse, how, dtype)
        got = base.distill(ctx, logits, ids, t, 1.0, lse, None, None, how)
        assert (got[0] > 20.0).all()


@pytest.mark.parametrize("how", ["two", "one"])
def test_what_lies_beyond_the_limit_has_no_mass(ctx, how):
    # more than 690 T below the largest: as if it were masked by -inf
    for dtype in TYPES:
        low = float(torch.finfo(TYPES[dtype]).min)
        x = np.full((3, 3000), -INF)
        x[1], x[2] = low, -700.0
        x[:, :9] = 0.0
        ids = np.arange(9, dtype=np.int32)[None].repeat(3, 0)
        t = base.rng(71).normal(size=(1, 9)).repeat(3, 0).astype(np.float32)
        lse = np.full(3, 4.0, np.float32)
        logits, _ = base.device_rows(x, dtype)
        loss, stats, grad = base.distill(ctx, logits, ids, t, 1.0, lse, None, None, how)
        assert np.isfinite(loss).all() and loss[0] == loss[1] == loss[2]
        assert np.array_equal(grad[0], grad[1]) and np.array_equal(grad[0], grad[2]) and not grad[:, 9:].any()
        assert stats is None or not stats[:, 2].any()
