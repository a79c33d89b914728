"""Listed entries to which the teacher gives nothing, by values far below the others, against a student that rules them out: such
entries have no part in the loss, however the list is shared out over warps and CTAs."""
import math

import numpy as np
import pytest
import torch

from oracle import specs_rows as R
from paper_2506_15733_b200 import binding
from tests import test_gpu_rows as base

pytestmark = pytest.mark.gpu
LOW = float(np.finfo(np.float32).min)


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    assert c.device_status() == 0, "device status word not clean at the end of the module"
    c.close()


def masked_lists(g, rows, V, K, kept, T):
    """Lists whose entries from ``kept`` on are masked, row by row in other ways, at ids where the student has -inf."""
    x = g.normal(size=(rows, V))
    ids = np.stack([g.permutation(V)[:K] for _ in range(rows)]).astype(np.int32)
    t = -np.sort(-g.normal(size=(rows, K)) * 2, axis=1)
    for r in range(rows):
        x[r, ids[r, kept:]] = -math.inf
        if r % 4 == 0:
            t[r, kept:] = LOW                              # the lowest value, as a mask
        elif r % 4 == 1:
            t[r, kept:] = t[r, 0] - 800 * T                # exp() of it is 0
        elif r % 4 == 2:                                   # ... and 0 only against the largest: 400 T below it, and 800 T
            n = kept + (K - kept) // 2
            t[r, kept:n] = t[r, 0] - 400 * T
            x[r, ids[r, kept:n]] = 1.0
            t[r, n:] = t[r, 0] - 800 * T
        else:                                              # masked all the same, where the student has something to say
            t[r, kept:] = LOW
            x[r, ids[r, kept:]] = 0.5
    return x, ids, t.astype(np.float32)


SHAPES = [(4, 200, 8, 3), (4, 3000, 64, 20), (4, 40003, 8, 3), (4, 40003, 8, 1), (8, 32003, 64, 20), (4, 151936, 64, 20)]


@pytest.mark.parametrize("how", ["two", "one", "one_in_place"])
@pytest.mark.parametrize("T", [1.0, 0.2])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", base.TYPES)
def test_masked_values_of_a_list_without_its_normaliser(ctx, dtype, shape, T, how):
    rows, V, K, kept = shape
    x, ids, t = masked_lists(base.rng(7200 + V + K + kept), rows, V, K, kept, T)
    logits, x = base.device_rows(x, dtype)
    want = R.distill(x, ids, t, T, None)
    assert np.isfinite(want[0]).all()
    base.check_distill(base.distill(ctx, logits, ids, t, T, None, None, None, how), want, dtype, np.float32(T), None, None)


@pytest.mark.parametrize("how", ["two", "one"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_values_of_lists_of_many_long_rows(ctx, dtype, how):
    rows, V, T = 155, 49301 if dtype == "f32" else 98403, 1.0
    x, ids, t = masked_lists(base.rng(7300), rows, V, 64, 20, T)
    logits, x = base.device_rows(x, dtype)
    want = R.distill(x, ids, t, T, None)
    assert np.isfinite(want[0]).all()
    base.check_distill(base.distill(ctx, logits, ids, t, T, None, None, None, how), want, dtype, T, None, None)


@pytest.mark.parametrize("tail", [False, True], ids=["list", "tail"])
@pytest.mark.parametrize("rows,V", [(4, 200), (4, 40003), (155, 98403)])
def test_what_the_teacher_wants_and_the_student_rules_out_is_infinite_all_the_same(ctx, rows, V, tail):
    g, K = base.rng(7400), 8
    x, ids, t = masked_lists(g, rows, V, K, 3, 1.0)
    x[:, :] = np.where(np.isinf(x), 0.25, x)
    for r in range(rows):
        x[r, ids[r, r % 3]] = -math.inf                    # one of the entries that have mass
    lse = (t[:, :3].max(1) + 3.0).astype(np.float32) if tail else None
    logits, x = base.device_rows(x, "bf16")
    want = R.distill(x, ids, t, 1.0, lse)
    assert (want[0] == math.inf).all()
    for how in ("two", "one"):
        base.check_distill(base.distill(ctx, logits, ids, t, 1.0, lse, None, None, how), want, "bf16", 1.0, None, None)


def test_a_student_without_entries(ctx):
    # nothing to say about what the teacher masks out: no loss; about what it wants: infinite
    x = np.full((2, 40003), -math.inf)
    ids = np.arange(0, 40000, 5000, dtype=np.int32)[None].repeat(2, 0)
    t = np.full((2, 8), LOW, np.float32)
    t[0] = -math.inf
    t[1, 5] = 0.0
    logits, x = base.device_rows(x, "f32")
    for how in ("two", "one"):
        loss, _, grad = base.distill(ctx, logits, ids, t, 1.0, None, None, None, how)
        assert loss[0] == 0.0 and loss[1] == math.inf
        assert not grad[0].any() and grad[1, ids[1, 5]] == -1.0 and np.count_nonzero(grad[1]) == 1
