"""A logit that is no number outside a list that has no mass itself: the remaining mass is held against it, so the loss is none
either."""
import math

import numpy as np
import pytest

from oracle import specs_rows as R
from paper_2506_15733_b200 import binding
from tests import test_gpu_rows as base

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("how", ["two", "one", "one_in_place"])
@pytest.mark.parametrize("rows,V,dtype", [(6, 300, "f32"), (6, 20011, "bf16"), (155, 98403, "f16")])
def test_numbers_that_are_none_outside_a_list_without_mass(rows, V, dtype, how):
    ctx = binding.Context(0)
    g, K = base.rng(91), 8
    x = g.normal(size=(rows, V))
    ids, t, _ = base.make_teacher(g, rows, V, K, 1.0, False, ragged=False)
    t[:5] = -math.inf
    ids[1] = -1                                            # nothing listed at all
    lse = np.full(rows, 8.0, np.float32)
    for r, v in ((0, V // 2), (1, V - 1), (2, 0), (3, V // 3)):
        x[r, v] = math.nan
        ids[r][ids[r] == v] = (v + 1) % V
    x[3] = np.where(np.isnan(x[3]), math.nan, -math.inf)   # ... and nothing else outside of it
    x[3, ids[3]] = 1.0
    logits, x = base.device_rows(x, dtype, 1, 1)
    want = R.distill(x, ids, t, 1.0, lse)
    assert np.isnan(want[0][:4]).all() and np.isnan(want[2][:4]).all() and np.isfinite(want[0][4:]).all()
    got = base.distill(ctx, logits, ids, t, 1.0, lse, None, None, how)
    assert np.isnan(got[0][:4]).all() and np.isnan(got[2][:4]).all()
    base.check_distill(got, want, dtype, 1.0, None, None)
    assert ctx.device_status() == 0
    ctx.close()
