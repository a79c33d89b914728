"""Lists without a normaliser whose values are all the lowest there are: their softmax is that of equal numbers, however low."""
import numpy as np
import pytest

from oracle import specs_rows as R
from paper_2506_15733_b200 import binding
from tests import test_gpu_rows as base

pytestmark = pytest.mark.gpu
LOW = np.finfo(np.float32).min


@pytest.mark.parametrize("how", ["two", "one", "one_in_place"])
@pytest.mark.parametrize("T", [1.0, 19.5, 0.2])
@pytest.mark.parametrize("rows,V,dtype", [(4, 1, "f32"), (6, 300, "f16"), (6, 40003, "bf16"), (155, 98403, "bf16")])
def test_a_list_of_lowest_values_is_a_list_of_equals(rows, V, dtype, T, how):
    ctx = binding.Context(0)
    g, K = base.rng(95), 9
    x = g.normal(size=(rows, V))
    ids, t, _ = base.make_teacher(g, rows, V, K, 1.0, False)
    t[:, :] = LOW
    t[1::4] = -1e30
    t[2::4] = 1e25
    t[3::4] = g.normal(size=(len(t[3::4]), K))
    logits, x = base.device_rows(x, dtype, 1, 1)
    T = float(np.float32(T))
    want = R.distill(x, ids, t, T, None)
    some = (ids >= 0).any(1)
    assert np.abs(want[3]["q"].sum(1) - some).max() < 1e-12
    base.check_distill(base.distill(ctx, logits, ids, t, T, None, None, None, how), want, dtype, T, None, None)
    assert ctx.device_status() == 0
    ctx.close()
