"""Zeros among tiny negative logits, where narrowing an interval of keys ends between the two: both zeros are one number."""
import numpy as np
import pytest
import torch

from oracle import specs_rows as R
from paper_2506_15733_b200 import binding
from tests import test_gpu_rows as base

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    assert c.device_status() == 0, "device status word not clean at the end of the module"
    c.close()


def zeros_and_less(rows, V):
    """The largest logit's key ends in ones, so that halving intervals of keys from there meets that of -0."""
    x = np.full((rows, V), -5.0) - base.rng(81).uniform(0, 1, (rows, V))
    x[:, 4000:5000] = 0.0
    x[:, 4000:5000:2] = -0.0
    x[:, 9000:10500] = -1e-40                            # (subnormal)
    x[:, 7] = np.nextafter(np.float32(2), np.float32(0))
    x[1::2] = x[1::2, ::-1]
    return base.device_rows(x, "f32")


@pytest.mark.parametrize("rows", [1, 3, 40, 200])
@pytest.mark.parametrize("K", [1001, 1002, 1020, 1024])
def test_the_largest_logits_end_among_tiny_negative_ones(ctx, rows, K):
    logits, x = zeros_and_less(rows, 20000)
    base.check_top(ctx, logits, x, K, 1.0)


@pytest.mark.parametrize("rows", [3, 200])
@pytest.mark.parametrize("top_k", [1001, 1020, 1024, 1500])
def test_draws_cut_off_among_tiny_negative_ones(ctx, rows, top_k):
    logits, x = zeros_and_less(rows, 20000)
    u = np.linspace(0.01, 0.9999, rows).astype(np.float32)
    kw = dict(top_k=np.full(rows, top_k, np.int32))
    base.check_sample(base.run_sample(ctx, logits, u, **kw), R.sample(x, u, **kw), x)
