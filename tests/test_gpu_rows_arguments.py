"""Arguments of the row operators that cannot be right: refused before anything is written."""
import pytest
import torch

from paper_2506_15733_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    assert c.device_status() == 0
    c.close()


def test_lists_and_statistics_of_another_pitch(ctx):
    dev = "cuda:0"
    x = torch.randn((4, 100), device=dev)
    ids, val = torch.full((4, 3), 5, dtype=torch.int32, device=dev), torch.zeros((4, 3), device=dev)
    loss, stats, grad = torch.full((4,), 5.0, device=dev), torch.zeros((4, 3), device=dev), torch.full_like(x, 5.0)
    for bad in (torch.zeros((4, 6), device=dev), torch.zeros((6, 2), device=dev), torch.zeros((3, 4), device=dev),
                torch.zeros((4, 3, 1), device=dev)):
        for call in (lambda: ctx.specs_top_logits(x, ids, bad), lambda: ctx.specs_distill_forward(x, ids, bad, loss),
                     lambda: ctx.specs_distill_backward(x, ids, bad, stats, grad),
                     lambda: ctx.specs_distill_step(x, ids, bad, loss, grad),
                     lambda: ctx.specs_distill_forward(x, ids, val, loss, bad),
                     lambda: ctx.specs_distill_backward(x, ids, val, bad, grad)):
            with pytest.raises(ValueError):
                call()
    torch.cuda.synchronize()
    assert (ids == 5).all() and (loss == 5).all() and (grad == 5).all() and not val.any() and not stats.any()
    # the right pitch: exact, with room behind the rows, or flat
    room = torch.zeros((9, 3), device=dev)
    ctx.specs_distill_forward(x, ids, room, loss, room.clone())
    ctx.specs_distill_forward(x, ids, val.view(-1), loss, stats.view(-1))


@pytest.mark.parametrize("T", [1e-45, 1e-40, 2.9e-39, 4e-39])
def test_temperatures_whose_inverse_is_no_float(ctx, T):
    dev = "cuda:0"
    x = torch.randn((4, 100), device=dev)
    ids, val = torch.full((4, 3), 5, dtype=torch.int32, device=dev), torch.zeros((4, 3), device=dev)
    loss, stats, grad = torch.full((4,), 5.0, device=dev), torch.ones((4, 3), device=dev), torch.full_like(x, 5.0)
    for call in (lambda: ctx.specs_top_logits(x, ids, val, temperature=T),
                 lambda: ctx.specs_distill_forward(x, ids, val, loss, temperature=T),
                 lambda: ctx.specs_distill_backward(x, ids, val, stats, grad, temperature=T),
                 lambda: ctx.specs_distill_step(x, ids, val, loss, grad, temperature=T)):
        with pytest.raises(binding.SpecsError) as e:
            call()
        assert e.value.status == 2
    torch.cuda.synchronize()
    assert (ids == 5).all() and (loss == 5).all() and (grad == 5).all()


def test_the_smallest_temperatures_that_are_taken(ctx):
    # all the mass on the largest logit, and finite numbers
    dev, T = "cuda:0", 1e-38
    x = torch.randn((4, 5000), device=dev) * 0.5
    x[:, 123] = 2.5
    ids, val, lse = torch.empty((4, 3), dtype=torch.int32, device=dev), torch.empty((4, 3), device=dev), torch.empty(4, device=dev)
    loss, grad = torch.empty(4, device=dev), torch.empty_like(x)
    ctx.specs_top_logits(x, ids, val, lse, temperature=T)
    assert (ids[:, 0] == 123).all() and ((lse / 2.5e38 - 1).abs() < 1e-6).all()
    ctx.specs_distill_step(x, ids, val, loss, grad, temperature=T)
    assert (loss == 0).all() and not grad.any()
