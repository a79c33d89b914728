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
