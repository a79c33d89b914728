"""What ``drafting.distill_loss`` promises torch: tensors that its backward pass needs may not change before it, and nothing is
silently left without a gradient."""
import pytest
import torch

from paper_2506_15733_b200 import binding, drafting

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def parts(ctx, rows=6, V=500, K=9):
    gen = torch.Generator(device="cuda:0").manual_seed(3)
    teacher = torch.randn((rows, V), generator=gen, device="cuda:0")
    logits = torch.randn((rows, V), generator=gen, device="cuda:0", requires_grad=True)
    return logits, drafting.teacher_lists(ctx, teacher, K), torch.rand(rows, generator=gen, device="cuda:0") + 0.5


@pytest.mark.parametrize("changed", ["ids", "values", "lse", "row_weight"])
def test_lists_and_weights_that_change_before_the_backward_pass(ctx, changed):
    logits, lists, weight = parts(ctx)
    loss = drafting.distill_loss(ctx, logits, lists, True, weight).sum()
    (weight if changed == "row_weight" else getattr(lists, changed)).add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    assert logits.grad is None


def test_lists_without_their_normaliser_and_weights(ctx):
    logits, lists, _ = parts(ctx)
    drafting.distill_loss(ctx, logits, lists, False).sum().backward()
    assert torch.isfinite(logits.grad).all() and logits.grad.any()


@pytest.mark.parametrize("wanted", ["values", "lse", "row_weight"])
def test_gradients_that_there_are_none_of(ctx, wanted):
    logits, lists, weight = parts(ctx)
    if wanted == "row_weight":
        weight.requires_grad_()
    else:
        getattr(lists, wanted).requires_grad_()
    with pytest.raises(ValueError, match="no gradient"):
        drafting.distill_loss(ctx, logits, lists, True, weight)
    with torch.no_grad():
        drafting.distill_loss(ctx, logits, lists, True, weight)


def test_a_teacher_of_inference_mode(ctx):
    logits, lists, weight = parts(ctx)
    drafting.distill_loss(ctx, logits, lists, True, weight).sum().backward()
    want, logits.grad = logits.grad, None
    with torch.inference_mode():
        lists = drafting.TeacherLists(lists.ids.clone(), lists.values.clone(), lists.lse.clone(), lists.temperature)
    drafting.distill_loss(ctx, logits, lists, True, weight).sum().backward()
    assert torch.equal(logits.grad, want)
