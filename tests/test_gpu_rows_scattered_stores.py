"""The streaming distillation kernel where its stores are slow: rows of the gradient that lie differently on 16-byte boundaries than
those of the logits are written element by element, while the stages that the logits come through are filled again.  The numbers
have to be those of the gradient that lies alike, bit for bit, in every repetition."""
import pytest
import torch

from paper_2506_15733_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=str)
@pytest.mark.parametrize("offset", [1, 5])
def test_gradients_do_not_depend_on_how_their_rows_lie(dtype, offset):
    ctx = binding.Context(0)
    rows, V, K = 460, 98403 if dtype != torch.float32 else 50021, 70
    gen = torch.Generator(device="cuda:0").manual_seed(offset)
    logits = (torch.randn((rows, V), generator=gen, device="cuda:0") * 2).to(dtype)
    ids = torch.randint(0, V, (rows, K), generator=gen, device="cuda:0", dtype=torch.int32)
    ids[::3] = torch.randint(0, V - K, (len(ids[::3]), 1), generator=gen, device="cuda:0", dtype=torch.int32) + \
        torch.arange(K, device="cuda:0", dtype=torch.int32)              # side by side
    values = torch.randn((rows, K), generator=gen, device="cuda:0")
    loss, stats = torch.empty(rows, device="cuda:0"), torch.empty((rows, 3), device="cuda:0")
    want, want_two = torch.empty_like(logits), torch.empty_like(logits)  # lie like the logits
    ctx.specs_distill_step(logits, ids, values, loss, want)
    ctx.specs_distill_forward(logits, ids, values, loss, stats)
    ctx.specs_distill_backward(logits, ids, values, stats, want_two)
    room = torch.empty((rows, V + 8), dtype=dtype, device="cuda:0")
    grad = room[:, offset:offset + V]
    for _ in range(6):
        grad.fill_(7)
        ctx.specs_distill_step(logits, ids, values, loss, grad)
        assert torch.equal(grad, want)
        grad.fill_(7)
        ctx.specs_distill_backward(logits, ids, values, stats, grad)
        assert torch.equal(grad, want_two)
    assert ctx.device_status() == 0
    ctx.close()
