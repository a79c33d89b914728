"""Draws from long rows in batches that are shared out over the SMs in other ways: the tokens are those that a row draws alone."""
import pytest
import torch

from paper_2506_15733_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [74, 75, 148, 149, 222, 223, 296, 297])
@pytest.mark.parametrize("V", [127990, 128256])
def test_tokens_do_not_depend_on_how_many_rows_there_are(rows, V):
    ctx = binding.Context(0)
    gen = torch.Generator(device="cuda:0").manual_seed(rows)
    logits = (torch.randn((rows, V), generator=gen, device="cuda:0") * 2).bfloat16()
    u = torch.rand(rows, generator=gen, device="cuda:0")
    greedy = torch.arange(rows, device="cuda:0") % 5 == 0
    kw = dict(temperature=torch.where(greedy, 0.0, 1.2), top_p=torch.rand(rows, generator=gen, device="cuda:0"),
              top_k=torch.randint(-1000, 2000, (rows,), generator=gen, device="cuda:0", dtype=torch.int32))
    many = torch.empty(rows, dtype=torch.int32, device="cuda:0")
    ctx.specs_sample_tokens(logits, u, many, **kw)
    for r in list(range(0, rows, 7)) + [rows - 1]:
        one = torch.empty(1, dtype=torch.int32, device="cuda:0")
        ctx.specs_sample_tokens(logits[r:r + 1], u[r:r + 1], one, **{k: v[r:r + 1] for k, v in kw.items()})
        assert one[0] == many[r]
    assert ctx.device_status() == 0
    ctx.close()
