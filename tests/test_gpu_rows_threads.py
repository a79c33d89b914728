"""The row operators called from several host threads at once, each with its own context, stream and vocabulary."""
import threading

import torch
import pytest

from paper_2506_15733_b200 import binding

pytestmark = pytest.mark.gpu
CALLS = 400


def calls_of(V, rows, failures, results, which):
    try:
        ctx = binding.Context(0)
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            gen = torch.Generator(device="cuda:0").manual_seed(V)
            logits = torch.randn((rows, V), generator=gen, device="cuda:0")
            ids, values = torch.empty((rows, 8), dtype=torch.int32, device="cuda:0"), torch.empty((rows, 8), device="cuda:0")
            loss, stats, grad = torch.empty(rows, device="cuda:0"), torch.empty((rows, 3), device="cuda:0"), torch.empty_like(logits)
            ctx.specs_top_logits(logits, ids, values)
            for _ in range(CALLS):
                ctx.specs_distill_step(logits, ids, values, loss, grad)
                ctx.specs_distill_forward(logits, ids, values, loss, stats)
                ctx.specs_distill_backward(logits, ids, values, stats, grad)
        stream.synchronize()
        assert ctx.device_status() == 0
        results[which] = (loss.cpu(), grad.sum(1).cpu())
        ctx.close()
    except Exception as e:                                 # reported by the test's own thread
        failures.append(f"V = {V}: {e!r}")


@pytest.mark.parametrize("sizes", [(150, 49300, 120000), (80, 400000, 480000), (160, 49000, 20000)], ids=str)
def test_threads_with_different_vocabularies(sizes):
    rows, *vocabularies = sizes
    failures, results = [], {}
    threads = [threading.Thread(target=calls_of, args=(V, rows, failures, results, i))
               for i, V in enumerate(vocabularies + vocabularies)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures, failures
    n = len(vocabularies)
    for i in range(n):                                     # the same numbers from both threads that had the same inputs
        for a, b in zip(results[i], results[i + n]):
            assert torch.equal(a, b)
