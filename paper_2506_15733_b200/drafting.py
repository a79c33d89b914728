"""What stands on either side of scoring: how a draft model writes the blocks that are scored, and how it is trained
to write blocks that the target keeps.

  draft_blocks     the candidate blocks of one step, token by token, with ``specs_sample_tokens``: ids, offsets, and the
                   generator's own log-probabilities, as ``specs_beam_step`` takes them (``loop.DraftBatch``)
  teacher_lists    the target's logits as their K largest and the log-sum-exp (``specs_top_logits``)
  distill_loss     the divergence of the draft's logits from such lists as a differentiable torch function
                   (``specs_distill_forward`` / ``specs_distill_backward``)

Marshalling only: every number is computed by the kernels.  A training step whose loss weights are known beforehand needs
neither the autograd graph nor a second read of the logits: ``Context.specs_distill_step`` gives loss and gradient in one
pass, and may write the gradient over the logits.
"""
from __future__ import annotations

from typing import Callable, NamedTuple, Optional

import torch

from . import binding


class DraftedBlocks(NamedTuple):
    """Blocks of equal length, block by block: what ``specs_beam_step`` takes of the generator."""
    token_ids: torch.Tensor          # int32 [blocks * length]
    block_offsets: torch.Tensor      # int64 [blocks + 1]
    gen_tok_logprob: torch.Tensor    # float32 [blocks * length]: log pi of the draft itself (temperature 1, all entries)
    draw_logprob: torch.Tensor       # float32 [blocks * length]: under the distribution that was drawn from


def draft_blocks(ctx: "binding.Context", next_logits: Callable[[int, Optional[torch.Tensor]], torch.Tensor], blocks: int,
                 length: int, uniforms: torch.Tensor, temperature=None, top_k=None, top_p=None,
                 min_p=None) -> DraftedBlocks:
    """Drafts ``blocks`` candidate blocks of ``length`` tokens in step.  ``next_logits(t, ids)`` returns the draft's logits
    [blocks, V] for token t, given the ids drawn for token t - 1 (int32 [blocks]; None for t = 0); ``uniforms`` float32
    [length, blocks] are the random numbers.  The settings are those of ``specs_sample_tokens``, per block."""
    dev = f"cuda:{ctx.device}"
    if tuple(uniforms.shape) != (length, blocks):
        raise ValueError(f"uniforms: expected [{length}, {blocks}], got {tuple(uniforms.shape)}")
    ids = torch.empty((length, blocks), dtype=torch.int32, device=dev)
    own, drawn = (torch.empty((length, blocks), dtype=torch.float32, device=dev) for _ in range(2))
    for t in range(length):
        logits = next_logits(t, ids[t - 1] if t else None)
        if logits.shape[0] != blocks:
            raise ValueError(f"next_logits: expected {blocks} rows, got {logits.shape[0]}")
        ctx.specs_sample_tokens(logits, uniforms[t], ids[t], own[t], drawn[t], temperature=temperature, top_k=top_k,
                                top_p=top_p, min_p=min_p)
    offsets = torch.arange(blocks + 1, dtype=torch.int64, device=dev) * length
    block_major = [x.t().contiguous().view(-1) for x in (ids, own, drawn)]
    return DraftedBlocks(block_major[0], offsets, block_major[1], block_major[2])


class TeacherLists(NamedTuple):
    ids: torch.Tensor                # int32 [rows, K]
    values: torch.Tensor             # float32 [rows, K]
    lse: torch.Tensor                # float32 [rows], at `temperature`
    temperature: float


def teacher_lists(ctx: "binding.Context", logits: torch.Tensor, K: int, temperature: float = 1.0) -> TeacherLists:
    """What is kept of a teacher's logits [rows, V]: K (id, logit) pairs and one number a row instead of V logits."""
    rows, dev = logits.shape[0], logits.device
    out = TeacherLists(torch.empty((rows, K), dtype=torch.int32, device=dev),
                       torch.empty((rows, K), dtype=torch.float32, device=dev),
                       torch.empty(rows, dtype=torch.float32, device=dev), float(temperature))
    ctx.specs_top_logits(logits, out.ids, out.values, out.lse, temperature=temperature)
    return out


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(fn, logits, ctx, lists, with_rest, row_weight):
        rows, dev = logits.shape[0], logits.device
        loss = torch.empty(rows, dtype=torch.float32, device=dev)
        stats = torch.empty((rows, 3), dtype=torch.float32, device=dev)
        lse = lists.lse if with_rest else None
        ctx.specs_distill_forward(logits, lists.ids, lists.values, loss, stats, temperature=lists.temperature,
                                  top_lse=lse, row_weight=row_weight)
        # torch watches over what it saves; tensors of inference mode (a teacher's, often) it does not save
        given = (lists.ids, lists.values, lse, row_weight)
        watched = [t is not None and not t.is_inference() for t in given]
        fn.save_for_backward(logits, stats, *(t if w else None for t, w in zip(given, watched)))
        fn.rest = (ctx, lists.temperature, [None if w else t for t, w in zip(given, watched)])
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(fn, grad_loss):
        logits, stats, *watched = fn.saved_tensors
        ctx, temperature, others = fn.rest
        ids, values, lse, row_weight = (o if w is None else w for w, o in zip(watched, others))
        grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        ctx.specs_distill_backward(logits, ids, values, stats, grad, temperature=temperature, top_lse=lse,
                                   row_weight=row_weight, grad_loss=grad_loss.float().contiguous())
        return grad, None, None, None, None


def distill_loss(ctx: "binding.Context", logits: torch.Tensor, lists: TeacherLists, with_rest: bool = True,
                 row_weight: Optional[torch.Tensor] = None) -> torch.Tensor:
    """float32 [rows]: the divergence of softmax(logits / T) from the teacher's lists, differentiable with respect to
    ``logits``.  ``with_rest``: the mass that a list leaves out is one more outcome; otherwise the lists are normalised by
    themselves.  Neither the logits nor the lists and weights may be changed between the forward and the backward pass
    (torch checks).  There is no gradient with respect to lists and weights: what requires one is refused."""
    if torch.is_grad_enabled():
        for name, t in (("lists.values", lists.values), ("lists.lse", lists.lse if with_rest else None),
                        ("row_weight", row_weight)):
            if t is not None and t.requires_grad:
                raise ValueError(f"{name} requires a gradient, and there is no gradient with respect to it: detach it")
    return _DistillLoss.apply(logits, ctx, lists, with_rest, row_weight)
