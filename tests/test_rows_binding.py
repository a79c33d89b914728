"""Sizes on their way into the C interface's 32-bit arguments."""
import ctypes

import torch

from paper_2506_15733_b200 import binding


def test_sizes_beyond_32_bits_do_not_turn_into_small_ones():
    wide = torch.empty((1, 2**32 + 100), dtype=torch.bfloat16, device="meta")
    _, _, stride, rows, V = binding.rows_arg(wide, wide.get_device(), "logits")
    assert (stride, rows) == (2**32 + 100, 1)
    assert ctypes.c_int32(V).value == V > binding.MAX_ROW_VOCAB            # refused, and not taken for 100 entries
    K = binding._list_length(torch.empty((1, 2**32 + 3), dtype=torch.int32, device="meta"), "top_ids")
    assert ctypes.c_int32(K).value == K > binding.MAX_TOP_LOGITS
    ordinary = torch.empty((3, 1000), dtype=torch.float32, device="meta")
    assert binding.rows_arg(ordinary, ordinary.get_device(), "logits")[2:] == (1000, 3, 1000)
