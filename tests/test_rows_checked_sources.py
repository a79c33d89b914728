"""Every kernel source of the row operators has index checks for the checked build, and so have the places that index by data."""
import os
import re

import pytest

from paper_2506_15733_b200 import build

PLACES = {
    "sample_rows.cu": ["push_entry", "push_entries", "sort_list", "narrow_list", "search", "add_masses", "sample_rows_kernel",
                       "top_rows_kernel"],
    "top_stream.cu": ["rank_list", "pick_row"],
    "distill_rows.cu": ["mark_listed", "list_sums", "read_slice", "distill_rows_kernel"],
    "distill_stream.cu": ["load_list"],
}


@pytest.mark.parametrize("source", PLACES)
def test_functions_that_index_by_data_check_their_indexes(source):
    with open(os.path.join(build.CSRC, source)) as f:
        text = f.read()
    for name in PLACES[source]:
        # from the function's definition to the brace that closes it in the first column
        found = re.search(r"^(?:template|__device__|__global__|void)[^;{}]*\b%s\([^;{}]*\) \{\n.*?^\}" % name, text, re.M | re.S)
        assert found, (source, name)
        assert "SPECS_IN_BOUNDS" in found.group(0), (source, name)
