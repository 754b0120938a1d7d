"""Registers of the built kernels of a decode step's operators, from the code
object's own metadata: none spills or uses scratch memory, and the products sum in
vector registers."""
import os
import re

import pytest

from test_gpu_product_tilings import _table
from test_operator_resources import READELF, _notes

# (scalar registers that do not fit, six of the scan, are kept in lanes of a vector register, not in memory)
KEYS = ("private_segment_fixed_size", "vgpr_spill_count", "agpr_count")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    from paper_2607_24062_amd import acrl
    if not os.path.exists(acrl.LIB_PATH) or not os.path.exists(READELF):
        pytest.skip("no built library or no llvm-readelf")
    with open(acrl.LIB_PATH, "rb") as f:
        lib = f.read()
    got = {}
    for notes in _notes(lib, tmp_path_factory.mktemp("co")):
        for k in re.split(r"\n  - (?=\.agpr_count)", notes):
            name = re.search(r"\.name:\s+(_Z\S*?(?:linear_(?:tile|rows)|moe_[a-z_]+|beam_[a-z]+)_kernel\S*)", k)
            if name:
                got[name.group(1)] = {key: int(re.search(r"\.%s:\s+(\d+)" % key, k).group(1)) for key in KEYS}
    return got


def test_every_kernel_is_looked_at(kernels):
    count = lambda what: sum(what in k for k in kernels)  # noqa: E731
    assert count("linear_tile_kernel") == 2 * len(_table()[0]) and count("linear_rows_kernel") == 4
    # up: three widths, the narrowest of pairs, too; down: the same of two and of three parts, and the narrowest of tiles of
    # two and of four rows
    for what, n in (("moe_logits", 2), ("moe_choose", 3), ("moe_up_kernel", 4), ("moe_up_few", 2), ("moe_down_kernel", 10),
                    ("moe_down_few", 2), ("moe_sum", 2), ("beam_scan", 2), ("beam_pick", 1), ("beam_reorder", 4)):
        assert count(what) == n, what


def test_no_scratch(kernels):
    for key in KEYS:
        assert {k: v[key] for k, v in kernels.items() if v[key]} == {}, key
