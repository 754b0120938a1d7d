"""Registers of the built kernels of the block-scaled FP8 operators and the
losses, from the code object's own metadata.  None spills: 132 spilled registers
made the product of 16384 x 5120 x 13824 five times as long.  The product's sums
stay out of the accumulation registers, from which every one would have to be
copied first."""
import os
import re
import shutil
import struct
import subprocess

import pytest

from test_gpu_product_tilings import _table

READELF = shutil.which("llvm-readelf") or "/opt/rocm/llvm/bin/llvm-readelf"
NAMES = r"(?:quantize_(?:row|block)128|product_(?:tile|rows)|policy_[a-z]+|pref_[a-z]+)_kernel"


def _notes(lib, tmp):
    """The metadata of every gfx950 code object in the library."""
    for m in re.finditer(rb"__CLANG_OFFLOAD_BUNDLE__", lib):  # magic, count, then (offset, size, triple length, triple)
        at = m.end()
        (n,) = struct.unpack_from("<Q", lib, at)
        at += 8
        for _ in range(n):
            off, size, tl = struct.unpack_from("<QQQ", lib, at)
            triple = lib[at + 24:at + 24 + tl]
            at += 24 + tl
            if b"gfx950" in triple and size:
                path = tmp / ("%d.co" % m.start())
                path.write_bytes(lib[m.start() + off:m.start() + off + size])
                yield subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True, check=True).stdout


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{mangled name: {metadata key: scratch bytes a lane, spilled registers, accumulation registers}}"""
    from paper_2607_24062_amd import acrl
    if not os.path.exists(acrl.LIB_PATH) or not os.path.exists(READELF):
        pytest.skip("no built library or no llvm-readelf")
    with open(acrl.LIB_PATH, "rb") as f:
        lib = f.read()
    got = {}
    for notes in _notes(lib, tmp_path_factory.mktemp("co")):
        for k in re.split(r"\n  - (?=\.agpr_count)", notes):
            name = re.search(r"\.name:\s+(_Z\S*?" + NAMES + r"\S*)", k)
            if name:
                got[name.group(1)] = {key: int(re.search(r"\.%s:\s+(\d+)" % key, k).group(1)) for key in
                                      ("private_segment_fixed_size", "vgpr_spill_count", "sgpr_spill_count", "agpr_count")}
    return got


def _of(kernels, what):
    return {k: v for k, v in kernels.items() if what in k}


def test_every_kernel_is_looked_at(kernels):
    tiles = _of(kernels, "product_tile_kernel")
    table, _, _ = _table()
    for tn, tm, *_ in table:
        assert len(_of(tiles, "Li%dELi%dE" % (tn, tm))) >= 2, (tn, tm)  # bf16 and float32 results
    assert len(tiles) == 2 * len(table) and len(_of(kernels, "product_rows_kernel")) == 4
    for what, n in (("quantize_row128", 2), ("quantize_block128", 2), ("policy_count", 1), ("policy_share", 1),
                    ("policy_sum", 1), ("policy_one", 1), ("policy_main", 4), ("pref_one", 1), ("pref_seq", 6),
                    ("pref_coef", 2)):
        assert len(_of(kernels, what + "_kernel")) == n, what


def test_no_scratch(kernels):
    for key in ("private_segment_fixed_size", "vgpr_spill_count", "sgpr_spill_count"):
        assert {k: v[key] for k, v in kernels.items() if v[key]} == {}


def test_products_sum_in_vector_registers(kernels):
    assert {k for k, v in _of(kernels, "product_").items() if v["agpr_count"]} == set()
