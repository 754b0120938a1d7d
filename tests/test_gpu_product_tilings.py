"""acrl_matmul_fp8 by each of its tilings, over rows long enough that the scales
of a tile pass through LDS in several parts: a kernel holds those of C blocks of
K at a time, in two places that it fills in turn.  ceil(K / 128) from C + 1 on
reads the second place, from 2 C + 1 on the first one again.

The choice of the tiling is evaluated on the host, from the table that
csrc/product.hip chooses by, so that other constants or another tiling there
cannot leave one without such a case."""
import os
import re

import numpy as np
import pytest

from gpu_util import torch_dev
from operators64 import e4m3_values

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# (outputs, tokens of a tile): sizes M, N that choose it, and C
TILINGS = {(32, 32): (19, 70, 32), (64, 32): (33, 4641, 16), (64, 64): (67, 5460, 16), (128, 64): (131, 5470, 8),
           (128, 128): (259, 6557, 8), (256, 128): (519, 7190, 8), (256, 256): (1029, 7213, 8)}


def _lengths(C):
    """K of C + 1, 2 C + 1, 2 C + 2 and 3 C + 2 blocks, the last one whole or cut."""
    return (128 * C + 32, 256 * C + 96, 256 * C + 192, 128 * (3 * C + 2))


CASES = [(tile, M, N, K) for tile, (M, N, C) in TILINGS.items() for K in _lengths(C)]


def _table():
    """[(outputs, tokens, K groups, us a turn, us a round, C)] of csrc/product.hip."""
    with open(os.path.join(ROOT, "paper_2607_24062_amd", "csrc", "product.hip")) as f:
        src = f.read()
    body = re.search(r"variants\[\] = \{(.*?)\};", src, re.S).group(1)
    rows = re.findall(r"\{(\d+), (\d+), (\d+), ([\d.]+)f, ([\d.]+)f,\s*launch_tiles<OUT, (\d+), (\d+), \d+, \d+, (\d+), \d+, (\d+), "
                      r"(?:true|false)>\}", body)
    assert len(rows) == body.count("launch_tiles") >= 1
    got = []
    for tn, tm, kg, turn, rnd, tn2, tm2, kg2, C in rows:
        assert (tn, tm, kg) == (tn2, tm2, kg2)
        got.append((int(tn), int(tm), int(kg), np.float32(turn), np.float32(rnd), int(C)))
    cus = int(re.search(r"constexpr int kCus = (\d+);", src).group(1))
    few = int(re.search(r"if \(p\.M <= (\d+)\) return", src).group(1))
    return got, cus, few


def _choice(table, cus, M, N, K):
    kb = -(-K // 128)
    cost = [np.float32(-(-(-(-N // tn) * -(-M // tm)) // cus)) * (np.float32(-(-kb // kg)) * turn + rnd)
            for tn, tm, kg, turn, rnd, _ in table]
    return table[int(np.argmin(cost))]


def _uncovered(cases):
    """{(outputs, tokens): what no case (M, N, K) of it shows}"""
    table, cus, few = _table()
    blocks = {row[:2]: [] for row in table}
    for M, N, K in cases:
        if M > few:
            blocks[_choice(table, cus, M, N, K)[:2]].append(K)
    lacks = {}
    for tn, tm, _, _, _, C in table:
        second = [K for K in blocks[tn, tm] if C < -(-K // 128) <= 2 * C]
        again = [K for K in blocks[tn, tm] if -(-K // 128) > 2 * C]
        miss = [what for what, ok in (("second place", second), ("first place again", again),
                                      ("cut block", any(K % 128 for K in again))) if not ok]
        if miss:
            lacks[tn, tm] = miss
    return lacks


def test_every_tiling_has_its_long_rows():
    assert _uncovered([case[1:] for case in CASES]) == {}
    table, cus, _ = _table()
    for tile, M, N, K in CASES:
        assert _choice(table, cus, M, N, K)[:2] == tile, (tile, M, N, K)
    # a list without them is seen to lack them
    short = [(M, N, K) for _, M, N, K in CASES if K < 1024]
    assert set(_uncovered(short)) == {row[:2] for row in table}


@pytest.mark.gpu
@pytest.mark.parametrize("tile,M,N,K", CASES)
def test_long_rows(tile, M, N, K):
    # codes of whole numbers -2 .. 2, scales 2^-2 .. 2^2: every sum stays below K 2^10 units of 2^-4, K <= 12544, and so
    # is exact in fp32 in any order
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    val, kb = e4m3_values(), -(-K // 128)
    codes = torch.tensor([int(np.flatnonzero(val == v)[0]) for v in range(-2, 3)], dtype=torch.uint8, device=dev)
    g = torch.Generator(device=dev).manual_seed(M + N + K)
    rand = lambda top, *shape: torch.randint(top, shape, generator=g, device=dev)  # noqa: E731
    nx, nw = rand(5, M, K), rand(5, N, K)
    ex, ew = rand(5, M, kb), rand(5, -(-N // 128), kb)
    xs, ws = torch.exp2(ex.float() - 2), torch.exp2(ew.float() - 2)
    spread = lambda e, rows, tile: (e.double() - 2).exp2().repeat_interleave(128, 1)[:, :K].repeat_interleave(tile, 0)[:rows]  # noqa: E731
    x = (nx - 2).double() * spread(ex, M, 1)
    w = (nw - 2).double() * spread(ew, N, 128)
    want = x @ w.t().contiguous()
    for dtype in (torch.float32, torch.bfloat16):
        y = acrl.acrl_matmul_fp8(codes[nx], xs, codes[nw], ws, out_dtype=dtype)
        assert torch.equal(y, want.float().to(dtype)), dtype
