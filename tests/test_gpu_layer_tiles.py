"""The layer products at sizes where each way to run them is the one chosen: 256, 128
and 64 wide tiles, sums in parts, operands copied to whole lines, operands read by
way of registers; dense and grouped, against the same 64-bit forms and bounds (the
products of 64-bit numbers are taken on the GPU here)."""
import pytest
import torch

from tests import layer_util as lu
from tests.gpu_util import device
from tests.test_gpu_layers import case, check_grouped, grouped_case, run_backward, run_forward

# rows, in, out, gated
DENSE = [(2056, 264, 6152, False), (2056, 6152, 130, True), (264, 2056, 6152, False),
         (1544, 264, 4104, True), (130, 4104, 6152, False), (4104, 130, 6152, False),
         (1032, 1032, 1032, False), (2600, 1031, 999, False), (40, 1544, 130, True),
         (520, 130, 1544, False), (5000, 7, 9, False), (9, 5000, 70, True),
         (2050, 2047, 2047, False), (264, 4104, 2600, False),
         (264, 2600, 4104, False), (4104, 264, 2600, False)]
# the ends of the groups, rows after them, in, out, gated
GROUPED = [([0, 700, 700, 1301, 2590, 2600], 30, 520, 4104, False),
           ([0, 1, 1200, 1456, 2600], 0, 4104, 520, True),
           ([0, 600, 1100, 1100, 2056], 300, 130, 6152, True),
           ([0, 257, 514, 1544], 7, 2056, 130, False),
           ([0, 10, 10, 25, 39, 40], 0, 6152, 1544, False),
           ([0, 33, 34, 130], 1, 1031, 999, False)]


def ways(dtype):
    """(side, grouped, tile, parts, copied) of the cases above"""
    out = set()
    for T, K, N, gated in DENSE:
        for side, p in enumerate(lu.plans(T, K, N, dtype, gated, True)):
            out.add((side, False, p[1], p[2] > 1, p[3] > 0))
    for off, left, K, N, gated in GROUPED:
        for side, p in enumerate(lu.plans(off[-1] + left, K, N, dtype, gated, True, len(off) - 1)):
            out.add((side, True, p[1], p[2] > 1, p[3] > 0))
    return out


@pytest.fixture
def on_gpu(monkeypatch):
    monkeypatch.setattr(lu, "ON_GPU", True)


def acts(case_, cases):
    return lu.ACTS[(2 + cases.index(case_)) % 5]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("size", DENSE, ids=str)
def test_dense(size, dtype, on_gpu):
    T, K, N, gated = size
    c = case(T, K, N, dtype, gated, seed=81)
    run_forward(c, acts(size, DENSE), gated, True, True, True)
    run_backward(c, acts(size, DENSE), gated)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("pad,shift", [(8, 8), (1, 0), (5, 3)])
def test_dense_rows_apart(pad, shift, dtype, on_gpu):
    """rows further apart than they are long: whole 16-byte pieces, or none"""
    for T, K, N in [(2056, 264, 4104), (1032, 520, 392)]:
        c = case(T, K, N, dtype, False, seed=82, pad=pad, shift=shift)
        run_forward(c, "gelu", False, True, True, True)
        run_backward(c, "gelu", False)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(lu.DTYPES))
@pytest.mark.parametrize("groups", GROUPED, ids=lambda g: str(g[2:]))
def test_groups(groups, dtype, on_gpu):
    off, left, K, N, gated = groups
    c = grouped_case(off, left, K, N, dtype, gated, seed=83)
    check_grouped(off, left, c, acts(groups, GROUPED), gated)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_offsets_past_32_bits(dtype, on_gpu):
    """rows so far apart that the last of x, of w, of z and of the residual begin past
    2^32 bytes, read and written in place"""
    T, K, N = 300, 72, 264
    step = (1 << 24) // (2 if dtype == "bf16" else 4) + 8
    c = case(T, K, N, dtype, False, seed=84)
    buf = torch.empty((T, step), dtype=lu.DTYPES[dtype], device=device())
    for name, at in (("x", 0), ("w", 128), ("z", 256), ("r", 640), ("dy", 1024)):
        rows, cols = c[name].shape
        buf[:rows, at:at + cols] = c[name]
        c[name] = buf[:rows, at:at + cols]
    run_forward(c, "silu", False, True, True, True, out=buf[:, 1408:1408 + N])
    run_backward(c, "silu", False)
    c = case(T, K, N, dtype, False, seed=85)        # and few rows, the last ones
    for name, at in (("x", 0), ("r", 128)):
        rows, cols = c[name].shape
        buf[:rows, at:at + cols] = c[name]
        c[name] = buf[rows - 9:rows, at:at + cols]
    run_forward(c, "silu", False, True, True, True)


@pytest.mark.parametrize("dtype", list(lu.DTYPES))
def test_the_cases_reach_every_way(dtype):
    """the sizes above still choose each tile for each product (a change of the rule
    that loses one is to bring a size that has it)"""
    got = ways(dtype)
    for side in range(3):
        for grouped in (False, True):
            tiles = {64, 128} if dtype == "fp32" else {64, 128, 256}
            assert tiles <= {w[2] for w in got if w[:2] == (side, grouped)}, (side, grouped)
        assert {False, True} == {w[3] for w in got if w[0] == side and not w[1]}, side
        assert {False, True} == {w[4] for w in got if w[0] == side}, side
    assert {64, 128} <= {w[2] for w in got if w[3]}
