"""Every way that a 4-bit product goes by its number of rows, columns and vectors: rows by the ten thousand, which the small matrices of the other tests do not have.
Compared are the first rows, the last ones (a part of a tile) and some between, with sums in 64 bits."""
import numpy as np
import pytest

import paper_2504_08860_amd as H
from test_operators_q4 import TYPES, agree, dtype, some_x, values

pytestmark = pytest.mark.gpu


def check(rows, cols, group, scales, zeros, counts, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes_shape, scales_shape = H.hbp_q4_shapes(rows, cols, group)
    codes = torch.randint(0, 256, codes_shape, dtype=torch.uint8, generator=g, device="cuda")
    s = (0.02 * (0.5 + torch.rand(scales_shape, generator=g, device="cuda"))).to(dtype(scales))
    z = torch.randint(4, 12, scales_shape, generator=g, device="cuda").to(dtype(scales)) if zeros else None
    some = torch.cat([torch.arange(40), torch.arange(rows // 2, min(rows // 2 + 80, rows)), torch.arange(max(rows - 70, 0), rows)])
    w = values(codes[some], s[some], None if z is None else z[some], cols, group)
    for name, vectors in counts:
        print(f"[q4 shapes] {rows} x {cols} group {group} {scales} zeros {zeros} {vectors} of {name}", flush=True)
        x = some_x(vectors, cols, name, seed)
        y = torch.full((vectors, rows), float("nan"), dtype=x.dtype, device="cuda")
        H.hbp_q4_mv(codes, s, x.cuda(), y, group=group, zeros=z)
        assert not torch.isnan(y).any()
        agree(y[:, some], x.double().numpy() @ w.T, x, name, what=f"{vectors} of {name}")


GROUPS = [32, 64, 128, 256, 512]


@pytest.mark.parametrize("scales", TYPES)
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", GROUPS)
def test_up_to_four_vectors_and_rows_for_every_wavefront(group, scales, zeros):
    """x in LDS as a whole, each wavefront through tiles by itself: from 65521 rows on"""
    for rows, cols in ((65_521, 100), (65_550, 1000), (131_071, 33), (70_003, 2049)):
        check(rows, cols, group, scales, zeros, [("bf16", 1), ("f16", 4), ("f32", 1), ("f16", 2), ("bf16", 3)], rows + group)


@pytest.mark.parametrize("zeros", [False, True])
def test_as_much_of_x_as_that_way_takes(zeros):
    """more than 64 KB of LDS for x, and one column more than it takes"""
    for cols, counts in ((8192, [("f16", 4), ("f32", 1)]), (8193, [("bf16", 4), ("bf16", 1)]), (7, [("f32", 1), ("bf16", 4)])):
        check(65_530, cols, 128, "f16", zeros, counts, cols)


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", GROUPS)
def test_up_to_four_vectors_and_fewer_rows(group, zeros):
    """one or two wavefronts over the rows, four or eight in all, two or four chunks of 128 columns at a time, one step or several"""
    for k, (rows, cols) in enumerate(((8200, 300), (8200, 1000), (9001, 2000), (8200, 4000), (8195, 8300), (500, 3000), (500, 20000), (100, 1500))):
        check(rows, cols, group, TYPES[(k + group) % 3], zeros, [("bf16", 1), ("f16", 4), ("f32", 1)], k + group)


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("rows,cols", [(8192, 1300), (8193, 900), (32_752, 500), (32_753, 500), (40_001, 1301)])
def test_five_to_sixteen_slots(rows, cols, group, zeros):
    """eight wavefronts over the columns up to 8192 rows, four by two beyond, four over the rows from 32753 on"""
    check(rows, cols, group, TYPES[(rows + group // 32) % 3], zeros, [("bf16", 5), ("f16", 16), ("f32", 2), ("f32", 5), ("bf16", 12)], rows + group)


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("scales", TYPES)
@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("rows", [16_368, 16_369, 20_011])
def test_more_slots(rows, group, scales, zeros):
    """two, three and four sets of sixteen; from 16369 rows on eight wavefronts over the rows, each with two tiles where there are two or three sets; more than one pass"""
    counts = [("bf16", 17), ("f16", 32), ("bf16", 33), ("f16", 48), ("bf16", 49), ("f16", 64), ("bf16", 70), ("f32", 6), ("f32", 10), ("f32", 11), ("f32", 16), ("f32", 21), ("f32", 23)]
    check(rows, [300, 1000, 641][rows % 3], group, scales, zeros, counts[:: 2 if rows == 20_011 else 1], rows + group)


@pytest.mark.parametrize("zeros", [False, True])
def test_infinities_where_rows_are_many(zeros):
    """Results that are computed again, in the ways through LDS and through tiles: infinities and NaN of x, and sums that fit where their terms do not."""
    import torch
    rows, cols, group = 65_600, 200, 64
    codes_shape, scales_shape = H.hbp_q4_shapes(rows, cols, group)
    codes = torch.randint(0, 256, codes_shape, dtype=torch.uint8, device="cuda")
    s = torch.full(scales_shape, 0.02, device="cuda")
    z = torch.full(scales_shape, 8.0, device="cuda") if zeros else None
    some = torch.cat([torch.arange(64), torch.arange(rows - 64, rows)])
    w = values(codes[some], s[some], None if z is None else z[some], cols, group)
    for vectors, name in ((1, "bf16"), (4, "f16"), (1, "f32"), (7, "bf16"), (40, "f16"), (20, "f32")):
        print(f"[q4 infinities] {vectors} of {name} zeros {zeros}", flush=True)
        x = some_x(vectors, cols, name, 6)
        y = torch.empty(vectors, rows, dtype=x.dtype, device="cuda")
        for kind in range(3):
            x[0] = 0
            x[0, 77] = [float("inf"), float("nan"), torch.finfo(x.dtype).max / 4][kind]
            H.hbp_q4_mv(codes, s, x.cuda(), y, group=group, zeros=z)
            got, col = y[0, some].cpu().double().numpy(), w[:, 77]
            if kind == 0:
                assert np.array_equal(got, np.where(col > 0, np.inf, np.where(col < 0, -np.inf, np.nan)), equal_nan=True)
            elif kind == 1:
                assert np.isnan(got).all()
            else:
                want = col * float(x[0, 77])
                assert np.isfinite(got).all() and (np.abs(got - want) <= 2.0 ** -7 * np.abs(want)).all()
            if vectors > 1:
                agree(y[1:, some], x[1:].double().numpy() @ w.T, x[1:], name)


@pytest.mark.parametrize("vectors", [1, 5])
def test_more_rows_than_one_launch_takes(vectors):
    check((1 << 26) + 133, 32, 32, "f16", True, [("bf16", vectors)], 1)
