"""Attention over a paged cache at the ends of what it takes: infinite values, long tails, large caps and scores, many long texts, large pages."""

import numpy as np
import pytest

import paper_2504_08860_amd as H
from test_operators_paged import INF, Batch, agree, cache_of
from test_operators_q4 import TINY, TYPES, UNIT, dtype


# Kernels: few rows, in pages of whole eights and of others; many rows, 128 and (a table with room for many positions) 256 a workgroup.
KERNELS = [dict(new=2, page=16), dict(new=2, page=5), dict(new=50, page=16), dict(new=200, page=16, kv_heads=2, wide=2048)]


@pytest.mark.gpu
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("dim", [8, 40, 64, 80, 96, 128, 136, 192, 256])
def test_infinite_values_that_all_rows_see(name, dim):
    """An infinite value in each eight positions of a step of 32 that some rows see more of, in columns of every quarter of a head: that column is infinite, all others are what they were."""
    import torch
    for how in KERNELS:
        new, page, kv_heads, wide = how["new"], how["page"], how.get("kv_heads", 1), how.get("wide", 0)
        b = Batch([(new, 94 + new)], name, kv_heads, 2, dim, page, seed=dim, wide=wide)     # (positions 64..93 are seen by all rows, 94 and 95 by some)
        want, off = b.reference()
        values = b.values.clone()
        for turn in range(4):
            columns = [(1, dim // 3, dim // 2 + 1, dim - 1)[(k + turn) % 4] for k in range(4)]
            signs = [INF, -INF, INF, -INF]
            (at, place) = b.slots(0, np.array([65, 73, 81, 89]))
            for k in range(4):
                b.values[int(at[k]), :, int(place[k]), columns[k]] = signs[k]
            print(f"[infinite values] {name} dim {dim} {how} turn {turn}", flush=True)
            got = b.attend()
            b.values.copy_(values)
            for k in range(4):
                assert (got[..., columns[k]] == signs[k]).all(), f"{how}: column {columns[k]}, eight {k}"
                got[..., columns[k]] = torch.from_numpy(want[..., columns[k]]).to(got)
            agree(got, want, off + UNIT[name] * np.abs(want), f"{how} turn {turn}")
