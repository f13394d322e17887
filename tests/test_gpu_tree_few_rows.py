"""Trees of up to 16 query rows, which go by the decode kernel's forms, against float64: contexts past 32768 positions
and batches whose tables are wide (four blocks of positions a tile), and 5 to 16 rows with windows, hidden pages, every
number of channels and type of queries. Bounds as in attention_check."""
import numpy as np
import pytest

from test_gpu_tree import attend, step

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu



@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("dim,page", [(64, 16), (64, 64), (128, 16), (128, 128), (256, 64)])
@pytest.mark.parametrize("new,group", [([1, 1, 1], 4), ([4, 2, 3], 1), ([2, 1, 2], 2), ([1, 0, 1], 3)])
def test_up_to_four_rows_over_long_contexts(new, group, dim, page, dtype):
    print("few rows, long", new, group, dim, page, dtype, flush=True)
    lens = [32801, 45, 1500]
    q, cache, table, masks = step(dim + page, lens, new, 1, group, dim, page, dtype)
    table[0, 7], table[2, 0] = -1, 2**30
    for window in (0, 64, 3000, 32790):
        attend(q, cache, table, lens, new, masks, page, dtype, window=window)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
def test_up_to_four_rows_of_a_large_batch(dim, dtype):
    print("few rows, batch", dim, dtype, flush=True)
    rng = np.random.default_rng(dim)
    new = [int(n) for n in rng.integers(0, 3, 700)]
    new[3] = 2
    lens = [n + int(c) for n, c in zip(new, rng.integers(0, 90, 700))]
    q, cache, table, masks = step(dim, lens, new, 2, 2, dim, 32, dtype)
    wide = np.full((700, 32), -1, dtype=np.int32)           # 1024 positions a request and two heads: 1.4e6
    wide[:, :table.shape[1]] = table
    attend(q, cache, wide, lens, new, masks, 32, dtype)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("dim,page", [(64, 64), (128, 16), (128, 64), (256, 32)])
@pytest.mark.parametrize("new,group", [([16, 9, 1, 0], 1), ([4, 3, 2, 4], 4), ([2, 2, 1, 2], 7), ([1, 1, 1, 1], 16),
                                       ([2, 1, 2, 2], 4), ([8, 5, 1, 0], 1)])
def test_up_to_sixteen_rows(new, group, dim, page, dtype):
    print("few rows", new, group, dim, page, dtype, flush=True)
    lens = [700, 130, 1, 2050]
    q, cache, table, masks = step(dim + page + group, lens, new, 2, group, dim, page, dtype)
    for window in (0, 64, 1000):
        attend(q, cache, table, lens, new, masks, page, dtype, window=window)
    table[0, 1], table[3, 2], table[3, 0] = -1, 2**30, -1
    attend(q, cache, table, lens, new, masks, page, dtype)
    # Whole tables of up to 512 positions are one launch.
    attend(q, cache, table[:, :512 // page], lens, new, masks, page, dtype)
