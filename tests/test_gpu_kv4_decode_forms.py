"""Every form of the decode kernel: block tables of the largest context (four blocks a tile), few and many
query rows, float32 queries, and batches of so many requests that a workgroup has several pieces."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from attention_check import TYPES, attend, cache_of, dev  # noqa: E402

pytestmark = pytest.mark.gpu
WIDE = 32768                  # positions of a block table from which tiles have four blocks


def batch(rng, lens, new, heads, group, dim, page, span, dtype, window=0, out="f16"):
    pages = 24
    cache = cache_of(rng.standard_normal((pages, heads, page, dim)), rng.standard_normal((pages, heads, page, dim)))
    table = np.full((len(lens), -(-span // page)), -1, dtype=np.int32)
    for r, n in enumerate(lens):
        table[r, :-(-n // page)] = rng.integers(0, pages, -(-n // page))
    q = dev(rng.standard_normal((sum(new), heads * group, dim)), torch.float32).to(TYPES[dtype])
    attend(q, cache, table, lens, new, page, window=window, out=out)


LENS = [1, 0, 2, 31, 32, 33, 127, 128, 129, 255, 513, 700, 1025]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("heads,group,dim,page", [(8, 4, 128, 64), (2, 4, 128, 16), (8, 4, 64, 64), (1, 1, 64, 16),
                                                  (2, 2, 256, 32), (1, 4, 256, 16), (1, 3, 128, 32)])
def test_tables_of_the_largest_context(heads, group, dim, page, dtype):
    """Short and empty requests in tables of 32768 positions, whole and windowed."""
    print("largest context", heads, group, dim, page, dtype, flush=True)
    rng = np.random.default_rng(dim + page)
    for window in (0, 100):
        batch(rng, LENS, [1] * len(LENS), heads, group, dim, page, WIDE, dtype, window)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("heads,group,dim,page,new", [
    (1, 4, 128, 64, 1), (1, 4, 64, 16, 1), (1, 4, 256, 64, 1),          # 4 rows
    (2, 4, 128, 16, 2), (1, 7, 256, 32, 1),                             # 8
    (1, 16, 128, 64, 1), (1, 5, 64, 32, 3), (1, 4, 256, 16, 4),         # 16
    (1, 8, 128, 64, 3), (1, 8, 64, 16, 4), (1, 10, 128, 16, 3),         # 32
    (1, 16, 64, 64, 3), (1, 16, 64, 16, 4)])                            # 64
def test_rows_of_every_form(heads, group, dim, page, new, dtype):
    """From 4 to 64 query rows a request and head, float16 and float32, in narrow and wide tables."""
    print("rows", heads, group, dim, page, new, dtype, flush=True)
    rng = np.random.default_rng(dim + group)
    lens = [n for n in LENS if n >= new] + [0]
    for span in (1088, WIDE):
        batch(rng, lens, [new] * len(lens), heads, group, dim, page, span, dtype, out="f32")


@pytest.mark.parametrize("heads,group,dim,page,span", [(8, 4, 128, 64, WIDE), (8, 4, 128, 16, 448), (4, 4, 64, 16, WIDE),
                                                       (4, 2, 256, 64, 448), (4, 2, 256, 32, WIDE)])
def test_more_pieces_than_workgroups(heads, group, dim, page, span):
    """400 requests: each workgroup has several of them, and several heads, one after another."""
    print("many pieces", heads, group, dim, page, span, flush=True)
    rng = np.random.default_rng(dim + span)
    lens = rng.integers(0, 440, 400).tolist()
    batch(rng, lens, [1] * 400, heads, group, dim, page, span, "f16")


def test_many_long_requests():
    """So many positions that tiles have four blocks without a wide table, shares of many units, and pieces
    that pass from one workgroup to the next."""
    print("many long requests", flush=True)
    rng = np.random.default_rng(3)
    lens = rng.integers(900, 2600, 80).tolist()
    batch(rng, lens, [1] * 80, 8, 4, 128, 64, 2624, "f16")
