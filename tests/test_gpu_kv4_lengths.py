"""Requests whose lengths are far past their block tables, up to the largest that int32 holds: windows see nothing, and
without one a token sees all that the table holds."""
import numpy as np
import pytest

from attention_check import TYPES, dev
from paper_2607_01127_amd import logbq as L
from test_gpu_tree import ints, step

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

LONGEST = 2**31 - 1


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("dim,page,group,new", [(64, 64, 4, 1), (64, 16, 1, 3), (128, 64, 4, 2), (128, 16, 2, 8), (256, 32, 4, 1),
                                                (64, 64, 4, 12), (128, 64, 4, 40), (256, 16, 2, 30)])
def test_lengths_far_past_the_table(dim, page, group, new, dtype):
    print("lengths", dim, page, group, new, dtype, flush=True)
    span = 4 * page
    q, (buffers, _, _), table, _ = step(dim, [span + 40], [new], 2, group, dim, page, dtype)
    table = dev(table[:, :4])
    masks = dev(np.array([(1 << (i + 1)) - 1 for i in range(new)], dtype=np.uint64).view(np.int64))
    starts = ints([0, new])

    def both(length, window):
        got = []
        for tree in (False, True):
            if tree and 0 < window < 64:
                continue
            out = torch.full(q.shape, 7.0, device=q.device, dtype=TYPES[dtype])
            lse = torch.full(q.shape[:2], 7.0, device=q.device)
            args = (q, buffers, table, ints([length]), starts)
            if tree:
                L.kv4_tree_attention(*args, masks, new, window=window, out=out, lse=lse)
            else:
                L.kv4_attention(*args, new, window=window, out=out, lse=lse)
            got.append((out, lse))
        return got

    # The longest length for which a window still ends in the table's reach, and longer ones.
    for length in (span + new + 2000, 2**30 + 7, LONGEST - 200, LONGEST - 100, LONGEST - 31, LONGEST):
        for window in (1, 31, 64, 65, 130, 1000):
            for out, lse in both(length, window):
                assert not out.any() and torch.isneginf(lse).all()
    want = both(span + new, 0)                     # all of the table is cached, the new tokens lie past it
    assert torch.isfinite(want[0][1]).all()
    for length in (2**30 + 7, LONGEST):
        for (a, b), (out, lse) in zip(both(length, 0), want):
            assert torch.equal(a, out) and torch.equal(b, lse)
        for (a, b), (out, lse) in zip(both(length, length - 1), want):         # a window of nearly all
            assert torch.isfinite(b).all()
