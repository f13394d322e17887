"""Attention over a cache that holds scales that are no numbers."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from attention_check import attend, cache_of, dev  # noqa: E402

pytestmark = pytest.mark.gpu
CALLS = [([3, 2], [330, 200]), ([150], [330]), ([70, 1, 90], [330, 64, 129])]


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (256, 32)])
def test_scales_that_are_no_numbers(dim, page, bad, which):
    """A position whose scale is NaN or infinite (a cache that was filled by other means): rows that do not
    see it, for causality or their window, are right; a NaN makes those that see it NaN."""
    print("no numbers", dim, page, bad, which, flush=True)
    rng = np.random.default_rng(dim)
    heads, pages, group = 1, 24, 2
    k, v = (rng.standard_normal((pages, heads, page, dim)) for _ in range(2))
    for new, lens in CALLS:
        for window in (0, 40):
            table = np.stack([rng.permutation(24) for _ in new]).astype(np.int32)[:, :-(-330 // page)]
            buffers, kv, vv = cache_of(k, v)
            starts = np.concatenate([[0], np.cumsum(new)])
            sees = np.zeros((sum(new), heads * group), dtype=bool)
            at = lens[0] - 1 - new[0] // 2                 # in the middle of the first request's new tokens
            page_id = int(table[0, at // page])
            (buffers.k_scales if which == "k" else buffers.v_scales)[page_id, :, at % page] = bad
            for r, (n, length) in enumerate(zip(new, lens)):
                held = np.flatnonzero(table[r] == page_id)
                for i in range(n):
                    p = length - n + i
                    for j in held * page + at % page:
                        if j <= p and (not window or j > p - window):
                            sees[starts[r] + i] = True
            assert sees.any() and not sees.all()
            q = dev(rng.standard_normal((sum(new), heads * group, dim)), torch.float32).half()
            res, lse = attend(q, (buffers, kv, vv), table, lens, new, page, window=window, rows=~sees)
            seen = torch.from_numpy(sees).cuda()
            if math.isnan(bad):
                assert bool(torch.isnan(res[seen]).all())
                assert bool(torch.isnan(lse[seen]).all()) == (which == "k")
