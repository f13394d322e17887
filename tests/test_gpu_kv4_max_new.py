"""Requests with more tokens than the call's bound says: the first max_new are answered, for the others
nothing is written."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from attention_check import attend, cache_of, dev  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group,dim", [(4, 128), (1, 64), (16, 64), (3, 256)])
@pytest.mark.parametrize("new,lens,bounds", [
    ([2], [300], [1]), ([2, 1, 3], [300, 64, 90], [1, 2]), ([9, 1, 40], [100, 33, 41], [1, 3, 8, 20]),
    ([200, 1, 70], [333, 128, 70], [1, 2, 17, 69, 199]), ([130], [130], [1, 64, 129]),
    ([5, 4], [3, 0], [1, 2, 4]), ([2, 2], [7000, 5], [1])])
def test_tokens_past_the_bound_are_left_out(new, lens, bounds, group, dim):
    print("max_new", new, lens, group, dim, flush=True)
    rng = np.random.default_rng(sum(lens) + dim)
    heads, page, pages = 2, 64, 6
    cache = cache_of(*(rng.standard_normal((pages, heads, page, dim)) for _ in range(2)))
    table = rng.integers(0, pages, (len(new), max(1, -(-max(lens) // page)))).astype(np.int32)
    q = dev(rng.standard_normal((sum(new), heads * group, dim)), torch.float32).half()
    index = np.concatenate([np.arange(n) for n in new])           # of a token in its request
    for most in bounds:
        for window in (0, 50):
            answered = index < most
            rows = np.repeat(answered[:, None], heads * group, 1)
            res, lse = attend(q, cache, table, lens, new, page, window=window, max_new=most, rows=rows)
            left = torch.from_numpy(~answered).cuda()
            assert bool(torch.isnan(res[left]).all()) and bool((lse[left] == 7).all())
