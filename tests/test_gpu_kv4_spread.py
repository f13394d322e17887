"""Attention where the scales of a request's keys span many orders of magnitude: a row's result depends on
what the row sees, in the measure in which it weighs, and on nothing else."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from attention_check import TYPES, attend, cache_of, dev  # noqa: E402

pytestmark = pytest.mark.gpu
CALLS = [([1], [330]), ([3, 2], [330, 200]), ([150], [330]), ([70, 1, 90], [330, 64, 129])]


@pytest.mark.parametrize("power", [8, 14, 20, 24, 30, 60, 100])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (256, 32)])
def test_keys_far_larger_than_the_rest(dim, page, power):
    """A few keys (in the first tile, and in a later one) are 2^power times the others and lie against the
    queries: they get no weight, and the others' logits are as exact as without them."""
    print("large keys", dim, page, power, flush=True)
    rng = np.random.default_rng(dim + power)
    heads, pages = 2, 25
    for places in ([3], [130, 131, 260]):
        k = rng.standard_normal((pages, heads, page, dim))
        table = np.stack([rng.permutation(pages)[:24] for _ in range(3)]).astype(np.int32)[:, :-(-330 // page)]
        for row in table:
            for p in places:
                k[row[p // page], :, p % page] = -(2.0 ** power) * (1 + rng.random(dim))
        cache = cache_of(k, rng.standard_normal(k.shape))
        for new, lens in CALLS:
            q = dev(0.5 + rng.random((sum(new), heads * 2, dim)), torch.float32)
            dtypes = ("f16", "bf16", "f32") if power == 30 else ("f16",)
            for dtype in dtypes:
                attend(q.to(TYPES[dtype]), cache, table[:len(new)], lens, new, page)


@pytest.mark.parametrize("dim,page", [(64, 32), (128, 16), (256, 64)])
def test_keys_of_every_size(dim, page):
    """Each token's keys by a power of two of its own, from 2^-60 to 2^4; and requests whose first half is
    tiny, or whose second half is."""
    print("keys of every size", dim, page, flush=True)
    rng = np.random.default_rng(dim)
    heads, pages = 1, 24
    base = rng.standard_normal((pages, heads, page, dim))
    size = np.exp2(rng.integers(-60, 5, (pages, heads, page, 1)).astype(np.float64))
    half = np.where(np.arange(pages)[:, None, None, None] < 3, 2.0 ** -40, 1.0)
    v = rng.standard_normal(base.shape)
    order = [np.arange(24), np.arange(24)[::-1]]
    for k in (base * size, base * half):
        cache = cache_of(k, v)
        for new, lens in CALLS:
            q = dev(rng.standard_normal((sum(new), 3, dim)), torch.float32)
            for o in order:
                table = np.stack([o] * len(new))[:, :-(-330 // page)]
                attend(q.half(), cache, table, lens, new, page)
                attend(q, cache, table, lens, new, page, window=100)
