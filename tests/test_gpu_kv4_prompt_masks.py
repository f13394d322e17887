"""Attention of prompts and chunks where a tile of positions shows a row nothing before the tiles that it
sees: hidden pages, windows, keys of nothing but zeros; with logits far from 0."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from attention_check import TYPES, attend, cache_of, dev  # noqa: E402

pytestmark = pytest.mark.gpu


def rows_at(rng, shape, level, scale, group):
    """Keys, and queries' one value, such that the logits lie about `level`, each row a little apart."""
    k = 0.5 + np.abs(rng.standard_normal(shape))
    q = level / (scale * shape[-1] * k.mean())
    return k, q


@pytest.mark.parametrize("level", [0.0, -80.0, -100.0, -300.0, 200.0])
@pytest.mark.parametrize("dim,page,width", [(128, 16, 22), (64, 64, 6), (256, 32, 11), (64, 16, 300),
                                            (128, 128, 40)])
def test_hidden_tiles_before_visible_ones(dim, page, width, level):
    """The first tiles' pages are negative or past the cache; wide tables are worked on in splits, some
    of which see nothing at all. One request alone, and beside others."""
    print("hidden tiles", dim, page, width, level, flush=True)
    rng = np.random.default_rng(dim + page)
    heads, group, pages = 2, 2, 24
    scale = dim ** -0.5
    k, qv = rows_at(rng, (pages, heads, page, dim), level, scale, group)
    v = rng.standard_normal(k.shape)
    cache = cache_of(k, v)
    n = width * page - 5
    for hidden in (128, n - 70):              # positions, up to a page's end, that are hidden
        table = rng.integers(0, pages, (3, width)).astype(np.int32)
        m = -(-hidden // page)
        table[0, :m] = -1
        table[2, :m:2], table[2, 1:m:2] = pages, 2 ** 30
        for new, lens in (([90], [n]), ([66, 1, 81], [n, n // 2, n])):
            q = dev(qv * (1 + 0.01 * rng.standard_normal((sum(new), heads * group, dim))), torch.float32).half()
            attend(q, cache, table[:len(new)], lens, new, page, scale=scale)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_zero_keys_outside_the_window(dim):
    """The first tile's keys are zero rows, or tiny ones, which only some rows of a wavefront see; the
    others' windows begin later, at logits of about -300."""
    print("zero keys", dim, flush=True)
    rng = np.random.default_rng(dim)
    heads, page, pages, scale = 1, 64, 5, dim ** -0.5
    for first in (0.0, 1e-38, 1e-30):
        k, qv = rows_at(rng, (pages, heads, page, dim), -300.0, scale, 1)
        k[0] *= first
        cache = cache_of(k, rng.standard_normal(k.shape))
        q = dev(qv * (1 + 0.01 * rng.standard_normal((290, 1, dim))), torch.float32)
        for dtype in ("f16", "bf16", "f32"):
            attend(q.to(TYPES[dtype]), cache, [[0, 1, 2, 3, 4]], [290], [290], page, scale=scale, window=16)


def test_tiny_keys_and_large_queries():
    """Keys whose scales are below 2^-117: a tile's factor has to stay a number other than 0."""
    print("tiny keys", flush=True)
    rng = np.random.default_rng(5)
    for dim in (64, 128, 256):
        k = rng.standard_normal((4, 1, 64, dim)) * 2.0 ** -122
        cache = cache_of(k, rng.standard_normal(k.shape))
        q = dev(rng.standard_normal((200, 2, dim)) * 2.0 ** 122, torch.float32)
        for dtype in ("bf16", "f32"):
            for new in ([200], [1]):
                attend(q[:new[0]].to(TYPES[dtype]), cache, [[2, 0, 3, 1]], [240], new, 64)
