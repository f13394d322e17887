"""Tokens whose masks hold no bit, in a window: depth is the number of bits less one, so such a token sees the
cached positions past cached - 1 - window, which are one position more than a tree's first node sees."""
import numpy as np
import pytest

from attention_check import HALF_ULP, dev, host
from paper_2607_01127_amd import logbq as L
from test_gpu_tree import exact, ints, step

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


# Windows that begin at the first and last position of a page and of a tile, and within them; one that holds more than
# there is. 1 to 16 query rows, 17 to 64, and more.
@pytest.mark.parametrize("window,cached", [(64, 383), (64, 384), (65, 300), (100, 130), (1000, 90), (200, 200), (200, 199)])
@pytest.mark.parametrize("dim,page,group,new", [(64, 64, 1, 3), (128, 16, 4, 2), (256, 32, 4, 4), (64, 16, 2, 12),
                                                (128, 64, 4, 9), (128, 32, 4, 30), (256, 64, 2, 50)])
def test_windows_of_empty_masks(window, cached, dim, page, group, new):
    print("empty masks", window, cached, dim, page, group, new, flush=True)
    lens, counts = [cached + new, 40 + new], [new, new]
    q, (buffers, k, v), table, masks = step(window + cached + dim, lens, counts, 2, group, dim, page, "f16")
    empty = np.arange(2 * new) % 3 == 1
    masks = [0 if e else m for e, m in zip(empty, masks)]
    starts, scale = np.array([0, new, 2 * new]), dim ** -0.5
    lse = torch.empty(q.shape[:2], device=DEV)
    out = L.kv4_tree_attention(q, buffers, dev(table), ints(lens), ints(starts),
                               dev(np.array(masks, dtype=np.uint64).view(np.int64)), new, window=window,
                               out=torch.empty(q.shape, device=DEV), lse=lse)
    # exact() counts an empty mask's depth as 0; with a window of one more it begins where depth -1 does.
    some, none = (exact(host(q), k, v, table, lens, starts, masks, page, scale, w, new) for w in (window, window + 1))
    pick = lambda i: np.where(empty.reshape((-1,) + (1,) * (some[i].ndim - 1)), none[i], some[i])  # noqa: E731
    ref, ref_lse, tol, lse_tol = (pick(i) for i in range(4))
    assert float(np.max(np.abs(host(lse) - ref_lse) / lse_tol)) <= 1.0
    assert float(np.max(np.abs(host(out) - ref) / (tol + HALF_ULP["f32"] * np.abs(ref)))) <= 1.0
