"""Appending with slots that several tokens name: what those hold is not specified, every other slot is."""
import numpy as np
import pytest

from oracle import serving_oracle as S
from paper_2607_01127_amd import logbq as L

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (256, 32)])
def test_shared_slots_touch_no_others(dim, page):
    print("shared slots", dim, page, flush=True)
    rng = np.random.default_rng(dim)
    tokens, heads, pages = 90, 3, 9
    x = rng.standard_normal((2, tokens, heads, dim)).astype(np.float32)
    slots = rng.permutation(pages * page)[:tokens].astype(np.int64)
    shared = slots[:4].copy()
    slots[10:30] = shared[rng.integers(0, 4, 20)]
    cache = L.kv4_cache(pages, heads, dim, page)
    for t in cache:
        t.fill_(1)
    k, v = (torch.from_numpy(y).cuda() for y in x)
    L.kv4_append(k, v, cache, torch.from_numpy(slots).cuda())
    alone = [t for t in range(tokens) if slots[t] not in shared]
    held = np.ones(pages * page, dtype=bool)
    held[shared] = False
    for codes, scales, unpack, y in ((cache.k_codes, cache.k_scales, S.unpack_keys, x[0]),
                                     (cache.v_codes, cache.v_scales, S.unpack_values, x[1])):
        want, want_scale = np.zeros((pages, heads, page, dim), dtype=np.uint8), np.ones((pages, heads, page))
        want[..., 0::2] = 1                                   # the byte 1: codes 1 and 0
        rows, row_scales = S.kv4_quantize(y.astype(np.float64))
        for t in alone:
            want[slots[t] // page, :, slots[t] % page] = rows[t]
            want_scale[slots[t] // page, :, slots[t] % page] = row_scales[t]
        at = lambda a: np.moveaxis(a, 1, 2).reshape(pages * page, heads, -1)[held]  # noqa: E731
        assert np.array_equal(at(unpack(codes.cpu().numpy())), at(want))
        assert np.array_equal(at(scales.float().cpu().numpy()[..., None]), at(want_scale[..., None]))
