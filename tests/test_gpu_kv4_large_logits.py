"""Attention whose logits are far larger than float32 resolves: a row's largest weight is 1 whatever its
logit, so equal keys share the weight and a key that stands out takes it."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from attention_check import DEV, TYPES, cache_of, dev, host  # noqa: E402
from paper_2607_01127_amd import logbq as L  # noqa: E402

pytestmark = pytest.mark.gpu
POWERS = [0, 20, 24, 28, 31, 33, 40, 60, 90]


def call(q, buffers, table, lens, new, out=torch.float32):
    lse = torch.empty(q.shape[:2], device=DEV)
    res = torch.full(q.shape, math.nan, device=DEV, dtype=out)
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    L.kv4_attention(q, buffers, dev(np.asarray(table, dtype=np.int32)), dev(np.asarray(lens, dtype=np.int32)),
                    dev(starts), max(new), out=res, lse=lse)
    return host(res), host(lse)


@pytest.mark.parametrize("dim,page,group", [(64, 16, 4), (128, 64, 2), (256, 32, 3), (64, 64, 16)])
@pytest.mark.parametrize("sign", [1, -1])
def test_equal_keys_share_the_weight(dim, page, group, sign):
    """All keys are one row, so a query's logits are equal to the last bit: the output is the mean of the
    values seen. Each weight is rounded to 16 bits (2^-15 covers it and the sums of up to 130 terms add
    130 2^-23); the log sum is the logit, whose float32 sum is off by (D + 16) 2^-23 of sum |q k|, plus
    log n, to 2^-22 of itself."""
    print("equal keys", dim, page, group, sign, flush=True)
    rng = np.random.default_rng(dim)
    pages = -(-130 // page)
    row = sign * (0.5 + rng.random(dim))
    v = rng.standard_normal((pages, 1, page, dim))
    table = rng.permutation(pages)[None]
    for power in POWERS:
        buffers, kk, vv = cache_of(np.broadcast_to(row * 2.0 ** power, v.shape), v)
        rows = vv[table[0], 0].reshape(-1, dim)
        for new in (1, 3, 130):
            q = dev(0.5 + rng.random((new, group, dim)), torch.float32)
            for dtype in ("f16", "f32"):
                res, lse = call(q.to(TYPES[dtype]), buffers, table, [130], [new])
                logit = host(q.to(TYPES[dtype])) @ kk[0, 0, 0] * dim ** -0.5
                for t in range(new):
                    n = 130 - new + t + 1
                    mean, size = rows[:n].mean(0), np.abs(rows[:n]).mean(0)
                    assert np.all(np.abs(res[t] - mean) <= size * (2.0 ** -15 + n * 2.0 ** -23)), (power, new, t)
                    want = logit[t] + math.log(n)
                    tol = (dim + 16) * 2.0 ** -23 * (np.abs(logit[t]) + 2) + 2.0 ** -22 * np.abs(want)
                    assert np.all(np.abs(lse[t] - want) <= tol), (power, new, t, lse[t], want)


@pytest.mark.parametrize("dim,page,group", [(64, 16, 4), (128, 64, 2), (256, 32, 3)])
def test_the_larger_of_large_ones_takes_the_weight(dim, page, group):
    """Keys of one direction at sizes 2^power (1 + position / 64), so that neighbours' logits differ by
    more than the error of either: the last position seen has all the weight for a positive direction, the
    first for a negative one. The output is that value, rounded to 16 bits at most."""
    print("one of large ones", dim, page, group, flush=True)
    rng = np.random.default_rng(dim)
    n, pages = 90, -(-90 // page)
    v = rng.standard_normal((pages, 1, page, dim))
    table = np.arange(pages)[None]
    grow = 1 + np.arange(pages * page).reshape(pages, 1, page, 1) / 64
    for sign in (1.0, -1.0):
        for power in POWERS[1:]:
            # Scales are rounded up to 8 bits and codes to nearest, so sizes come in steps: positions that
            # share one with their neighbours are left to the other test.
            buffers, kk, vv = cache_of(np.full(v.shape, sign * 2.0 ** power) * grow, v)
            size, rows = kk[:, 0].reshape(-1, dim)[:, 0], vv[:, 0].reshape(-1, dim)
            for new in (1, 2, n):
                q = dev(0.5 + rng.random((new, group, dim)), torch.float32)
                res, _ = call(q.half(), buffers, table, [n], [new])
                for t in range(new):
                    seen = size[:n - new + t + 1]
                    best = np.flatnonzero(seen == seen.max())
                    if best.size == 1:
                        want = rows[best[0]]
                        assert np.all(np.abs(res[t] - want) <= 2.0 ** -15 * np.abs(want)), (power, sign, new, t)
