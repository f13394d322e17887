"""Adapters in calls whose bound of a request's tokens is far above them. Tolerances as in test_gpu_adapters."""
import numpy as np
import pytest

from test_gpu_adapters import call, check, make

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new,k,n,adapters,rank,mixed", [
    ([1], 32, [1], 1, 8, False), ([1], 2048, [2048, 512, 512], 2, 16, True), ([1] * 5, 4096, [300], 3, 64, True),
    ([1] * 70, 96, [257, 64], 7, 128, True), ([3, 0, 32, 1], 544, [33, 1000, 5, 64], 4, 24, True),
    ([33], 1024, [129], 1, 40, False), ([100, 1, 0, 64, 31], 1376, [511, 70], 3, 96, True),
    ([2, 4, 1, 3], 512, [260], 2, 8, True)])
def test_a_loose_bound_of_tokens(new, k, n, adapters, rank, mixed, dtype):
    """A server may know no more than the most tokens of any request."""
    print("loose bound", new[:6], k, n, adapters, rank, mixed, dtype, flush=True)
    d = make(len(new) + k, new, k, n, adapters, rank, dtype)
    rng = np.random.default_rng(k)
    adapter = [int(rng.integers(-1, adapters)) if i else 0 for i in range(len(new))]
    ranks = [int(rng.integers(0, rank + 1)) if i else max(1, rank - 3) for i in range(adapters)] if mixed else None
    scales = rng.uniform(-2, 2, adapters) if mixed else None
    if mixed:
        for a, b in zip(d["a"], d["b"]):
            for i, r in enumerate(ranks):
                a[i, r:] = float("nan")
                b[i, :, r:] = float("nan")
    for bound in (4, 5, 32, 33, max(new) + 100, 2**31 + 5):
        if bound >= max(new):
            outs = [torch.full_like(y, 5.0) for y in d["ys"]]
            check(d, d["ys"], call(d, adapter, bound, scales, ranks, outs), adapter, scales, ranks)
