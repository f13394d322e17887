"""Adapters in pools of any size."""
import pytest

from test_gpu_adapters import call, check, make

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("k,n,rank,adapters", [(4096, [4096, 1024, 1024], 16, 700), (512, [28672], 128, 20)])
def test_a_small_call_in_pools_small_and_large(k, n, rank, adapters, dtype):
    """One request, whose adapter lies in a small pool and in one of more than 128 MiB of B."""
    print("pool", k, n, rank, adapters, dtype, flush=True)
    d = make(k, [1], k, n, 1, rank, dtype)
    check(d, d["ys"], call(d, [0], 1, outs=[torch.empty_like(y) for y in d["ys"]]), [0])
    assert 2 * adapters * rank * sum(n) > 128 << 20
    at = adapters - 2
    for name in ("a", "b"):
        pools = [torch.zeros((adapters, *w.shape[1:]), dtype=w.dtype, device=DEV) for w in d[name]]
        for pool, w in zip(pools, d[name]):
            pool[at] = w[0]
        d[name] = pools
    large = call(d, [at], 1, outs=[torch.empty_like(y) for y in d["ys"]])
    d["a"], d["b"] = ([p[at:at + 1] for p in pools] for pools in (d["a"], d["b"]))
    check(d, d["ys"], large, [0])
