"""Adapters of activations with infinities."""
import pytest

from test_gpu_adapters import call, make

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new,requests", [(1, 1), (1, 300), (3, 40), (5, 3), (40, 2), (70, 2)])
def test_an_infinite_activation(new, requests, dtype):
    """x A^T is infinite for an adapter of one rank, and so is every output where B is not 0, with B's sign. The
    other tokens are what they are without it."""
    k, n, rank = 256, [300, 17], 8
    print("infinite", new, requests, dtype, flush=True)
    d = make(new, [new] * requests, k, n, 2, rank, dtype)
    ids, ranks, t = [0] * requests, [1, 8], new - 1
    for a in d["a"]:
        a[0, 0, 9] = 0.5
    clean = call(d, ids, new, ranks=ranks, outs=[torch.empty_like(y) for y in d["ys"]])
    for sign in (1.0, -1.0):
        d["x"][t, 9] = sign * float("inf")
        got = call(d, ids, new, ranks=ranks, outs=[torch.empty_like(y) for y in d["ys"]])
        for out, before, b in zip(got, clean, d["b"]):
            want = sign * torch.sign(b[0, :, 0].float()) * float("inf")
            some = b[0, :, 0] != 0
            assert torch.equal(out[t][some], want[some])
            others = torch.arange(len(out), device=DEV) != t
            assert torch.equal(out[others], before[others])
