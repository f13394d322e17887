"""Low-rank adapters beside the linears, against float64.

h_r = sum_k x_k a_rk is a float32 sum of products that are exact (float16 by float16, or two bfloat16 by
bfloat16): off by at most (K + 16) 2^-23 sum |x_k a_rk|. The second product takes h as two float16 numbers about
its token's largest (2^-22 of itself, 2^-24 of the largest) or three bfloat16 ones (2^-23), times the scale
(2^-24), in a float32 sum of up to 3 R terms: (3 R + 8) 2^-23 of sum |s h_r b_r|; the sum with y rounds twice.
"""
import ctypes

import numpy as np
import pytest

from oracle import serving_oracle as S
from paper_2607_01127_amd import logbq as L

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
    return t if dtype is None else t.to(dtype)


def host(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def ints(v):
    return dev(np.asarray(v, dtype=np.int32))


def make(seed, new, k, n, adapters, rank, dtype):
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = sum(new)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    return dict(x=r(t, k).half(), ys=[r(t, m) for m in n], a=[(r(adapters, rank, k) * k ** -0.5).to(TYPES[dtype]) for _ in n],
                b=[(r(adapters, m, rank) * 0.3).to(TYPES[dtype]) for m in n],
                starts=ints(np.concatenate([[0], np.cumsum(new)])))


def call(d, adapter, max_new, scales=None, ranks=None, outs=None, **kw):
    return L.linear_adapters(d["x"], d["ys"], d["a"], d["b"], d["starts"], ints(adapter), max_new,
                             scales=None if scales is None else dev(np.asarray(scales, dtype=np.float32)),
                             ranks=None if ranks is None else ints(ranks), outs=outs, **kw)


def check(d, ys, got, adapter, scales=None, ranks=None):
    x, starts = host(d["x"]), host(d["starts"]).tolist()
    k = x.shape[1]
    for y, a, b, out in zip(ys, d["a"], d["b"], got):
        a, b, y, out = host(a), host(b), host(y), host(out)
        n = a.shape[0]
        ranks_ = [a.shape[1]] * n if ranks is None else [min(max(r, 0), a.shape[1]) for r in ranks]
        scales_ = [1.0] * n if scales is None else [float(np.float32(s)) for s in scales]
        a = [a[i][:ranks_[i]] for i in range(n)]
        ref = S.adapters(x, y, a, b, starts, adapter, ranks_, scales_)
        tol = 2.0 ** -23 * (np.abs(ref) + np.abs(y))
        for r, i in enumerate(adapter):
            rows = slice(starts[r], starts[r + 1])
            if not 0 <= i < n:
                assert np.array_equal(out[rows], y[rows])
                continue
            if not ranks_[i] or starts[r] == starts[r + 1]:
                continue
            size, bb = np.abs(x[rows]) @ np.abs(a[i]).T, np.abs(b[i][:, :ranks_[i]])
            h = np.abs(x[rows] @ a[i].T)
            e = (k + 16) * 2.0 ** -23 * size + (2.0 ** -22 + (3 * ranks_[i] + 8) * 2.0 ** -23) * h + \
                2.0 ** -24 * h.max(1, keepdims=True)
            tol[rows] += abs(scales_[i]) * (e @ bb.T)
        off = np.abs(out - ref) / np.maximum(tol, 1e-300)
        assert float(off.max(initial=0.0)) <= 1.0, float(off.max())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new,k,n,adapters,rank,mixed", [
    ([1], 32, [1], 1, 8, False), ([1], 2048, [2048, 512, 512], 2, 16, True), ([1] * 5, 4096, [300], 3, 64, True),
    ([1] * 70, 96, [257, 64], 7, 128, True), ([3, 0, 32, 1], 544, [33, 1000, 5, 64], 4, 24, True),
    ([33], 1024, [129], 1, 40, False), ([100, 1, 0, 64, 31], 1376, [511, 70], 3, 96, True),
    ([700, 5, 401], 2048, [260, 128, 64], 2, 32, True), ([2000], 64, [96], 1, 8, False)])
def test_against_float64(new, k, n, adapters, rank, mixed, dtype):
    print("adapters", new[:6], k, n, adapters, rank, mixed, dtype, flush=True)
    d = make(len(new) + k, new, k, n, adapters, rank, dtype)
    rng = np.random.default_rng(k)
    adapter = [int(rng.integers(-1, adapters)) if i else 0 for i in range(len(new))]
    ranks = [int(rng.integers(0, rank + 1)) if i else max(1, rank - 3) for i in range(adapters)] if mixed else None
    scales = rng.uniform(-2, 2, adapters) if mixed else None
    if mixed:      # what lies past an adapter's rank is not its own
        for a, b in zip(d["a"], d["b"]):
            for i, r in enumerate(ranks):
                a[i, r:] = float("nan")
                b[i, :, r:] = float("nan")
    outs = [torch.full_like(y, 5.0) for y in d["ys"]]
    got = call(d, adapter, max(new), scales, ranks, outs)
    check(d, d["ys"], got, adapter, scales, ranks)
    before = [y.clone() for y in d["ys"]]
    in_place = call(d, adapter, max(new), scales, ranks)
    assert all(a is b for a, b in zip(in_place, d["ys"])) and all(torch.equal(a, b) for a, b in zip(in_place, got))
    d["ys"] = before
    assert all(torch.equal(a, b) for a, b in zip(call(d, adapter, max(new) + 100, scales, ranks, outs), got)) or max(new) <= 32


def test_rows_that_are_left_as_they_were():
    # Requests end before the tokens do, begin after the first, one is cut at max_new, ids lie outside the pool.
    d = make(0, [64], 128, [70], 2, 8, "f16")
    d["starts"] = ints([3, 10, 50, 50, 61])
    for max_new, cut in ((40, 50), (32, 42), (16, 26)):
        outs = [torch.full_like(d["ys"][0], 5.0)]
        call(d, [1, 0, 1, -1], max_new, outs=outs)
        out = outs[0]
        assert bool((out[:3] == 5).all()) and bool((out[61:] == 5).all()) and bool((out[cut:50] == 5).all())
        assert not bool((out[3:cut] == 5).any()) and torch.equal(out[50:61], d["ys"][0][50:61])
        ref = [torch.full_like(d["ys"][0], 5.0)]
        L.linear_adapters(d["x"][10:cut].contiguous(), [d["ys"][0][10:cut].contiguous()], d["a"], d["b"],
                          ints([0, cut - 10]), ints([0]), cut - 10, outs=[ref[0][10:cut]])
        assert float((ref[0][10:cut] - out[10:cut]).abs().max()) < 1e-5
    outs = [torch.full_like(d["ys"][0], 5.0)]
    call(d, [2, 2**31 - 1, -2**31, -1], 64, outs=outs)
    assert torch.equal(outs[0][3:61], d["ys"][0][3:61])
    d["starts"] = ints([-5, 70, 20, 90, 64])              # starts out of range or falling
    call(d, [0, 0, 0, 0], 64, outs=outs)
    assert torch.isfinite(outs[0]).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_values_far_apart_and_no_numbers(dtype):
    d = make(1, [1, 1, 1, 1, 40], 256, [90], 1, 16, dtype)
    d["a"][0][0, 3] *= 1000.0
    d["x"][1] *= 1e-6                                     # subnormal float16 activations
    d["x"][2] *= 3000.0
    d["b"][0][0, :, 3] = 0.0                              # the largest h meets nothing
    adapter = [0] * 5
    got = call(d, adapter, 40, outs=[torch.empty_like(y) for y in d["ys"]])
    check(d, d["ys"], got, adapter)
    clean = got[0].clone()
    d["x"][0, 5] = float("nan")
    d["x"][7, 9] = float("inf")
    d["ys"][0][3, 4] = float("inf")
    got = call(d, adapter, 40, outs=[torch.empty_like(y) for y in d["ys"]])[0]
    assert torch.isnan(got[0]).all() and not torch.isfinite(got[7]).any()
    assert torch.isinf(got[3, 4]) and torch.isfinite(got[3]).sum() == 89
    rest = [t for t in range(44) if t not in (0, 3, 7)]
    assert torch.equal(got[rest], clean[rest])


def test_same_results_each_time_and_in_a_graph():
    d = make(2, [1] * 9, 4096, [1024, 300], 4, 32, "bf16")
    adapter = ints([0, 1, 2, 3, -1, 0, 0, 1, 2])
    work = torch.empty(L.linear_adapters_workspace_bytes(9, 2, 32), dtype=torch.uint8, device=DEV)
    outs = [torch.empty_like(y) for y in d["ys"]]
    run = lambda o, w=None: L.linear_adapters(d["x"], d["ys"], d["a"], d["b"], d["starts"], adapter, 1, outs=o,  # noqa: E731
                                              workspace=w)
    run(outs, work)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(outs, work)
    for i in range(3):
        d["x"].copy_(torch.randn_like(d["x"]))
        adapter.copy_(adapter.roll(1))
        work.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        want = run([torch.empty_like(y) for y in d["ys"]])
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = L.linear_adapters(d["x"], d["ys"], d["a"], d["b"], d["starts"], adapter, 1,
                            outs=[torch.empty_like(y) for y in d["ys"]], stream=stream)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_beside_the_linears():
    # y of logbq_linear_multi, adapted in place, equals the product with the merged weights.
    k, n = 512, (256, 128)
    lin = []
    for i, m in enumerate(n):
        w = torch.randn(m, k, generator=torch.Generator(device=DEV).manual_seed(i), device=DEV) * 0.05
        lin.append(L.encode(w, L.fit_device(w)))
    d = make(4, [5, 1, 2], k, n, 2, 16, "f16")
    ys = L.linear_multi(d["x"], *zip(*lin))
    before = [y.clone() for y in ys]
    d["ys"] = ys
    got = call(d, [1, -1, 0], 5, scales=[0.5, 2.0])
    check(d, before, got, [1, -1, 0], [0.5, 2.0])


@pytest.mark.parametrize("most", [1, 40])
def test_projections_without_features_need_no_buffers(most):
    """Each of four projections left out in turn, with null pointers, and all of them."""
    new, k, n = [most, 1, most], 96, [40, 300, 0, 7]
    d = make(7, new, k, n, 2, 16, "f16")
    ids = [1, -1, 0]
    want = [torch.empty_like(y) for y in d["ys"]]
    check(d, d["ys"], call(d, ids, most, outs=want), ids)
    tokens, where = sum(new), ints(ids)
    work = torch.empty(L.linear_adapters_workspace_bytes(tokens, 4, 16), dtype=torch.uint8, device=DEV)
    pointers, sizes = ctypes.c_void_p * 4, ctypes.c_int64 * 4
    for left in [set(), {0}, {1}, {3}, {0, 1}, {0, 1, 2, 3}]:
        outs = [torch.full_like(y, 3.0) for y in d["ys"]]
        at = lambda ts: pointers(*[None if i in left | {2} else t.data_ptr() for i, t in enumerate(ts)])  # noqa: E731
        assert L.lib().logbq_linear_adapters(
            d["x"].data_ptr(), tokens, k, 4, at(d["a"]), at(d["b"]),
            sizes(*[0 if i in left else m for i, m in enumerate(n)]), 1, 2, 16, None, None, d["starts"].data_ptr(),
            where.data_ptr(), 3, most, at(d["ys"]), at(outs), work.data_ptr(), work.numel(), L._stream(None)) == L.OK
        for i in range(4):
            assert torch.equal(outs[i], want[i]) if i not in left else bool((outs[i] == 3.0).all())


def test_more_tiles_than_a_grid_has_rows():
    """40000 requests of a token, as a step of up to five takes them."""
    n, adapters = 40000, 5
    d = make(11, [1] * n, 32, [16], adapters, 8, "f16")
    ids = [i % (adapters + 1) - 1 for i in range(n)]
    outs = [torch.empty_like(y) for y in d["ys"]]      # the call would update ys otherwise
    for most in (5, 1):
        check(d, d["ys"], call(d, ids, most, outs=outs), ids)


@pytest.mark.parametrize("most,rank", [(100, 128), (100, 16), (20, 64), (3, 8)])
def test_starts_that_do_not_ascend_stay_within_the_buffers(most, rank):
    tokens, requests, k, n = 100, 50, 64, 300
    d = make(most, [tokens], k, [n, n], 2, rank, "f16")
    d["starts"] = ints([0, tokens] * (requests // 2) + [-7])
    need = L.linear_adapters_workspace_bytes(tokens, 2, rank)
    held = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device=DEV)
    outs = [torch.full((tokens + 8, n), 7.0, device=DEV) for _ in range(2)]
    call(d, [0, 1] * (requests // 2), most, outs=[o[:tokens] for o in outs], workspace=held[:need])
    assert bool((held[need:] == 0x5a).all()) and all(bool((o[tokens:] == 7.0).all()) for o in outs)


@pytest.mark.parametrize("new", [1, 3])
def test_a_pool_that_goes_past_the_cache(new):
    """More weights than 128 MiB, two and four requests an adapter."""
    for requests in (36, 72):
        d = make(new, [new] * requests, 64, [33000], 18, 128, "bf16")
        ids = [r % 19 - 1 for r in range(requests)]
        outs = [torch.empty_like(y) for y in d["ys"]]
        rows = slice(0, 8 * new)
        call(d, ids, new, outs=outs)
        part = {k: ([v[0][rows]] if k == "ys" else v[rows] if k == "x" else v) for k, v in d.items()}
        part["starts"] = d["starts"][:9]
        check(part, part["ys"], [outs[0][rows]], ids[:8])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new,k,n,rank", [
    (1, 4096, [4096, 1024, 1024], 16), (1, 512, [257, 1, 300, 64], 128), (1, 32, [1], 8), (4, 2048, [700, 33], 16),
    (3, 96, [255], 128), (1, 4128, [640], 8)])
def test_small_calls(new, k, n, rank, dtype):
    """Calls of one launch, in place and out of it, and beside others that take two."""
    d = make(k + rank, [new, 0, 1, new, 1], k, n, 3, rank, dtype)
    ids, ranks, scales = [2, 1, 0, -1, 1], [rank, max(1, rank - 3), 0], [0.5, -1.5, 2.0]
    for a, b in zip(d["a"], d["b"]):
        for i, r in enumerate(ranks):
            a[i, r:] = float("nan")
            b[i, :, r:] = float("nan")
    outs = [torch.empty_like(y) for y in d["ys"]]
    check(d, d["ys"], call(d, ids, new, scales, ranks, outs=outs), ids, scales, ranks)
    before = [y.clone() for y in d["ys"]]
    call(d, ids, new, scales, ranks)
    assert all(torch.equal(a, b) for a, b in zip(d["ys"], outs))
    many = {key: [torch.cat([y] * 90) for y in before] if key == "ys" else v for key, v in d.items()}
    many["x"] = torch.cat([d["x"]] * 90)
    starts, total = host(d["starts"]), d["x"].shape[0]
    many["starts"] = ints(np.concatenate([starts[:-1] + i * total for i in range(90)] + [[90 * total]]))
    big = [torch.empty_like(y) for y in many["ys"]]
    check(many, many["ys"], call(many, ids * 90, new, scales, ranks, outs=big), ids * 90, scales, ranks)
