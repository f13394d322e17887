"""Draft trees: ancestor masks and positions (exact), and attention of trees over the 4-bit cache against float64
with the bounds of attention_check (sums over the positions that a node sees)."""
import math

import numpy as np
import pytest

from attention_check import HALF_ULP, TYPES, cache_of, dev, host
from oracle import serving_oracle as S
from paper_2607_01127_amd import logbq as L

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def ints(v):
    return dev(np.asarray(v, dtype=np.int32))


def some_tree(rng, n):
    return [int(rng.integers(max(-1, i - 4), i)) if rng.random() < 0.8 else int(rng.integers(-1, max(1, i))) for i in range(n)]


# ------------------------------------------------------------------ tables

def check_tables(parents, new, lens):
    starts = np.concatenate([[0], np.cumsum(new)])
    want, places = S.tree_tables(parents, starts.tolist(), lens)
    got = L.tree_tables(ints(parents), ints(starts), ints(lens))
    masks = got["masks"].cpu().numpy().view(np.uint64)
    positions = got["positions"].cpu().numpy()
    assert {t: int(masks[t]) for t in want} == want
    assert {t: int(positions[t]) for t in places} == places


@pytest.mark.parametrize("seed,n", [(0, 1), (1, 5), (2, 70), (3, 1000)])
def test_tables_random(seed, n):
    print("tree tables", n, flush=True)
    rng = np.random.default_rng(seed)
    new = rng.integers(0, 70, n)
    parents = [p for m in new for p in some_tree(rng, int(m))]
    check_tables(parents, new, rng.integers(-3, 5000, n).tolist())


def test_tables_edges():
    chain = list(range(-1, 63))
    check_tables(chain, [64], [64])                        # the longest path
    check_tables([-1] * 64, [64], [100])
    check_tables(list(range(63, -1, -1)), [64], [70])      # parents that do not come before their nodes
    check_tables([0, 1, 2, -2**31, 2**31 - 1], [5], [5])
    check_tables(chain + [3, 4], [66], [2**31 - 1])        # nodes past the 64th
    check_tables([0] + chain[:3], [1, 3], [0, 1])          # lengths shorter than the nodes


def test_tables_leave_the_rest_alone_and_run_in_a_graph():
    out = dict(masks=torch.full((9,), 5, dtype=torch.int64, device=DEV),
               positions=torch.full((9,), 6, dtype=torch.int32, device=DEV))
    parents, starts, lens = ints([-1] * 9), ints([2, 4, 4, 7]), ints([10, 10, 10])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.tree_tables(parents, starts, lens, out=out)
    for i in range(3):
        parents.copy_(ints([-1, -1, -1, 0 if i else -1, -1, 0, 1, -1, -1]))
        graph.replay()
        torch.cuda.synchronize()
        assert out["masks"].tolist() == [5, 5, 1, 3 if i else 2, 1, 3, 7, 5, 5]
        assert out["positions"].tolist() == [6, 6, 8, 9 if i else 8, 7, 8, 9, 6, 6]


# ------------------------------------------------------------------ attention

def exact(q, k, v, table, lens, starts, masks, page, scale, window, max_new):
    tokens, q_heads, dim = q.shape
    heads = k.shape[1]
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    lse, lse_tol = np.full((tokens, q_heads), -np.inf), np.zeros((tokens, q_heads))
    for r in range(len(lens)):
        a, b = int(starts[r]), int(starts[r + 1])
        cached = int(lens[r]) - (b - a)
        for t in range(a, min(b, a + max_new)):
            bits = int(masks[t]) & ((1 << min(b - a, max_new)) - 1)
            depth = max(0, bin(bits).count("1") - 1)
            j = np.arange(max(0, cached + depth - window + 1 if window else 0), max(0, cached))
            nodes = [cached + i for i in range(min(b - a, max_new)) if bits >> i & 1 and cached + i >= 0]
            j = np.concatenate([j, np.array(nodes, dtype=np.int64)]).astype(np.int64)
            j = j[j < table.shape[1] * page]
            j = j[(table[r, j // page] >= 0) & (table[r, j // page] < k.shape[0])]
            if not j.size:
                continue
            ids, off = table[r, j // page], j % page
            for h in range(q_heads):
                kk, vv = k[ids, h * heads // q_heads, off], v[ids, h * heads // q_heads, off]
                s = scale * (kk @ q[t, h])
                d = (dim + 16) * 2.0 ** -23 * (abs(scale) * (np.abs(kk) @ np.abs(q[t, h])) + 2)
                w = np.exp(s - s.max())
                total = w.sum()
                w /= total
                size = w @ np.abs(vv)
                out[t, h], lse[t, h] = w @ vv, s.max() + math.log(total)
                e = w * (2 * d + 2.0 ** -15)
                tol[t, h] = (e @ np.abs(vv) + (e.sum() + j.size * 2.0 ** -23) * size +
                             j.size * 2.0 ** -126 * np.abs(vv).max(0))
                lse_tol[t, h] = w @ d + j.size * 2.0 ** -24 + 2.0 ** -22 * (abs(lse[t, h]) + 1)
    return out, lse, tol, lse_tol


def attend(q, cache, table, lens, new, masks, page, out="f32", scale=None, window=0, max_new=None, **kw):
    """One call, checked; rows that no request has keep what they held."""
    buffers, k, v = cache
    table = np.asarray(table, dtype=np.int32)
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    scale = q.shape[2] ** -0.5 if scale is None else scale
    most = max(new) if max_new is None else max_new
    lse = torch.full(q.shape[:2], 7.0, device=DEV)
    res = torch.full(q.shape, 7.0, device=DEV, dtype=TYPES[out])
    bits = dev(np.array(masks, dtype=np.uint64).view(np.int64))
    L.kv4_tree_attention(q, buffers, dev(table), ints(lens), dev(starts), bits, most, scale=scale, window=window,
                         out=res, lse=lse, **kw)
    ref, ref_lse, tol, lse_tol = exact(host(q), k, v, table, lens, starts, masks, page, scale, window, most)
    got, got_lse = host(res), host(lse)
    mine = np.zeros(q.shape[0], dtype=bool)
    for a, b in zip(starts[:-1], starts[1:]):
        mine[a:min(b, a + most)] = True
    assert (got[~mine] == 7).all() and (got_lse[~mine] == 7).all()
    got, got_lse, ref, ref_lse, tol, lse_tol = (x[mine] for x in (got, got_lse, ref, ref_lse, tol, lse_tol))
    empty = np.isneginf(ref_lse)
    assert np.array_equal(np.isneginf(got_lse), empty)
    assert not got[empty].any() and not np.isnan(got).any()
    off = np.abs(got_lse[~empty] - ref_lse[~empty]) / lse_tol[~empty]
    assert float(np.max(off, initial=0.0)) <= 1.0, float(off.max())
    tol = tol + HALF_ULP[out] * np.abs(ref) + (2.0 ** -25 if out == "f16" else 0.0)
    off = np.abs(got - ref) / np.where(tol > 0, tol, 1e-300)
    assert float(np.max(off, initial=0.0)) <= 1.0, float(off.max())
    return res, lse


def step(seed, lens, new, heads, group, dim, page, dtype, spare=2):
    rng = np.random.default_rng(seed)
    used = [-(-max(0, n) // page) for n in lens]
    pages, width = sum(used) + spare, max(used) + 1
    order = rng.permutation(pages)
    table, at = np.full((len(lens), width), -1, dtype=np.int32), 0
    for r, n in enumerate(used):
        table[r, :n] = order[at:at + n]
        at += n
    k = rng.standard_normal((pages, heads, page, dim)) * np.exp(rng.uniform(-1, 1, (pages, heads, page, 1)))
    v = rng.standard_normal((pages, heads, page, dim)) * np.exp(rng.uniform(-2, 2, (pages, heads, page, 1)))
    q = dev(rng.standard_normal((sum(new), heads * group, dim)).astype(np.float32), TYPES[dtype])
    parents = [p for n in new for p in some_tree(rng, n)]
    starts = np.concatenate([[0], np.cumsum(new)]).tolist()
    masks, _ = S.tree_tables(parents, starts, lens)
    return q, cache_of(k, v), table, [masks[t] for t in range(sum(new))]


SHAPES = [  # lens, new, heads, group, dim, page: rows of 1 to 32, of 33 to 64 and more, several tiles of them
    ([1], [1], 1, 1, 64, 16), ([7], [7], 1, 4, 64, 16), ([700], [7], 2, 4, 64, 64), ([130], [16], 1, 4, 128, 64),
    ([500, 64, 1, 200], [9, 13, 1, 16], 2, 4, 128, 64), ([300, 17], [64, 17], 1, 4, 128, 16),
    ([190, 128, 64], [24, 64, 33], 1, 1, 128, 32), ([150], [64], 1, 16, 64, 128), ([90, 33], [12, 30], 2, 5, 256, 16),
    ([1000], [3], 1, 7, 256, 64), ([2500, 5, 40], [40, 3, 2], 1, 2, 128, 64), ([65, 66, 127, 128, 129], [1, 2, 63, 64, 1], 1, 1, 64, 64)]


@pytest.mark.parametrize("dtype,out", [("f16", "f16"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("lens,new,heads,group,dim,page", SHAPES)
def test_attention(lens, new, heads, group, dim, page, dtype, out):
    print("tree", lens, new, heads, group, dim, page, dtype, flush=True)
    q, cache, table, masks = step(sum(lens), lens, new, heads, group, dim, page, dtype)
    res, lse = attend(q, cache, table, lens, new, masks, page, out)
    again, again_lse = attend(q, cache, table, lens, new, masks, page, out)
    assert torch.equal(res, again) and torch.equal(lse, again_lse)


@pytest.mark.parametrize("window", [64, 65, 100, 1000])
@pytest.mark.parametrize("dim,page,group", [(64, 64, 1), (128, 16, 4), (256, 32, 2)])
def test_windows(window, dim, page, group):
    lens, new = [400, 70, 64, 129], [20, 33, 64, 1]
    q, cache, table, masks = step(window, lens, new, 1, group, dim, page, "f16")
    attend(q, cache, table, lens, new, masks, page, "f32", window=window)


@pytest.mark.parametrize("group", [1, 2, 4])
def test_bits_past_the_tokens_make_no_depth(group):
    """A window goes by the bits of the request's own tokens, max_new of them at most."""
    lens, new = [300, 200, 128], [7, 20, 64]
    q, cache, table, masks = step(17, lens, new, 1, group, 64, 16, "f16")
    starts = np.concatenate([[0], np.cumsum(new)]).tolist()
    for a, b in zip(starts[:-1], starts[1:]):
        for t in range(a, b):
            masks[t] |= (2**64 - 1) >> (b - a) << (b - a)
    attend(q, cache, table, lens, new, masks, 16, "f32", window=70)
    attend(q, cache, table, lens, new, [2**64 - 1] * sum(new), 16, "f32", window=70, max_new=8)


def test_a_chain_is_what_causal_attention_computes():
    for dim, page in ((64, 64), (128, 16), (128, 128), (256, 64)):
        lens, new = [900, 20, 333], [30, 20, 1]
        q, (buffers, _, _), table, _ = step(dim, lens, new, 2, 4, dim, page, "f16")
        starts = ints(np.concatenate([[0], np.cumsum(new)]))
        masks = dev(np.array([(1 << (i + 1)) - 1 for n in new for i in range(n)], dtype=np.uint64).view(np.int64))
        args = (q, buffers, dev(table), ints(lens), starts)
        outs = [torch.empty(q.shape, device=DEV) for _ in range(2)]
        lses = [torch.empty(q.shape[:2], device=DEV) for _ in range(2)]
        L.kv4_attention(*args, 30, out=outs[0], lse=lses[0])
        L.kv4_tree_attention(*args, masks, 30, out=outs[1], lse=lses[1])
        # Both are within 2^-14 of the exact weights (16 bits each) of values up to 6 scales.
        assert float((outs[0] - outs[1]).abs().max()) <= 2.0 ** -12 * float(outs[0].abs().max())
        assert float((lses[0] - lses[1]).abs().max()) <= 1e-4


def test_masks_that_are_no_trees():
    # Nothing, itself left out, bits past the request, everything.
    lens, new = [40, 6], [6, 6]
    q, cache, table, _ = step(3, lens, new, 1, 2, 64, 16, "f16")
    masks = [0, 0b11110, 1 << 63, 2**64 - 1, 0b10, 0b100000 | 1 << 40, 0, 0, 1 << 5, 1 << 63, 0b111111, 1]
    attend(q, cache, table, lens, new, masks, 16)


def test_hidden_pages_and_short_tables():
    lens, new = [300, 200, 90, 5], [20, 7, 64, 9]
    q, cache, table, masks = step(5, lens, new, 1, 4, 128, 16, "f16")
    table[0, 3:6], table[1, 0], table[1, 5] = -1, 2**30, -7
    table[2, :] = -1                                       # nothing at all is seen
    attend(q, cache, table, lens, new, masks, 16)
    attend(q, cache, table[:, :4], lens, new, masks, 16)    # requests longer than the table: their nodes are past it
    attend(q, cache, table, lens, new, masks, 16, window=64)


def test_lengths_that_do_not_fit():
    lens, new = [3, 0, -5, 64], [5, 4, 3, 64]              # shorter than the nodes
    q, cache, table, masks = step(6, lens, new, 2, 2, 64, 16, "f16")
    attend(q, cache, table, lens, new, masks, 16)


def test_a_cache_without_pages_and_a_table_without_columns():
    q = torch.randn(5, 4, 64, device=DEV).half()
    bits, starts, lens = dev(np.full(5, 31, dtype=np.int64)), ints([0, 3, 5]), ints([10, 2])
    for pages, width in ((0, 0), (0, 2), (2, 0)):
        out, lse = torch.full_like(q, 7.0), torch.zeros(5, 4, device=DEV)
        L.kv4_tree_attention(q, L.kv4_cache(pages, 2, 64, 16), torch.zeros((2, width), dtype=torch.int32, device=DEV), lens,
                             starts, bits, 3, out=out, lse=lse)
        assert not out.any() and torch.isneginf(lse).all()


def test_max_new_leaves_tokens_out():
    lens, new = [100, 30], [20, 6]
    q, cache, table, masks = step(7, lens, new, 1, 4, 128, 16, "f16")
    full, _ = attend(q, cache, table, lens, new, masks, 16)
    part, _ = attend(q, cache, table, lens, new, masks, 16, max_new=8)
    assert torch.equal(full[20:], part[20:])


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_values_and_scales_that_are_no_numbers_reach_only_rows_that_see_them(dim):
    lens, new = [200], [20]
    q, (buffers, k, v), table, masks = step(8, lens, new, 1, 4, dim, 16, "f16")
    starts = ints([0, 20])
    bits = dev(np.array(masks, dtype=np.uint64).view(np.int64))
    call = lambda: L.kv4_tree_attention(q, buffers, dev(table), ints(lens), starts, bits, 20,  # noqa: E731
                                        out=torch.empty(q.shape, device=DEV))
    clean = call()
    node = 11                                              # its key's and value's scales are no numbers
    page, off = int(table[0, (180 + node) // 16]), (180 + node) % 16
    buffers.k_scales[page, 0, off] = float("nan")
    buffers.v_scales[page, 0, off] = float("inf")
    sees = torch.tensor([bool(m >> node & 1) for m in masks], device=DEV)
    got = call()
    assert not torch.isfinite(got[sees]).any() or torch.isnan(got[sees]).any(-1).all()
    assert torch.isfinite(got[~sees]).all()
    assert float((got[~sees] - clean[~sees]).abs().max()) <= 2.0 ** -13 * float(clean.abs().max())
    q[4, 1] = float("nan")
    got = call()
    assert torch.isnan(got[4, 1]).all() and torch.isfinite(got[~sees][:, 0]).all()


@pytest.mark.parametrize("factor,scale", [(2.0 ** 14, None), (1.0, 2.0 ** 26), (1.0, -3.0)])
def test_far_logits(factor, scale):
    # Logits past 2^20 take the careful way.
    lens, new = [150, 90], [10, 40]
    q, cache, table, masks = step(9, lens, new, 1, 4, 128, 16, "f32")
    attend(q * factor, cache, table, lens, new, masks, 16, scale=scale)


def test_keys_of_scales_far_apart():
    rng = np.random.default_rng(10)
    lens, new, page, dim = [192], [12], 64, 128
    k = rng.standard_normal((3, 1, page, dim)) * np.exp2(rng.integers(-60, 1, (3, 1, page, 1)).astype(float))
    v = rng.standard_normal((3, 1, page, dim)) * np.exp2(rng.integers(-30, 30, (3, 1, page, 1)).astype(float))
    q = dev(rng.standard_normal((12, 4, dim)).astype(np.float32))
    masks, _ = S.tree_tables(some_tree(rng, 12), [0, 12], lens)
    attend(q, cache_of(k, v), np.array([[2, 0, 1]]), lens, new, [masks[i] for i in range(12)], page)


def test_strided_queries_another_stream_and_graphs():
    lens, new = [500, 64, 1, 200], [9, 13, 1, 16]
    q, (buffers, k, v), table, masks = step(11, lens, new, 2, 4, 128, 64, "f16")
    wide = torch.randn(q.shape[0], 12, 128, device=DEV).half()
    wide[:, :8] = q
    attend(wide[:, :8], (buffers, k, v), table, lens, new, masks, 64)
    bits, starts, table, lens = dev(np.array(masks, dtype=np.uint64).view(np.int64)), ints([0, 9, 22, 23, 39]), dev(table), ints(lens)
    work = torch.empty(L.KV4_WORKSPACE_BYTES, dtype=torch.uint8, device=DEV)
    out = torch.empty_like(q)
    run = lambda o, w, **kw: L.kv4_tree_attention(q, buffers, table, lens, starts, bits, 16, out=o, workspace=w, **kw)  # noqa: E731
    want = run(torch.empty_like(q), None).clone()
    graphs = []
    for _ in range(2):                                     # two graphs share a workspace
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            run(out, work)
    for i in range(4):
        work.fill_(255 * (i & 1))
        out.zero_()
        graphs[i & 1].replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        q.copy_(q.roll(1, 0))
        want = run(torch.empty_like(q), None).clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = run(torch.empty_like(q), None, stream=stream)
    stream.synchronize()
    assert torch.equal(got, want)


def test_long_and_short_requests_share_the_chip():
    # Pieces of one request on many workgroups, many requests on one.
    lens, new = [6000] + [70] * 30, [40] + [2] * 30
    q, cache, table, masks = step(12, lens, new, 2, 4, 64, 64, "f16")
    attend(q, cache, table, lens, new, masks, 64)


@pytest.mark.parametrize("dim,most", [(64, 24), (128, 3)])
def test_more_requests_than_a_workgroup_has_threads(dim, most):
    rng = np.random.default_rng(dim)
    new = [int(n) for n in rng.integers(0, most + 1, 700)]
    new[13] = most
    lens = [n + int(c) for n, c in zip(new, rng.integers(0, 90, 700))]
    q, cache, table, masks = step(dim, lens, new, 1, 2, dim, 32, "f16")
    attend(q, cache, table, lens, new, masks, 32)
