"""Buffers whose offsets pass 32 bits: what lies at their ends is as in small ones, bit for bit."""
import pytest

from paper_2607_01127_amd import logbq as L

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def normal(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("group", [2, 4])
def test_trees_in_the_last_pages_of_a_long_cache(group):
    """4.4 GB of codes of keys, and as many of values; 8 nodes of 2 and 4 query heads each take the two ways."""
    heads, dim, page, pages, length, new = 8, 256, 1024, 4200, 2500, 8
    table = torch.tensor([[4199, 3, 4198]], dtype=torch.int32, device=DEV)
    k, v, q = normal(length, heads, dim), normal(length, heads, dim, seed=1), normal(new, heads * group, dim, seed=2).half()
    turn = L.Rotation(10000.0 ** (-torch.arange(dim // 2, device=DEV) / 128.0))
    at = torch.arange(length, device=DEV)
    outs = []
    for number, ids in ((3, torch.tensor([0, 1, 2], device=DEV)), (pages, table[0].long())):
        cache = L.kv4_cache(number, heads, dim, page, DEV)
        slots = ids[at // page] * page + at % page
        L.kv4_append_rotated(None, k, v, cache, slots, at.int(), turn)
        tables = L.tree_tables(ints([-1, 0, 0, 1, -1, 4, 3, 3]), ints([0, new]), ints([length]))
        lse = torch.empty(new, heads * group, device=DEV)
        outs.append((L.kv4_tree_attention(q, cache, ids.int()[None], ints([length]), ints([0, new]), tables["masks"], new,
                                          lse=lse), lse, *L.kv4_read(cache, slots)))
        del cache
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    assert float(outs[0][2].abs().sum()) > 0 and bool(torch.isfinite(outs[0][1]).all())


def test_rotation_of_long_rows():
    """2.6e9 elements, in place."""
    tokens, heads, dim = 20001, 1024, 128
    q = torch.empty(tokens, heads, dim, dtype=torch.float16, device=DEV)
    q[:2], q[-3:] = normal(2, heads, dim).half(), normal(3, heads, dim, seed=1).half()
    positions = torch.arange(tokens, dtype=torch.int32, device=DEV)
    turn = L.Rotation(10000.0 ** (-torch.arange(64, device=DEV) / 64.0))
    ends = [(s, L.qk_rotate(q[s].clone(), None, positions[s].clone(), turn)[0])
            for s in (slice(0, 2), slice(tokens - 3, None))]
    L.qk_rotate(q, None, positions, turn, q_out=q)
    assert all(torch.equal(q[s], want) for s, want in ends)


@pytest.mark.parametrize("new", [2, 40])
def test_adapters_at_the_end_of_a_long_pool(new):
    """2.5e9 weights of B; requests of a few tokens and of more."""
    adapters, k, n, rank = 300, 64, 65536, 128
    a, b = (normal(1, rank, k) / 8).bfloat16(), (normal(1, n, rank, seed=1) / 8).bfloat16()
    pool_a, pool_b = (torch.empty(adapters, *x.shape[1:], dtype=x.dtype, device=DEV) for x in (a, b))
    pool_a[-1], pool_b[-1] = a[0], b[0]
    x, y, starts = normal(new, k, seed=2).half(), normal(new, n, seed=3), ints([0, new])
    want = L.linear_adapters(x, [y], [a], [b], starts, ints([0]), new, outs=[torch.empty_like(y)])[0]
    got = L.linear_adapters(x, [y], [pool_a], [pool_b], starts, ints([adapters - 1]), new, outs=[torch.empty_like(y)])[0]
    assert torch.equal(got, want) and not torch.equal(got, y)


def test_adapters_of_long_outputs():
    """2.2e9 elements of y, in place."""
    tokens, k, n, rank, last = 33001, 64, 65536, 8, 70
    a, b = [(normal(2, rank, k) / 8).half()], [normal(2, n, rank, seed=1).half()]
    x, y = normal(tokens, k, seed=2).half(), torch.zeros(tokens, n, device=DEV)
    y[-last:] = normal(last, n, seed=3)
    want = L.linear_adapters(x[-last:].clone(), [y[-last:].clone()], a, b, ints([0, last]), ints([1]), last)[0]
    L.linear_adapters(x, [y], a, b, ints([0, tokens - last, tokens]), ints([0, 1]), tokens)
    assert torch.equal(y[-last:], want)
