"""Outputs of more than 16 MiB, which are stored past the cache: bit for bit what parts of the call give, whose outputs
are smaller."""
import pytest

from paper_2607_01127_amd import logbq as L

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("tokens,hq,heads,dim,pairs,interleaved", [
    (2101, 32, 8, 128, 64, False), (4200, 32, 2, 64, 16, False), (1301, 28, 4, 256, 96, True)])
def test_streamed_outputs(tokens, hq, heads, dim, pairs, interleaved, dtype):
    print("streamed", tokens, hq, heads, dim, pairs, interleaved, dtype, flush=True)
    g = torch.Generator(device=DEV).manual_seed(tokens)
    draw = lambda h: torch.randn(tokens, h, dim, generator=g, device=DEV).to(dtype)  # noqa: E731
    q, k, v, weight = draw(hq), draw(heads), draw(heads), 1 + 0.2 * torch.randn(dim, generator=g, device=DEV)
    positions = torch.randint(0, 100000, (tokens,), generator=g, device=DEV).int()
    turn = L.Rotation(10000.0 ** (-torch.arange(pairs, device=DEV) / pairs), interleaved)
    page = 64
    pages = -(-tokens // page) + 1
    slots = torch.randperm(pages * page, generator=g, device=DEV)[:tokens]
    slots[11] = -1
    parts = [slice(a, a + 500) for a in range(0, tokens, 500)]
    assert tokens * hq * dim * 2 > 16 << 20 and 500 * (hq + heads) * dim * 4 <= 16 << 20
    whole, pieces = L.kv4_cache(pages, heads, dim, page), L.kv4_cache(pages, heads, dim, page)
    got = L.kv4_append_rotated(q, k, v, whole, slots, positions, turn, weight, weight)
    want = torch.cat([L.kv4_append_rotated(q[s], k[s], v[s], pieces, slots[s], positions[s], turn, weight, weight)
                      for s in parts])
    assert torch.equal(got, want) and torch.isfinite(got).all()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(whole, pieces))
    got = L.qk_rotate(q, k, positions, turn, weight, weight)
    want = zip(*(L.qk_rotate(q[s], k[s], positions[s], turn, weight, weight) for s in parts))
    assert all(torch.equal(a, torch.cat(b)) for a, b in zip(got, want))
    again, _ = L.qk_rotate(q, None, positions, turn, weight, q_out=q)       # in place
    assert again is q and torch.equal(q, got[0])
