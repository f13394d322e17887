"""The serving example: its step's operators together, against the same decoder in plain float32
torch, and its two ways through the cache (a prompt at once, or token by token)."""
import pytest

from paper_2607_01127_amd import logbq as L

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def plain_logits(d, tokens):
    """The decoder on one sequence in float32, with the codes' weights and the 4-bit values of keys
    and values (as the cache gives them back)."""
    s, x = d.shape, d.embedding[tokens].float()
    pos = torch.arange(len(tokens), device=x.device)
    w = lambda lin, name: L.dequantize(*lin[name])  # noqa: E731
    for lin, _ in d.layers:
        h = d._norm(x).float()
        q = d._rotate((h @ w(lin, "q").T).view(len(tokens), s.heads, s.dim), pos)
        k = d._rotate((h @ w(lin, "k").T).view(len(tokens), s.kv_heads, s.dim), pos)
        v = (h @ w(lin, "v").T).view(len(tokens), s.kv_heads, s.dim)
        cache = L.kv4_cache(-(-len(tokens) // 64), s.kv_heads, s.dim, 64)
        L.kv4_append(k, v, cache, pos)
        k, v = L.kv4_read(cache, pos, torch.float32)
        k, v = (y.repeat_interleave(s.heads // s.kv_heads, 1).transpose(0, 1).contiguous() for y in (k, v))
        score = q.transpose(0, 1).contiguous() @ k.transpose(1, 2).contiguous() * s.dim ** -0.5
        score.masked_fill_(pos[None, None] > pos[None, :, None], float("-inf"))
        a = (torch.softmax(score, -1) @ v).transpose(0, 1).reshape(len(tokens), -1)
        x = x + a @ w(lin, "o").T
        h = d._norm(x).float()
        x = x + (torch.nn.functional.silu(h @ w(lin, "gate").T) * (h @ w(lin, "up").T)) @ w(lin, "down").T
    return d._norm(x).float() @ d.head.float().T


def test_example_against_plain_torch_and_itself():
    """Tolerance: activations are rounded to float16 between operators (2^-11 of themselves, about
    ten times along the two layers), and a key or value that lies near a threshold may take the
    neighbouring code, a change of up to a quarter of one of 64 channels; both leave the logits
    (standard deviation about 1) within a few hundredths, so 0.1 for the mean and 0.5 for any one."""
    from paper_2607_01127_amd.serve_example import Batch, Decoder, Shape
    d = Decoder(Shape(), pages=32, page=64, seed=3)
    g = torch.Generator().manual_seed(1)
    texts = [torch.randint(0, 1000, (n,), generator=g).tolist() for n in (130, 1, 67)]
    together = Batch(d, 3, 256).step(texts)
    plain = torch.cat([plain_logits(d, torch.tensor(t, device="cuda")) for t in texts])
    off = (together - plain).abs()
    assert off.mean() < 0.1 and off.max() < 0.5, (off.mean(), off.max())
    # The same texts a few tokens at a time: chunks, single tokens and idle requests in one batch.
    batch, parts = Batch(d, 3, 256), [[], [], []]
    at = [0, 0, 0]
    for take in ((50, 1, 3), (1, 0, 1), (30, 0, 1), (1, 0, 2), (48, 0, 60)):
        step = [t[a:a + n] for t, a, n in zip(texts, at, take)]
        rows = batch.step(step).split([len(x) for x in step])
        at = [a + n for a, n in zip(at, take)]
        for r in range(3):
            parts[r].append(rows[r])
    off = (torch.cat([torch.cat(p) for p in parts]) - together).abs()
    assert off.mean() < 0.1 and off.max() < 0.5, (off.mean(), off.max())


def test_example_generates_and_scores():
    from paper_2607_01127_amd.serve_example import Batch, Decoder, Shape
    d = Decoder(Shape(layers=1), pages=16, page=16, seed=4)
    prompts = [[1, 2, 3], list(range(40))]
    chosen, logprobs, entropies, last = Batch(d, 2, 64).generate(prompts, 5)
    assert [len(c) for c in chosen] == [5, 5] and logprobs.shape == entropies.shape == (2, 5)
    # Greedy: the chosen token is the first alternative, with the same log probability.
    assert last["top_index"][:, 0].tolist() == [c[-1] for c in chosen]
    assert torch.equal(last["top_logprob"][:, 0], logprobs[:, -1])
    assert bool((logprobs <= 0).all()) and bool((entropies >= 0).all())
    # Scoring a prompt with its continuation gives the continuation's log probabilities again.
    whole = [p + c for p, c in zip(prompts, chosen)]
    score = Batch(d, 2, 64).score(whole).split([len(w) - 1 for w in whole])
    for s, lp in zip(score, logprobs):
        assert float((s[-5:] - lp).abs().max()) < 0.5
    with pytest.raises(ValueError):
        Batch(d, 1, 32).step([list(range(33))])
