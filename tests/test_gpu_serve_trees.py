"""The serving example's steps with drafted trees and adapters: their operators together, as they would be used.
Tolerances of logits as in the example's other tests: activations rounded to float16 between operators, and keys or
values that take the neighbouring code, leave them within 0.1 in the mean and 0.5 for any one."""
import pytest

from paper_2607_01127_amd import logbq as L

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def near(a, b):
    off = (a - b).abs()
    assert off.mean() < 0.1 and off.max() < 0.5, (off.mean(), off.max())


def texts(*lengths, seed=1):
    g = torch.Generator().manual_seed(seed)
    return [torch.randint(0, 1000, (n,), generator=g).tolist() for n in lengths]


TREES = [([7, 300, 4, 5, 6, 4], [-1, 0, 0, 1, 1, 3]), ([9], [-1]), ([1, 2, 3, 4], [-1, -1, 1, 0])]


def path_of(parents, node):
    path = [node]
    while parents[path[0]] >= 0:
        path.insert(0, parents[path[0]])
    return path


def test_a_node_sees_its_path():
    """The logits of a node are those of the text continued along its path."""
    from paper_2607_01127_amd.serve_example import Batch, Decoder, Shape
    d = Decoder(Shape(), pages=120, page=16, seed=3)
    prompts = texts(130, 1, 67)
    batch = Batch(d, 3, 256)
    batch.step(prompts)
    rows = batch.step([t for t, _ in TREES], [p for _, p in TREES]).split([len(t) for t, _ in TREES])
    for text, (tokens, parents), got in zip(prompts, TREES, rows):
        for node in range(len(tokens)):
            path = path_of(parents, node)
            near(got[node], Batch(d, 1, 256).step([text + [tokens[i] for i in path]])[-1])


def test_kept_paths_are_text():
    """After a path is kept the requests go on as if it had been their text; pages of the others come back."""
    from paper_2607_01127_amd.serve_example import Batch, Decoder, Shape
    d = Decoder(Shape(layers=1), pages=80, page=16, seed=5)
    prompts = texts(31, 1, 16)
    batch = Batch(d, 3, 128)
    batch.step(prompts)
    used = d.used
    batch.step([t for t, _ in TREES], [p for _, p in TREES])
    assert d.used == used + 2                  # 31 + 6 and 16 + 4 tokens open a page each
    paths = [[0, 1, 3, 5], [0], []]
    batch.keep(paths)
    assert batch.lengths == [35, 2, 16] and d.used == used + 1 and int((batch.table >= 0).sum()) == d.used
    held = torch.cat([batch.table[batch.table >= 0], d.free[d.used:]])
    assert sorted(held.tolist()) == list(range(80))
    whole = [t + [tree[i] for i in p] for t, (tree, _), p in zip(prompts, TREES, paths)]
    again = Batch(d, 3, 128)
    again.step(whole)
    near(batch.step([[11, 12], [13], [14]]), again.step([[11, 12], [13], [14]]))
    # The values moved without loss: what the last request keeps of its cache is as before.
    cache = d.layers[0][1]
    slots = torch.arange(80 * 16, device="cuda")
    before = [x.clone() for x in cache]
    L.kv4_append(*L.kv4_read(cache, slots, torch.float32), cache, slots)
    assert all(torch.equal(a, b) for a, b in zip(before, cache))


def test_drafts_are_checked_by_greedy_decoding():
    """With drafts that hold the answer a step keeps all of it; with drafts that do not, one token."""
    from paper_2607_01127_amd.serve_example import Batch, Decoder, Shape, repeated
    d = Decoder(Shape(layers=1), pages=200, page=16, seed=7)
    prompts = texts(20, 3)
    first, taken = Batch(d, 2, 128).speculate(prompts, 9, lambda text: ([text[-1]], [-1]))
    assert taken == 9 and [len(c) for c in first] == [9, 9]
    answers = {tuple(p): c for p, c in zip(prompts, first)}

    def known(text):
        """The answer's next four tokens below the root, beside wrong ones."""
        p = next(p for p in answers if list(p) == text[:len(p)])
        rest = answers[p][len(text) - len(p):][:4]
        wrong = [(t + 1) % 1000 for t in rest]
        up = [0] * len(wrong) + [len(wrong) + i if i else 0 for i in range(len(rest))]
        return [text[-1]] + wrong + rest, [-1] + up

    drafted, taken = Batch(d, 2, 128).speculate(prompts, 9, known)
    # Trees and single tokens round differently, so a choice between two near logits may fall the other way.
    same = sum(a == b for x, y in zip(drafted, first) for a, b in zip(x, y))
    assert taken < 9 or same < 18
    assert [len(c) for c in drafted] == [9, 9]
    assert len(Batch(d, 2, 128).speculate(prompts, 5, repeated)[0][0]) == 5
    for bad in (([[1], []], 2), ([[1], [2]], 0)):
        with pytest.raises(ValueError):
            Batch(d, 2, 64).speculate(*bad, repeated)


def test_the_draft_from_the_text():
    from paper_2607_01127_amd.serve_example import repeated
    assert repeated([5]) == ([5], [-1])
    assert repeated([5, 6, 7, 5, 6, 8, 5], 2, 2) == ([5, 6, 8, 7], [-1, 0, 1, 1])


def plain_logits(d, tokens, merged):
    """The decoder on one sequence in float32, with the adapter merged into its query, key and value weights."""
    s, x = d.shape, d.embedding[tokens].float()
    pos = torch.arange(len(tokens), device=x.device)
    for i, (lin, _) in enumerate(d.layers):
        w = {n: L.dequantize(*lin[n]) for n in lin}
        for n, delta in zip("qkv", merged[i]):
            w[n] = w[n] + delta
        h = d._norm(x).float()
        q = d._rotate((h @ w["q"].T).view(len(tokens), s.heads, s.dim), pos)
        k = d._rotate((h @ w["k"].T).view(len(tokens), s.kv_heads, s.dim), pos)
        v = (h @ w["v"].T).view(len(tokens), s.kv_heads, s.dim)
        cache = L.kv4_cache(-(-len(tokens) // 64), s.kv_heads, s.dim, 64)
        L.kv4_append(k, v, cache, pos)
        k, v = L.kv4_read(cache, pos, torch.float32)
        k, v = (y.repeat_interleave(s.heads // s.kv_heads, 1).transpose(0, 1).contiguous() for y in (k, v))
        score = q.transpose(0, 1).contiguous() @ k.transpose(1, 2).contiguous() * s.dim ** -0.5
        score.masked_fill_(pos[None, None] > pos[None, :, None], float("-inf"))
        a = (torch.softmax(score, -1) @ v).transpose(0, 1).reshape(len(tokens), -1)
        x = x + a @ w["o"].T
        h = d._norm(x).float()
        x = x + (torch.nn.functional.silu(h @ w["gate"].T) * (h @ w["up"].T)) @ w["down"].T
    return d._norm(x).float() @ d.head.float().T


def test_adapters_of_several_requests():
    """A step with adapters against merged weights; a request without one, and the same adapter twice."""
    from paper_2607_01127_amd.serve_example import Adapters, Batch, Decoder, Shape
    d = Decoder(Shape(), pages=60, page=64, seed=3)
    ranks, ids = (8, 5, 16), (1, -1, 2, 1)
    adapters = Adapters(d, ranks, scale=0.5, seed=2)
    prompts = texts(90, 40, 1, 33)
    got = Batch(d, 4, 256, adapters, ids).step(prompts).split([len(p) for p in prompts])
    plain = []
    for text, i in zip(prompts, ids):
        merged = [[0.0] * 3 if i < 0 else [0.5 * b[i, :, :ranks[i]].float() @ a[i, :ranks[i]].float()
                                           for a, b in zip(*layer)] for layer in adapters.layers]
        plain.append(plain_logits(d, torch.tensor(text, device="cuda"), merged))
    near(torch.cat(list(got)), torch.cat(plain))
    # One token at a time after the prompt, and as drafts.
    batch = Batch(d, 4, 256, adapters, ids)
    batch.step([p[:-1] or p for p in prompts])
    rows = batch.step([p[-1:] if len(p) > 1 else [] for p in prompts])
    near(rows, torch.stack([g[-1] for g, p in zip(got, prompts) if len(p) > 1]))
    chosen, _ = Batch(d, 4, 256, adapters, ids).speculate(prompts, 4, lambda text: ([text[-1], 1, 2], [-1, 0, 0]))
    assert [len(c) for c in chosen] == [4] * 4
