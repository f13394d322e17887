"""Which tokens drafts leave: exactly those of greedy decoding, in as few steps as the drafts allow, within the room that
greedy decoding needs. The decoder is one whose next token is a whole number made of all that a token sees and of where
it stands, as the cache holds them, so that nothing depends on a rounding."""
import numpy as np
import pytest

from paper_2607_01127_amd import logbq as L

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"
VOCAB, BITS = 1000, 11


def sums(seen):
    """The next token after (token, position) pairs; its texts come to repeat one token."""
    return sum((t + 1) * (7 * p + 3) for t, p in seen) % VOCAB


def powers(seen):
    """One whose texts do not."""
    return sum(pow(t + 2, p % 5 + 2, 991) * (7 * p + 3) for t, p in seen) % 991


def greedy(text, steps, rule=sums):
    text, n = list(text), len(text)
    for _ in range(steps):
        text.append(rule(list(zip(text, range(len(text))))))
    return text[n:]


class Counting:
    """Stands where a Decoder does; keys and values are the bits of tokens and positions, which the 4-bit cache holds
    exactly (0 and 6 times a scale of 1)."""

    def __init__(self, pages, page, rule=sums):
        self.rule = rule
        self.page, self.device = page, DEV
        self.layers = [(None, L.kv4_cache(pages, 1, 64, page, DEV)) for _ in range(2)]
        self.free = torch.randperm(pages, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV).int()
        self.used = 0

    def step(self, tokens, tables, max_new, adapters=None, adapter=None):
        t = tokens.cpu().numpy()
        places = tables["positions"].cpu().numpy()
        rows = np.zeros((len(t), 1, 64), dtype=np.float32)
        rows[:, 0, 63] = 6
        for i in range(BITS):
            rows[:, 0, i], rows[:, 0, 20 + i] = 6 * (t >> i & 1), 6 * (places >> i & 1)
        rows = torch.from_numpy(rows).to(DEV)
        for _, cache in self.layers:
            L.kv4_append(rows, rows.flip(-1), cache, tables["slots"])
        table, starts = tables["table"].cpu().numpy(), tables["q_starts"].tolist()
        masks = tables["masks"].cpu().numpy().view(np.uint64) if "masks" in tables else None
        logits = torch.zeros(len(t), VOCAB, device=DEV)
        for r, length in enumerate(tables["seq_lens"].tolist()):
            a, b = starts[r], starts[r + 1]
            if a == b:
                continue
            at = np.arange(length)
            slots = torch.from_numpy(table[r, at // self.page].astype(np.int64) * self.page + at % self.page).to(DEV)
            held = []
            for _, cache in self.layers:
                k, v = L.kv4_read(cache, slots)
                assert torch.equal(k, v.flip(-1))
                bits = (k[:, 0].cpu().numpy() / 6).astype(np.int64)
                held.append([(int(x[:BITS] @ (1 << np.arange(BITS))), int(x[20:20 + BITS] @ (1 << np.arange(BITS)))) for x in bits])
            assert held[0] == held[1]
            cached = length - (b - a)
            # What earlier steps left is a text: each position once, in order.
            assert [p for _, p in held[0][:cached]] == list(range(cached))
            for i in range(b - a):
                bits = (2 << i) - 1 if masks is None else int(masks[a + i])
                seen = held[0][:cached] + [held[0][cached + j] for j in range(b - a) if bits >> j & 1]
                assert sorted(p for _, p in seen) == list(range(len(seen)))
                logits[a + i, self.rule(seen)] = 1.0
        return logits


def drafts(prompts, steps, shape, rule=sums):
    """A draft of the text's true continuation: shape(rest) makes (tokens, parents) below the root from it."""
    whole = [list(p) + greedy(p, steps + 40, rule) for p in prompts]

    def draft(text):
        text = list(text)
        rest = next(w for w in whole if w[:len(text)] == text)[len(text):]
        tokens, parents = shape(rest)
        return [text[-1]] + tokens, [-1] + parents
    return draft


def wrong(t):
    return (t + 1) % VOCAB


SHAPES = {
    "none": lambda rest: ([], []),
    "wrong": lambda rest: ([wrong(t) for t in rest[:5]], [0, 1, 2, 3, 4]),
    "chain of 4": lambda rest: (rest[:4], [0, 1, 2, 3]),
    # Wrong ones first and beside, and a wrong one with right ones below it.
    "beside": lambda rest: ([wrong(rest[0]), rest[0], wrong(rest[1]), rest[1], rest[2], rest[1]], [0, 0, 2, 2, 4, 1]),
    # Right tokens that hang from the wrong place.
    "elsewhere": lambda rest: ([rest[0], rest[2], rest[1], rest[2]], [0, 1, 0, 3]),
}


def steps_needed(prompt, steps, draft, rule):
    """A step adds one token and, before it, the longest path below the root that is the text's continuation."""
    whole, taken = list(prompt) + greedy(prompt, steps + 40, rule), 1
    at = len(prompt) + 1
    while at < len(prompt) + steps:
        tokens, parents = draft(whole[:at])
        most = 0
        for node in range(1, len(tokens)):
            path = []
            while node:
                path.insert(0, tokens[node])
                node = parents[node]
            if path == whole[at:at + len(path)]:
                most = max(most, len(path))
        at, taken = at + most + 1, taken + 1
    return taken


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("steps", [1, 2, 9, 30])
@pytest.mark.parametrize("rule", [sums, powers])
def test_chosen_tokens_and_steps(rule, steps, shape, page):
    from paper_2607_01127_amd.serve_example import Batch
    prompts = [[5, 6, 7] * 10, [9], list(range(300, 316))]
    d = Counting(40, page, rule)
    draft = drafts(prompts, steps, SHAPES[shape], rule)
    chosen, taken = Batch(d, 3, 192).speculate(prompts, steps, draft)
    assert chosen == [greedy(p, steps, rule) for p in prompts]
    assert taken == max(steps_needed(p, steps, draft, rule) for p in prompts)


def test_generate_is_greedy_too():
    from paper_2607_01127_amd.serve_example import Batch
    prompts = [[5, 6, 7] * 10, [9]]
    batch = Batch(Counting(20, 16), 2, 64)
    batch.decoder.lp_work = torch.zeros(L.LOGPROBS_WORKSPACE_BYTES, dtype=torch.uint8, device=DEV)
    assert batch.generate(prompts, 9)[0] == [greedy(p, 9) for p in prompts]


@pytest.mark.parametrize("page", [16, 32])
def test_requests_that_are_done_take_no_room(page):
    """One draft is right and another wrong, so one request has its tokens long before the other; tables and pages hold
    no more than greedy decoding needs."""
    from paper_2607_01127_amd.serve_example import Batch
    prompts, steps = [[3] * 20, [8, 1]], 13
    right, never = drafts(prompts, steps, SHAPES["chain of 4"]), drafts(prompts, steps, SHAPES["wrong"])
    pages = sum(-(-(len(p) + steps - 1) // page) for p in prompts)
    d = Counting(pages, page)
    batch = Batch(d, 2, 20 + steps - 1)
    chosen, taken = batch.speculate(prompts, steps, lambda text: (right if text[0] == 3 else never)(text))
    assert chosen == [greedy(p, steps) for p in prompts] and taken == steps
    assert batch.lengths == [len(p) + steps - 1 for p in prompts] and d.used == pages
    held = torch.cat([batch.table[batch.table >= 0], d.free[d.used:]])
    assert sorted(held.tolist()) == list(range(pages))


@pytest.mark.parametrize("spare", [0, 1, 3])
def test_large_drafts_in_little_room(spare):
    """Trees of 64 nodes where the table or the free pages end: what greedy decoding has room for works."""
    from paper_2607_01127_amd.serve_example import Batch
    prompts, steps, page = [[3] * 30, [8] * 15, [2]], 20, 16
    full = lambda rest: (rest[:3] + [wrong(rest[0])] * 60, [0, 1, 2] + [0] * 60)  # noqa: E731
    pages = sum(-(-(len(p) + steps - 1) // page) for p in prompts)
    batch = Batch(Counting(pages + spare, page), 3, 49)
    chosen, taken = batch.speculate(prompts, steps, drafts(prompts, steps, full))
    assert chosen == [greedy(p, steps) for p in prompts] and taken < steps
    assert batch.lengths == [len(p) + steps - 1 for p in prompts] and batch.decoder.used == pages


def test_a_draft_without_a_root_is_refused():
    from paper_2607_01127_amd.serve_example import Batch
    with pytest.raises(ValueError):
        Batch(Counting(20, 16), 1, 64).speculate([[1, 2]], 4, lambda text: ([], []))


def test_a_decoder_s_tokens_are_its_greedy_ones():
    """Every chosen token against one pass over the prompt with the chosen tokens: its logit is the row's largest, but
    for what the steps' roundings can move two logits by (0.5 each, as in the example's other tests)."""
    from paper_2607_01127_amd.serve_example import Batch, Decoder, Shape
    d = Decoder(Shape(layers=1), pages=300, page=16, seed=7)
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, 1000, (n,), generator=g).tolist() for n in (20, 3)]
    plain = Batch(d, 2, 128).generate(prompts, 9)[0]

    def known(text):
        whole = next((p + c for p, c in zip(prompts, plain) if (p + c)[:len(text)] == list(text)), list(text))
        rest = whole[len(text):][:4]
        bad = [wrong(t) for t in rest]
        return [text[-1]] + bad + rest, [-1] + [0] * len(bad) + [len(bad) + i if i else 0 for i in range(len(rest))]

    seen = []
    for draft in (lambda text: ([text[-1]], [-1]), known, lambda text: ([text[-1], wrong(plain[0][0])], [-1, 0])):
        chosen, taken = Batch(d, 2, 128).speculate(prompts, 9, draft)
        for p, c in zip(prompts, chosen):
            rows = Batch(d, 1, 128).step([p + c[:-1]])[len(p) - 1:]
            assert len(c) == 9 and float((rows.amax(1) - rows[torch.arange(9), torch.tensor(c)]).max()) < 1.0
        seen.append((chosen, taken))
    assert seen[0][1] == 9
    if seen[1][0] == plain:                      # else two near logits fell the other way, which ends a draft
        assert seen[1][1] == 3
