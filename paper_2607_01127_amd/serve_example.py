"""A small decoder served with this library: 4-bit linears with low-rank adapters beside them, a paged 4-bit
key/value cache, attention over it, drafted trees, and the log probabilities of what it answers.

    python -m paper_2607_01127_amd.serve_example

The decoder is Llama-style (RMS norm, rotary embedding, grouped key/value heads, gated MLP) with
random weights, each projection quantized with its own codebook; the embedding and the output head
stay in 16 bits, as in the paper (Sec. 4). A step is what a serving program runs for any mixture of
prompts and single tokens:

    batch_tables -> for each layer: linear_multi (q, k, v), linear_adapters, kv4_append_rotated,
    kv4_attention, linear (o), linear_multi (gate, up), linear (down) -> output head, token_logprobs

A step of drafted trees (speculative decode) takes its positions from tree_tables and kv4_tree_attention for
the attention. Nothing in a step waits for the GPU; the lengths that the host needs are its own.
"""
from __future__ import annotations

import math
from dataclasses import dataclass

import torch

from . import inputs
from . import logbq as L


@dataclass(frozen=True)
class Shape:
    hidden: int = 512
    inter: int = 1024
    heads: int = 8
    kv_heads: int = 2
    dim: int = 64
    layers: int = 2
    vocab: int = 1000


class Decoder:
    """Random weights of a shape, and the caches of its layers."""

    def __init__(self, shape: Shape, pages: int, page: int = 64, seed: int = 0, device="cuda"):
        self.shape, self.page, self.device = shape, page, device
        s, g = shape, torch.Generator(device=device).manual_seed(seed)
        kv = s.kv_heads * s.dim
        sizes = dict(q=(s.heads * s.dim, s.hidden), k=(kv, s.hidden), v=(kv, s.hidden),
                     o=(s.hidden, s.heads * s.dim), gate=(s.inter, s.hidden),
                     up=(s.inter, s.hidden), down=(s.hidden, s.inter))
        self.layers = []
        for layer in range(s.layers):
            lin = {}
            for name, (n, k) in sizes.items():
                w = inputs.student_t_weights(n, k, 4, 0.7 / math.sqrt(k), [seed, layer, inputs.PROJ[name], 0],
                                             device=device)
                p = L.fit_device(w)
                lin[name] = L.encode(w, p)               # (codes, codebook)
            self.layers.append((lin, L.kv4_cache(pages, s.kv_heads, s.dim, page, device)))
        self.embedding = torch.randn((s.vocab, s.hidden), generator=g, device=device).half()
        self.head = (torch.randn((s.vocab, s.hidden), generator=g, device=device) * s.hidden ** -0.5).half()
        self.rotation = 10000.0 ** (-torch.arange(0, s.dim, 2, device=device).float() / s.dim)
        self.turn = L.Rotation(self.rotation)
        self.free = torch.randperm(pages, generator=g, device=device).int()      # ids of pages
        self.used = 0                      # the first of them, which its batches have taken
        self.kv_work = torch.empty(L.KV4_WORKSPACE_BYTES, dtype=torch.uint8, device=device)
        self.lp_work = torch.zeros(L.LOGPROBS_WORKSPACE_BYTES, dtype=torch.uint8, device=device)

    def _norm(self, x):
        return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5)).half()

    def _rotate(self, x, positions):
        angle = positions[:, None, None].float() * self.rotation
        a, b = x.float().chunk(2, -1)
        c, s = angle.cos(), angle.sin()
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    def step(self, tokens, tables, max_new: int, adapters=None, adapter=None):
        """float32 logits [tokens][vocab] of the step's tokens, whose keys and values go into the
        caches; `tables` is batch_tables' result with the block table as "table", and with tree_tables'
        masks and positions where the tokens are the nodes of drafts. `adapters` (Adapters) go to the
        requests by `adapter` (int32 [requests])."""
        s, t = self.shape, tokens.numel()
        x = self.embedding[tokens].float()
        lengths = (tables["table"], tables["seq_lens"], tables["q_starts"])
        for i, (lin, cache) in enumerate(self.layers):
            h = self._norm(x)
            qkv = L.linear_multi(h, *zip(*(lin[n] for n in ("q", "k", "v"))))
            if adapters is not None:
                L.linear_adapters(h, qkv, *adapters.layers[i], tables["q_starts"], adapter, max_new,
                                  scales=adapters.scales, ranks=adapters.ranks)
            q, k, v = (y.view(t, -1, s.dim) for y in qkv)
            q = L.kv4_append_rotated(q, k, v, cache, tables["slots"], tables["positions"], self.turn,
                                     q_out=q if q.is_contiguous() else None)
            if "masks" in tables:
                a = L.kv4_tree_attention(q, cache, *lengths, tables["masks"], max_new, workspace=self.kv_work)
            else:
                a = L.kv4_attention(q, cache, *lengths, max_new, workspace=self.kv_work)
            x = x + L.linear(a.view(t, -1), *lin["o"])
            gate, up = L.linear_multi(self._norm(x), *zip(*(lin[n] for n in ("gate", "up"))))
            x = x + L.linear((torch.nn.functional.silu(gate) * up).half(), *lin["down"])
        return (self._norm(x) @ self.head.T).float()


class Adapters:
    """Random low-rank adapters beside a decoder's query, key and value projections. They share a pool of
    `rank` ranks; `ranks` says how many each has."""

    def __init__(self, decoder: Decoder, ranks, scale: float = 1.0, seed: int = 0, dtype=torch.bfloat16):
        s, device = decoder.shape, decoder.device
        g = torch.Generator(device=device).manual_seed(seed)
        rank, n = -(-max(ranks) // 8) * 8, len(ranks)
        self.ranks = torch.tensor(ranks, dtype=torch.int32).to(device)
        self.scales = torch.full((n,), scale, device=device)
        draw = lambda *shape: torch.randn(shape, generator=g, device=device)  # noqa: E731
        self.layers = []
        for _ in range(s.layers):
            widths = [s.heads * s.dim, s.kv_heads * s.dim, s.kv_heads * s.dim]
            self.layers.append(([(draw(n, rank, s.hidden) * s.hidden ** -0.5).to(dtype) for _ in widths],
                                [(draw(n, w, rank) * rank ** -0.5).to(dtype) for w in widths]))


class Batch:
    """Requests that are served together. The host keeps their lengths. Pages are taken from the decoder
    for good, so that batches of one decoder may live side by side. `adapter` names each request's adapter
    of `adapters` (negative: none)."""

    def __init__(self, decoder: Decoder, requests: int, most: int, adapters: Adapters = None, adapter=None):
        self.decoder = decoder
        self.lengths = [0] * requests
        width = -(-most // decoder.page)
        self.table = torch.full((requests, width), -1, dtype=torch.int32, device=decoder.device)
        self.adapters = adapters
        self.adapter = None if adapters is None else torch.tensor(adapter, dtype=torch.int32).to(decoder.device)

    def step(self, new_tokens, parents=None):
        """One step: a list of token lists (one a request, empty for none) -> logits of all of them
        in order. With `parents` (a list of lists, indexes among the request's tokens, negative for
        none) the tokens are the nodes of drafted trees, at most 64 a request."""
        d, page = self.decoder, self.decoder.page
        new = [len(x) for x in new_tokens]
        ints = torch.tensor([self.lengths, new], dtype=torch.int32).to(d.device)
        tokens = torch.tensor(sum(new_tokens, []), dtype=torch.int64).to(d.device)
        pages = sum(-(-(a + b) // page) - -(-a // page) for a, b in zip(self.lengths, new))
        total = [a + b for a, b in zip(self.lengths, new)]
        if max(total) > self.table.shape[1] * page or d.used + pages > d.free.numel():
            raise ValueError("the cache or the block table is too small for this step")
        tables = L.batch_tables(ints[0], ints[1], d.free[d.used:], self.table, page, len(tokens))
        if parents is not None:
            up = torch.tensor(sum(parents, []), dtype=torch.int32).to(d.device)
            tables.update(L.tree_tables(up, tables["q_starts"], tables["seq_lens"]))
        self.slots, self.nodes = tables["slots"], new
        logits = d.step(tokens, dict(tables, table=self.table), max(new), self.adapters, self.adapter)
        self.lengths, d.used = total, d.used + pages
        return logits

    def keep(self, paths):
        """After a step of trees: of each request's nodes, those of `paths` (lists of indexes, rising) stay,
        as its next cached tokens in order; the pages that only others had go back. What the cache holds
        reads back exactly and is appended as the same codes, so keys and values move without loss."""
        d, page = self.decoder, self.decoder.page
        at, source, to, left, lengths = 0, [], [], [], []
        for r, (total, path) in enumerate(zip(self.lengths, paths)):
            nodes = self.nodes[r]
            source += [at + i for j, i in enumerate(path) if i != j]
            to += [at + j for j, i in enumerate(path) if i != j]
            at += nodes
            lengths.append(total - nodes + len(path))
            left += [(r, c) for c in range(-(-lengths[-1] // page), -(-total // page))]
        if source:
            source, to = (self.slots[torch.tensor(i).to(d.device)] for i in (source, to))
            for _, cache in d.layers:
                L.kv4_append(*L.kv4_read(cache, source, torch.float32), cache, to)
        if left:
            rows, columns = (torch.tensor(i).to(d.device) for i in zip(*left))
            d.free[d.used - len(left):d.used] = self.table[rows, columns]
            self.table[rows, columns] = -1
            d.used -= len(left)
        self.lengths = lengths

    def _within_room(self, trees):
        """Of each tree the first nodes, which are a tree too: those that the block table has room for, and where
        the decoder has too few free pages for all of them, those that need none (the roots aside)."""
        d, page = self.decoder, self.decoder.page
        most = self.table.shape[1] * page
        left = [max(1, most - n) for n in self.lengths]
        trees = [(t[:m], p[:m]) for m, (t, p) in zip(left, trees)]
        pages = sum(-(-(n + len(t)) // page) - -(-n // page) for n, (t, _) in zip(self.lengths, trees))
        if d.used + pages > d.free.numel():
            own = [max(1, -n % page) for n in self.lengths]
            trees = [(t[:m], p[:m]) for m, (t, p) in zip(own, trees)]
        return trees

    def speculate(self, prompts, steps: int, draft):
        """Greedy continuation with drafts: draft(text) gives (tokens, parents) of a tree whose root,
        node 0, is the text's last token; of the drafted tokens below it the longest path that greedy
        decoding would have taken stays. Drafts are cut to the room that there is, so whatever generate
        has room for works, and a request that has its tokens takes no further part. Returns the chosen
        tokens (`steps` of each request, a list of lists) and the number of steps that it took."""
        if steps < 1 or not all(prompts):
            raise ValueError("speculate needs a step and a token of each prompt")
        logits = self.step(prompts)
        ends = torch.tensor([len(p) for p in prompts]).cumsum(0) - 1
        chosen, taken = [[t] for t in logits[ends.to(self.decoder.device)].argmax(1).tolist()], 1
        while min(len(c) for c in chosen) < steps:
            trees = [draft(p + c) if len(c) < steps else ([], []) for p, c in zip(prompts, chosen)]
            if any(len(c) < steps and not t for c, (t, _) in zip(chosen, trees)):
                raise ValueError("a draft has its root at least")
            trees = self._within_room(trees)
            best = self.step([t for t, _ in trees], [p for _, p in trees]).argmax(1).tolist()
            taken += 1
            paths, at = [], 0
            for c, (tokens, parents) in zip(chosen, trees):
                path = [0] if tokens else []
                while path:
                    answer = best[at + path[-1]]
                    c.append(answer)
                    below = [i for i in range(path[-1] + 1, len(tokens))
                             if parents[i] == path[-1] and tokens[i] == answer]
                    if not below or len(c) == steps:
                        break
                    path.append(below[0])
                paths.append(path)
                at += len(tokens)
            self.keep(paths)
        return chosen, taken

    def generate(self, prompts, steps: int, top: int = 5):
        """Greedy continuation: the chosen tokens [requests][steps] (a list of lists), their log
        probabilities and entropies, and the alternatives of the last step. Each request begins with a
        token at least."""
        if steps < 1 or not all(prompts):
            raise ValueError("generate needs a step and a token of each prompt")
        d = self.decoder
        logits = self.step(prompts)
        ends = torch.tensor([len(p) for p in prompts]).cumsum(0) - 1
        logits = logits[ends.to(d.device)]
        chosen, logprobs, entropies = [[] for _ in prompts], [], []
        for i in range(steps):
            best = logits.argmax(1)
            got = L.token_logprobs(logits, best, top, workspace=d.lp_work)
            logprobs.append(got["logprob"])
            entropies.append(got["entropy"])
            for r, token in enumerate(best.tolist()):        # the answer leaves the GPU here
                chosen[r].append(token)
            if i + 1 < steps:
                logits = self.step([[c[-1]] for c in chosen])
        return chosen, torch.stack(logprobs, 1), torch.stack(entropies, 1), got

    def score(self, texts):
        """Log probabilities of the texts' own tokens but the first (float32 [sum of lengths - 1])."""
        logits = self.step(texts)
        keep = torch.tensor([i for i, last in enumerate(j + 1 == len(t) for t in texts for j in range(len(t)))
                             if not last], dtype=torch.int64).to(logits.device)
        targets = torch.tensor([token for t in texts for token in t[1:]], dtype=torch.int64).to(logits.device)
        return L.token_logprobs(logits[keep], targets, workspace=self.decoder.lp_work)["logprob"]


def repeated(text, branches: int = 3, length: int = 4):
    """A draft from the text itself: what followed the last token before, the latest places first."""
    tokens, parents = [text[-1]], [-1]
    places = [i for i in range(len(text) - 2, -1, -1) if text[i] == text[-1]][:branches]
    for place in places:
        at = 0
        for token in text[place + 1:place + 1 + length]:
            same = [i for i in range(1, len(tokens)) if parents[i] == at and tokens[i] == token]
            if not same:
                tokens.append(token)
                parents.append(at)
            at = same[0] if same else len(tokens) - 1
    return tokens, parents


def main():
    decoder = Decoder(Shape(), pages=64)
    prompts = [list(range(5, 105)), [7, 8, 9], list(range(300, 377))]
    chosen, logprobs, entropies, last = Batch(decoder, len(prompts), 512).generate(prompts, steps=16)
    for r, tokens in enumerate(chosen):
        print(f"request {r}: {tokens}")
        print(f"  log probabilities {[round(x, 2) for x in logprobs[r].tolist()]}")
    score = Batch(decoder, len(prompts), 512).score(prompts)
    drafted, taken = Batch(decoder, len(prompts), 512).speculate(prompts, 16, repeated)
    same = sum(a == b for a, b in zip(sum(drafted, []), sum(chosen, [])))
    print(f"with drafts: {same} of {16 * len(prompts)} tokens alike in {taken} steps")
    adapted = Batch(decoder, len(prompts), 512, Adapters(decoder, (8, 5), seed=1), (0, -1, 1))
    print(f"with adapters: {adapted.generate(prompts, steps=4)[0]}")
    print(f"perplexity of the prompts: {math.exp(-score.mean().item()):.1f}; alternatives at the end "
          f"{last['top_index'].tolist()}")


if __name__ == "__main__":
    main()
