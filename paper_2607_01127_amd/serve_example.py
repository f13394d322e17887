"""A small decoder served with this library: 4-bit linears, a paged 4-bit key/value cache, attention
over it and the log probabilities of what it answers.

    python -m paper_2607_01127_amd.serve_example

The decoder is Llama-style (RMS norm, rotary embedding, grouped key/value heads, gated MLP) with
random weights, each projection quantized with its own codebook; the embedding and the output head
stay in 16 bits, as in the paper (Sec. 4). A step is what a serving program runs for any mixture of
prompts and single tokens:

    batch_tables -> for each layer: linear_multi (q, k, v), kv4_append, kv4_attention, linear (o),
    linear_multi (gate, up), linear (down) -> output head, token_logprobs

Nothing in a step waits for the GPU; the lengths that the host needs are its own.
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

    def step(self, tokens, tables, max_new: int):
        """float32 logits [tokens][vocab] of the step's tokens, whose keys and values go into the
        caches; `tables` is batch_tables' result with the block table as "table"."""
        s, t = self.shape, tokens.numel()
        x = self.embedding[tokens].float()
        for lin, cache in self.layers:
            q, k, v = L.linear_multi(self._norm(x), *zip(*(lin[n] for n in ("q", "k", "v"))))
            q = self._rotate(q.view(t, s.heads, s.dim), tables["positions"])
            k = self._rotate(k.view(t, s.kv_heads, s.dim), tables["positions"])
            L.kv4_append(k, v.view(t, s.kv_heads, s.dim), cache, tables["slots"])
            a = L.kv4_attention(q, cache, tables["table"], tables["seq_lens"], tables["q_starts"],
                                max_new, workspace=self.kv_work)
            x = x + L.linear(a.view(t, -1), *lin["o"])
            gate, up = L.linear_multi(self._norm(x), *zip(*(lin[n] for n in ("gate", "up"))))
            x = x + L.linear((torch.nn.functional.silu(gate) * up).half(), *lin["down"])
        return (self._norm(x) @ self.head.T).float()


class Batch:
    """Requests that are served together. The host keeps their lengths. Pages are taken from the decoder
    for good, so that batches of one decoder may live side by side."""

    def __init__(self, decoder: Decoder, requests: int, most: int):
        self.decoder = decoder
        self.lengths = [0] * requests
        width = -(-most // decoder.page)
        self.table = torch.full((requests, width), -1, dtype=torch.int32, device=decoder.device)

    def step(self, new_tokens):
        """One step: a list of token lists (one a request, empty for none) -> logits of all of them
        in order."""
        d, page = self.decoder, self.decoder.page
        new = [len(x) for x in new_tokens]
        ints = torch.tensor([self.lengths, new], dtype=torch.int32).to(d.device)
        tokens = torch.tensor(sum(new_tokens, []), dtype=torch.int64).to(d.device)
        pages = sum(-(-(a + b) // page) - -(-a // page) for a, b in zip(self.lengths, new))
        total = [a + b for a, b in zip(self.lengths, new)]
        if max(total) > self.table.shape[1] * page or d.used + pages > d.free.numel():
            raise ValueError("the cache or the block table is too small for this step")
        tables = L.batch_tables(ints[0], ints[1], d.free[d.used:], self.table, page, len(tokens))
        logits = d.step(tokens, dict(tables, table=self.table), max(new))
        self.lengths, d.used = total, d.used + pages
        return logits

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


def main():
    decoder = Decoder(Shape(), pages=64)
    prompts = [list(range(5, 105)), [7, 8, 9], list(range(300, 377))]
    chosen, logprobs, entropies, last = Batch(decoder, len(prompts), 512).generate(prompts, steps=16)
    for r, tokens in enumerate(chosen):
        print(f"request {r}: {tokens}")
        print(f"  log probabilities {[round(x, 2) for x in logprobs[r].tolist()]}")
    score = Batch(decoder, len(prompts), 512).score(prompts)
    print(f"perplexity of the prompts: {math.exp(-score.mean().item()):.1f}; alternatives at the end "
          f"{last['top_index'].tolist()}")


if __name__ == "__main__":
    main()
