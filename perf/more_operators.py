"""More operators of a serving step, as cases that can be timed and checked: the per-head norm and
position rotation of queries and keys, the same on the way into the 4-bit cache, ancestor masks of
drafted trees, attention of such trees over the cache, and low-rank adapters beside the quantized
linears.

Rotation. Pair i of a head's first R = 2 len(inv_freq) channels is (i, i + R/2), or (2i, 2i + 1)
where interleaved; it is turned by position * inv_freq[i] and multiplied by ``factor``. A norm, where
there is one, comes first: x / sqrt(mean(x^2) + eps) * weight over the head's channels. What goes into
the cache is rounded to float32 once and then to codes.

Cache format. A layer's cache is four buffers over ``pages`` pages of ``page`` tokens, for H
key/value heads of D channels:
  k_codes   uint8 [pages][H][page][D/2]             low nibble = even channel
  v_codes   uint8 [pages][H][page/8][16][8][D/32]   8 tokens, interleaved: 16 channel groups of
                                                    D/16 channels, 8 tokens each
  k_scales, v_scales  bfloat16 [pages][H][page]
A code is a nibble sign<<3 | magnitude that stands for +-(0, .5, 1, 1.5, 2, 3, 4, 6)[magnitude]
times its token's and head's scale, the smallest bfloat16 s with 6 s >= max |x| over the row.
The magnitude is the number of thresholds (.25, .75, 1.25, 1.75, 2.5, 3.5, 5) s at or below |x|.

Trees. The new tokens of a request are nodes; a node's parent comes before it, and a negative parent
(or one that does not come before it) is the last cached token. Bit j of a node's mask is set where
node j is the node itself or an ancestor; its position is the cached length plus its depth. A node
sees the cached tokens and the nodes of its mask.

Adapters. y_i[t] + scale[a] (x[t] A_i[a]^T) B_i[a]^T with a the adapter of the request that token t
belongs to (negative: none) and rank[a] rows of A_i[a], columns of B_i[a].

Where ``own`` is false, run() computes the operators with elementary torch operations in float32
(angles and what goes into codes in float64); where it is true, it calls the library.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda:0"
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
THRESHOLDS = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6


def listed():
    return [
        # A decode step of 32 sequences in the 4096-wide decoder, as the linears write it.
        _rotate("rotate_decode_32", tokens=32, heads=8, group=4, dim=128, turned=128, dtype="f32",
                to="f16", norm=True),
        # A ragged prompt in the 2048-wide decoder: half of the channels turned, pairs interleaved.
        _rotate("rotate_prompt_6001", tokens=6001, heads=8, group=4, dim=64, turned=32,
                dtype="bf16", to="bf16", norm=False, interleaved=True),
        # The queries, keys and values of one decode step of 48 sequences, into the cache.
        _append("append_rotated_decode_48", tokens=48, heads=8, group=4, dim=128, turned=128,
                page=64, dtype="f32", norm=True),
        # A prompt of 8191 tokens, into the cache.
        _append("append_rotated_prompt_8191", tokens=8191, heads=8, group=4, dim=128, turned=128,
                page=64, dtype="f32", norm=False),
        # One draft of seven tokens.
        _tables("tree_tables_1x7", requests=1, nodes=7, hi=700),
        # A full batch of large drafts.
        _tables("tree_tables_256x64", requests=256, nodes=64, hi=16000),
        # The smallest attention call: one sequence, a draft of seven tokens.
        _attention("tree_2048w_1x700_n7", requests=1, lo=700, hi=700, nodes=7, heads=8, group=4,
                   dim=64, page=64),
        # Ordinary speculative decode of the 4096-wide decoder: ragged lengths and drafts.
        _attention("tree_4096w_24x4000_n24", requests=24, lo=300, hi=4100, nodes=24, heads=8,
                   group=4, dim=128, page=64),
        # Two long contexts with large drafts, bfloat16: the most products of one step.
        _attention("tree_4096w_2x100000_n64", requests=2, lo=60000, hi=100000, nodes=64, heads=8,
                   group=4, dim=128, page=64, dtype="bf16"),
        # One token through an adapter beside query, key and value projections of 4096 features.
        _adapters("adapters_decode_1", requests=1, new=1, k=4096, n=(4096, 1024, 1024), adapters=1,
                  rank=16, dtype="f16"),
        # 64 sequences with 40 adapters of mixed ranks beside the gate and up projections.
        _adapters("adapters_decode_64", requests=64, new=1, k=4096, n=(14336, 14336), adapters=40,
                  rank=64, dtype="bf16", mixed=True),
        # Ragged prompts of 7 sequences (about 5000 tokens) with 3 adapters and without.
        _adapters("adapters_prompts_7", requests=7, new=1201, k=4096, n=(4096, 1024, 1024),
                  adapters=3, rank=32, dtype="f16"),
    ]


def _rotate(name, tokens, heads, group, dim, turned, dtype, to, norm, interleaved=False):
    return dict(name=name, kind="rotate", tokens=tokens, heads=heads, group=group, dim=dim,
                turned=turned, dtype=dtype, to=to, norm=norm, interleaved=interleaved)


def _append(name, tokens, heads, group, dim, turned, page, dtype, norm, interleaved=False):
    return dict(name=name, kind="append", tokens=tokens, heads=heads, group=group, dim=dim,
                turned=turned, page=page, dtype=dtype, norm=norm, interleaved=interleaved)


def _tables(name, requests, nodes, hi):
    return dict(name=name, kind="tables", requests=requests, nodes=nodes, lo=hi // 8, hi=hi)


def _attention(name, requests, lo, hi, nodes, heads, group, dim, page, dtype="f16", window=0):
    return dict(name=name, kind="attention", requests=requests, lo=lo, hi=hi, nodes=nodes,
                heads=heads, group=group, dim=dim, page=page, dtype=dtype, window=window)


def _adapters(name, requests, new, k, n, adapters, rank, dtype, mixed=False):
    return dict(name=name, kind="adapters", requests=requests, new=new, k=k,
                n=",".join(str(v) for v in n), adapters=adapters, rank=rank, dtype=dtype,
                mixed=mixed)


def _log_int(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))
    return min(max(int(v), lo), hi)


def draw(rng):
    kind = rng.choice(["rotate", "append", "append", "tables", "attention", "attention",
                       "attention", "adapters", "adapters"])
    if kind == "tables":
        hi = _log_int(rng, 8, 131071)
        return dict(kind=kind, requests=_log_int(rng, 1, 256), nodes=rng.randint(1, 64), lo=hi // 8, hi=hi)
    if kind in ("rotate", "append"):
        dim = rng.choice([64, 128, 128, 256])
        heads, group = rng.choice([(8, 4), (8, 4), (8, 1), (4, 8), (2, 16), (1, 7), (3, 5)])
        case = dict(kind=kind, tokens=_log_int(rng, 1, 8191), heads=heads, group=group, dim=dim,
                    turned=rng.choice([dim, dim, dim // 2, dim // 4, 3 * dim // 4]),
                    dtype=rng.choice(["f32", "f16", "bf16"]), norm=rng.random() < 0.5,
                    interleaved=rng.random() < 0.3)
        while case["tokens"] * heads * (group + 2) * dim > 8191 * 48 * 128:
            case["tokens"] = case["tokens"] // 2 + 1
        if kind == "rotate":
            return dict(case, to=rng.choice(["f32", "f16", "bf16"]))
        return dict(case, page=rng.choice([16, 32, 64, 128]))
    if kind == "adapters":
        prompts = rng.random() < 0.5
        case = dict(kind=kind, requests=_log_int(rng, 1, 12 if prompts else 128),
                    new=_log_int(rng, 2, 1500) if prompts else rng.choice([1, 1, 1, 4]),
                    k=32 * _log_int(rng, 16, 448), adapters=_log_int(rng, 1, 48),
                    rank=8 * _log_int(rng, 1, 16), dtype=rng.choice(["f16", "bf16"]),
                    mixed=rng.random() < 0.5)
        n = [_log_int(rng, 200, 14336) for _ in range(rng.randint(1, 4))]
        # No more of weights and of products than in the largest listed cases.
        while case["rank"] * (case["k"] * len(n) + sum(n)) * case["adapters"] > 100_000_000:
            case["adapters"], case["rank"] = case["adapters"] // 2 + 1, max(8, case["rank"] // 16 * 8)
            if case["adapters"] <= 2 and case["rank"] == 8:
                n = n[:1]
        while case["requests"] * case["new"] * (case["k"] + 4 * sum(n)) > 60_000_000:
            if case["new"] > 4:
                case["new"] = case["new"] // 2
            elif case["requests"] > 1:
                case["requests"] //= 2
            else:
                n = n[:1]
        return dict(case, n=",".join(str(v) for v in n))
    heads, group = rng.choice([(8, 4), (8, 4), (8, 1), (4, 8), (2, 16), (1, 7), (3, 5)])
    case = dict(kind="attention", requests=_log_int(rng, 1, 64), nodes=_log_int(rng, 1, 64),
                heads=heads, group=group, dim=rng.choice([64, 128, 128, 256]),
                page=rng.choice([16, 32, 64, 128]), dtype=rng.choice(["f16", "bf16", "f32"]),
                window=rng.choice([0, 0, 0, rng.randint(64, 5000)]))
    case["hi"] = _log_int(rng, max(20, case["nodes"]), 131071)
    part = rng.uniform(0.1, 1.0)
    # No more cached values, and no more query-key pairs, than the largest listed case.
    while (case["requests"] * case["hi"] * heads * case["dim"] > 2 * 100000 * 8 * 128
           or case["requests"] * case["hi"] * case["nodes"] * heads * group * case["dim"]
           > 2 * 80000 * 64 * 32 * 128):
        if case["hi"] > 400:
            case["hi"] //= 2
        else:
            case["requests"] = max(1, case["requests"] // 2)
    case["lo"] = max(case["nodes"], int(case["hi"] * part))
    return case


# ------------------------------------------------------------------ lengths

def _spread(n, lo, hi):
    """Lengths spread evenly over [lo, hi]."""
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _ragged(n, most):
    """Numbers of tokens of n requests, 1 to most."""
    return [1 + (most - 1) * (7 - i % 7) // 7 for i in range(n)]


def _seen_cached(case):
    """Cached tokens that the drafts of each request see."""
    out = []
    for length, n in zip(_spread(case["requests"], case["lo"], case["hi"]),
                         _ragged(case["requests"], case["nodes"])):
        cached = length - n
        out.append(min(cached, case["window"]) if case["window"] else cached)
    return out


def _widths(case):
    return [int(v) for v in case["n"].split(",")]


def _adapter_of(case):
    """The adapter of each request; among several requests every sixth has none."""
    n = case["requests"]
    return [-1 if n > 1 and i % 6 == 5 else i * 7 % case["adapters"] for i in range(n)]


def _adapter_ranks(case):
    """Ranks of the adapters: all of the pool's, or mixed ones from 1 up."""
    most, n = case["rank"], case["adapters"]
    return [max(1, most * (1 + i % 4) // 4 - i % 3) if case["mixed"] else most for i in range(n)]


def _adapter_tokens(case):
    return [case["new"]] * case["requests"] if case["new"] <= 4 else _ragged(case["requests"], case["new"])


# ------------------------------------------------------------------ inputs

def _generator(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + stream)
    return g


def _keys(shape, g):
    """Keys (or queries) as projections give them: a few channels much larger than the rest."""
    wide = torch.exp(0.7 * torch.randn(shape[-2:], generator=g, device=DEV))
    return torch.randn(shape, generator=g, device=DEV) * wide


def _values(shape, g):
    """Values whose size varies from token to token."""
    size = torch.exp(0.5 * torch.randn(shape[:-1] + (1,), generator=g, device=DEV))
    return torch.randn(shape, generator=g, device=DEV) * size


def _ints(v, dtype=torch.int32):
    return torch.tensor(np.asarray(v), dtype=dtype).to(DEV)


def _quantize(x):
    """(codes, one a byte, and bfloat16 scales) of float rows [...][D]."""
    x = x.float()
    size = x.abs()
    size = torch.where(torch.isfinite(size), size, torch.zeros_like(size)).amax(-1)
    down = ((size / 6).view(torch.int32) & -65536).view(torch.float32)
    up = (down.view(torch.int32) + 65536).view(torch.float32)
    scale = torch.where(6 * down < size, up, down)
    mag = torch.zeros(x.shape, dtype=torch.uint8, device=x.device)
    for t in THRESHOLDS:
        mag += x.abs() >= (t * scale)[..., None]
    mag *= (scale > 0)[..., None]
    return mag | (((x < 0) & (mag > 0)).to(torch.uint8) << 3), scale.to(torch.bfloat16)


def _pack(c):
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _pack_values(c):
    """Codes [...][page][D] of values in the cache's interleaved layout."""
    page, dim = c.shape[-2:]
    c = c.reshape(c.shape[:-2] + (page // 8, 8, 16, dim // 16))
    return _pack(c.transpose(-3, -2)).contiguous()


def _filled_cache(pages, case, g):
    """A cache whose every slot is written, made in parts."""
    shape = (case["heads"], case["page"], case["dim"])
    part = max(1, (1 << 25) // (shape[0] * shape[1] * shape[2]))
    got = [[], [], [], []]
    for at in range(0, pages, part):
        n = min(part, pages - at)
        k, ks = _quantize(_keys((n, shape[1], shape[0], shape[2]), g).transpose(1, 2))
        v, vs = _quantize(_values((n,) + shape, g))
        for to, x in zip(got, (_pack(k), ks, _pack_values(v), vs)):
            to.append(x)
    return tuple(torch.cat(x).contiguous() for x in got)


def _empty_cache(pages, case):
    h, page, dim = case["heads"], case["page"], case["dim"]
    codes = dict(dtype=torch.uint8, device=DEV)
    scales = dict(dtype=torch.bfloat16, device=DEV)
    return (torch.zeros((pages, h, page, dim // 2), **codes), torch.zeros((pages, h, page), **scales),
            torch.zeros((pages, h, page // 8, 16, 8, dim // 32), **codes),
            torch.zeros((pages, h, page), **scales))


def _prepare_rotate(case, seed):
    g, rng = _generator(seed, 1), np.random.default_rng(seed)
    t, h, dim, dtype = case["tokens"], case["heads"], case["dim"], DTYPES[case["dtype"]]
    hq = h * case["group"]
    # Positions of a few requests, one of them far on.
    starts = np.sort(rng.integers(0, t + 1, 2))
    far = rng.integers(0, 131072, 3)
    positions = np.concatenate([far[0] + np.arange(starts[0]), far[1] + np.arange(starts[1] - starts[0]),
                                far[2] + np.arange(t - starts[1])])
    i = torch.arange(0, case["turned"], 2, dtype=torch.float64)
    s = dict(kind=case["kind"], q=_keys((t, hq, dim), g).to(dtype), k=_keys((t, h, dim), g).to(dtype),
             positions=_ints(positions), interleaved=case["interleaved"],
             inv_freq=(10000.0 ** (-i / case["turned"])).float().to(DEV), q_weight=None, k_weight=None)
    if case["norm"]:
        for name in ("q_weight", "k_weight"):
            s[name] = 1 + 0.2 * torch.randn(dim, generator=g, device=DEV)
    if case["kind"] == "rotate":
        to = DTYPES[case["to"]]
        s["q_out"], s["k_out"] = torch.empty_like(s["q"], dtype=to), torch.empty_like(s["k"], dtype=to)
        return s
    page = case["page"]
    pages = -(-t // page) + 5
    # Slots as a step's map gives them: runs of at most a page, in any order, one token skipped.
    order = rng.permutation(pages)
    slots = (order[:, None] * page + np.arange(page)).reshape(-1)[:t]
    if t > 8:
        slots[int(rng.integers(t))] = -1
    return dict(s, v=_values((t, h, dim), g).to(dtype), cache=_empty_cache(pages, case),
                slots=_ints(slots, torch.int64), q_out=torch.empty_like(s["q"], dtype=torch.float16))


def _drafts(case, rng):
    """(lengths with the drafts, numbers of nodes, parents of all nodes), requests in any order."""
    n = case["requests"]
    length, new = np.array(_spread(n, case["lo"], case["hi"])), np.array(_ragged(n, case["nodes"]))
    turn = rng.permutation(n)
    length, new = np.maximum(length[turn], new[turn]), new[turn]
    # Most nodes go on from one of the last few; some branch from anywhere.
    parents = [max(-1, i - 1 - int(rng.integers(0, 4))) if rng.random() < 0.8
               else int(rng.integers(-1, i)) if i else -1 for m in new for i in range(m)]
    return length, new, np.array(parents, dtype=np.int64)


def _masks(new, parents):
    """Ancestor masks, as unsigned 64-bit numbers."""
    out, at = np.zeros(len(parents), dtype=np.uint64), 0
    for m in new:
        for i in range(m):
            p = parents[at + i]
            out[at + i] = np.uint64(1 << i) | (out[at + p] if 0 <= p < i else np.uint64(0))
        at += m
    return out


def _prepare_tables(case, seed):
    rng = np.random.default_rng(seed)
    length, new, parents = _drafts(case, rng)
    return dict(kind="tables", parents=_ints(parents), seq_lens=_ints(length),
                q_starts=_ints(np.concatenate([[0], np.cumsum(new)])), nodes=len(parents),
                out=dict(masks=torch.empty(len(parents), device=DEV, dtype=torch.int64),
                         positions=torch.empty(len(parents), device=DEV, dtype=torch.int32)))


def _prepare_attention(case, seed):
    g, rng = _generator(seed, 2), np.random.default_rng(seed)
    length, new, parents = _drafts(case, rng)
    page = case["page"]
    width = -(-int(length.max()) // page)
    used = -(-length // page)
    order = rng.permutation(int(used.sum()) + 2).astype(np.int32)
    table, at = np.full((len(length), width), -1, dtype=np.int32), 0
    for r, n in enumerate(used):
        table[r, :n] = order[at:at + n]
        at += n
    cache = _filled_cache(len(order), case, g)
    tokens, hq, dtype = len(parents), case["heads"] * case["group"], DTYPES[case["dtype"]]
    q = torch.randn((tokens, hq, case["dim"]), generator=g, device=DEV) * 0.9
    out_dtype = torch.bfloat16 if dtype == torch.bfloat16 else torch.float16
    return dict(kind="attention", q=q.to(dtype), cache=cache, table=_ints(table),
                seq_lens=_ints(length), q_starts=_ints(np.concatenate([[0], np.cumsum(new)])),
                masks=_ints(_masks(new, parents).view(np.int64), torch.int64), max_new=int(new.max()),
                window=case["window"], scale=case["dim"] ** -0.5,
                out=torch.empty((tokens, hq, case["dim"]), device=DEV, dtype=out_dtype),
                lse=torch.empty((tokens, hq), device=DEV),
                # A workspace, as a program keeps one for all its layers.
                work=torch.zeros(1 << 28, dtype=torch.uint8, device=DEV),
                token_request=_ints(np.repeat(np.arange(len(new)), new), torch.int64))


def _prepare_adapters(case, seed):
    g = _generator(seed, 3)
    new, widths, rank = _adapter_tokens(case), _widths(case), case["rank"]
    t, k, dtype = sum(new), case["k"], DTYPES[case["dtype"]]
    ranks = _adapter_ranks(case)
    a, b = [], []
    keep = (torch.arange(rank, device=DEV) < _ints(ranks)[:, None]).float()
    for n in widths:
        a.append((torch.randn((case["adapters"], rank, k), generator=g, device=DEV) * k ** -0.5
                  * keep[:, :, None]).to(dtype))
        b.append((torch.randn((case["adapters"], n, rank), generator=g, device=DEV) * 0.02
                  * keep[:, None, :]).to(dtype))
    y = [0.7 * torch.randn((t, n), generator=g, device=DEV) for n in widths]
    ids = _adapter_of(case)
    return dict(kind="adapters", x=torch.randn((t, k), generator=g, device=DEV).half(), ys=y, a=a, b=b,
                q_starts=_ints(np.concatenate([[0], np.cumsum(new)])), adapter=_ints(ids),
                ranks=_ints(ranks), scales=2 * torch.rand(case["adapters"], generator=g, device=DEV),
                max_new=max(new), host=(new, ids, ranks), outs=[torch.empty_like(v) for v in y], work=None)


def prepare(case, seed):
    make = dict(rotate=_prepare_rotate, append=_prepare_rotate, tables=_prepare_tables,
                attention=_prepare_attention, adapters=_prepare_adapters)
    return make[case["kind"]](case, seed)


# ------------------------------------------------------------------ the plain forms

def _plain_turned(x, weight, s, dtype):
    """Rows normed and rotated in a type; angles in float64."""
    x = x.to(dtype)
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight
    angle = s["positions"].double()[:, None, None] * s["inv_freq"].double()
    c, sn = torch.cos(angle).to(dtype), torch.sin(angle).to(dtype)
    r = 2 * s["inv_freq"].numel()
    y = x.clone()
    first, second = (slice(0, r, 2), slice(1, r, 2)) if s["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
    u, v = x[..., first], x[..., second]
    y[..., first] = u * c - v * sn
    y[..., second] = v * c + u * sn
    return y


def _plain_rotate(s):
    return dict(q=_plain_turned(s["q"], s["q_weight"], s, torch.float32).to(s["q_out"].dtype),
                k=_plain_turned(s["k"], s["k_weight"], s, torch.float32).to(s["k_out"].dtype))


def _byte_table():
    """The two values of a code byte."""
    one = torch.tensor(MAGNITUDES + tuple(-x for x in MAGNITUDES), device=DEV)
    return torch.stack([one.repeat(16), one.repeat_interleave(16)], 1)


def _decoded(codes, scales, values):
    """float32 rows [...][H][page][D] of a cache's codes."""
    x = _byte_table()[codes.int()].flatten(-2)
    if values:
        x = x.transpose(-3, -2).flatten(-2).flatten(-3, -2)
    return x * scales.float()[..., None]


def _plain_append(s):
    kc, ks, vc, vs = s["cache"]
    pages, h, page = ks.shape
    dim = 2 * kc.shape[-1]
    slot = s["slots"]
    put = slot >= 0
    at = torch.where(put, slot, pages * page)     # a token with no slot goes to a row past the end
    p, o = at // page, at % page
    k, k_scale = _quantize(_plain_turned(s["k"], s["k_weight"], s, torch.float64).float())
    v, v_scale = _quantize(s["v"])
    rows = torch.zeros((pages + 1, page, h, dim), dtype=torch.uint8, device=DEV)
    rows[p, o] = k
    scales = torch.zeros((pages + 1, page, h), dtype=torch.bfloat16, device=DEV)
    scales[p, o] = k_scale
    new_kc, new_ks = _pack(rows[:-1].transpose(1, 2)), scales[:-1].transpose(1, 2)
    rows, scales = torch.zeros_like(rows), torch.zeros_like(scales)
    rows[p, o] = v
    scales[p, o] = v_scale
    new_vc, new_vs = _pack_values(rows[:-1].transpose(1, 2)), scales[:-1].transpose(1, 2)
    # The cache was empty, so what it holds now is the new rows; read back through the map.
    k = _decoded(new_kc, new_ks, False).transpose(1, 2).flatten(0, 1)
    v = _decoded(new_vc, new_vs, True).transpose(1, 2).flatten(0, 1)
    keep, row = put[:, None, None], slot.clamp(min=0)
    q = _plain_turned(s["q"], s["q_weight"], s, torch.float32)
    return dict(q=q.half(), k=(k[row] * keep).half(), v=(v[row] * keep).half())


def _plain_tables(s):
    starts = s["q_starts"].long()
    n = starts.numel() - 1
    new = starts[1:] - starts[:-1]
    request = torch.repeat_interleave(torch.arange(n, device=DEV), new, output_size=s["nodes"])
    index = torch.arange(s["nodes"], device=DEV) - starts[request]
    parent = s["parents"].long()
    has = (parent >= 0) & (parent < index)
    up = torch.where(has, parent + starts[request], torch.zeros_like(parent))
    mask, depth = torch.ones_like(parent) << index, has.long()
    # Paths twice as long each time.
    for _ in range(6):
        mask = mask | torch.where(has, mask[up], torch.zeros_like(mask))
        depth = depth + torch.where(has, depth[up], torch.zeros_like(depth))
        has, up = has & has[up], torch.where(has, up[up], up)
    position = s["seq_lens"].long()[request] - new[request] + depth
    return dict(masks=mask, positions=position.int())


def _plain_attention(s):
    kc, ks, vc, vs = s["cache"]
    q, table, starts = s["q"].float(), s["table"], s["q_starts"].long()
    n, width = table.shape
    h, page, dim = kc.shape[1], kc.shape[2], 2 * kc.shape[3]
    group, most, span = q.shape[1] // h, s["max_new"], width * page
    pages = table.clamp(min=0).long()
    k = _decoded(kc[pages], ks[pages], False).transpose(1, 2).reshape(n, h, span, dim)
    v = _decoded(vc[pages], vs[pages], True).transpose(1, 2).reshape(n, h, span, dim)
    new = starts[1:] - starts[:-1]
    row = torch.arange(most, device=DEV)
    token = (starts[:-1, None] + row).clamp(max=q.shape[0] - 1)
    qp = q[token].reshape(n, most, h, group, dim).permute(0, 2, 3, 1, 4)
    score = torch.matmul(qp.reshape(n, h, group * most, dim), k.transpose(2, 3)) * s["scale"]
    del k
    score = score.reshape(n, h, group, most, span)
    place = torch.arange(span, device=DEV)
    cached = (s["seq_lens"].long() - new)[:, None, None]              # [n][1][1]
    mask = s["masks"][token][:, :, None]                              # [n][most][1]
    depth = ((mask >> torch.arange(64, device=DEV)) & 1).sum(-1, keepdim=True) - 1
    seen = place < cached
    if s["window"]:
        seen = seen & (place > cached + depth - s["window"])
    node = place - cached
    inside = (node >= 0) & (node < new[:, None, None])
    seen = seen | (inside & (((mask >> node.clamp(0, 63)) & 1) > 0))
    seen = seen & (table >= 0).repeat_interleave(page, 1)[:, None]
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    score = score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score.reshape(n, h, group * most, span), v)
    out = out.reshape(n, h, group, most, dim) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + torch.log(total)).squeeze(-1)
    which = s["token_request"]
    at = torch.arange(q.shape[0], device=DEV) - starts[which]
    out = out.permute(0, 3, 1, 2, 4)[which, at].flatten(1, 2)
    lse = lse.permute(0, 3, 1, 2)[which, at].flatten(1, 2)
    return dict(out=out.to(s["out"].dtype), lse=lse)


def _plain_adapters(s):
    new, ids, ranks = s["host"]
    x = s["x"].float()
    outs = []
    for y, a, b in zip(s["ys"], s["a"], s["b"]):
        out, at = y.clone(), 0
        for n, i in zip(new, ids):
            if i >= 0:
                h = torch.matmul(x[at:at + n], a[i, :ranks[i]].float().t())
                out[at:at + n] += s["scales"][i] * torch.matmul(h, b[i, :, :ranks[i]].float().t())
            at += n
        outs.append(out)
    return outs


# ------------------------------------------------------------------ a pass

def run(s):
    kind = s["kind"]
    if not own:
        plain = dict(rotate=_plain_rotate, append=_plain_append, tables=_plain_tables,
                     attention=_plain_attention, adapters=_plain_adapters)
        return plain[kind](s)
    from paper_2607_01127_amd import logbq as L
    if kind == "tables":
        L.tree_tables(s["parents"], s["q_starts"], s["seq_lens"], out=s["out"])
        return dict(s["out"])
    if kind == "attention":
        L.kv4_tree_attention(s["q"], s["cache"], s["table"], s["seq_lens"], s["q_starts"], s["masks"],
                             s["max_new"], scale=s["scale"], window=s["window"], out=s["out"],
                             lse=s["lse"], workspace=s["work"])
        return dict(out=s["out"], lse=s["lse"])
    if kind == "adapters":
        if s["work"] is None:
            need = L.linear_adapters_workspace_bytes(s["x"].shape[0], len(s["a"]), s["a"][0].shape[1])
            s["work"] = torch.empty(need, dtype=torch.uint8, device=DEV)
        return L.linear_adapters(s["x"], s["ys"], s["a"], s["b"], s["q_starts"], s["adapter"],
                                 s["max_new"], scales=s["scales"], ranks=s["ranks"], outs=s["outs"],
                                 workspace=s["work"])
    rotation = L.Rotation(s["inv_freq"], interleaved=s["interleaved"])
    if kind == "rotate":
        q, k = L.qk_rotate(s["q"], s["k"], s["positions"], rotation, q_weight=s["q_weight"],
                           k_weight=s["k_weight"], eps=EPS, q_out=s["q_out"], k_out=s["k_out"])
        return dict(q=q, k=k)
    q = L.kv4_append_rotated(s["q"], s["k"], s["v"], s["cache"], s["slots"], s["positions"], rotation,
                             q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, q_out=s["q_out"])
    k, v = L.kv4_read(s["cache"], s["slots"])
    return dict(q=q, k=k, v=v)


# ------------------------------------------------------------------ what a pass needs

def work(case):
    kind = case["kind"]
    if kind == "rotate":
        rows = case["tokens"] * case["heads"] * (case["group"] + 1)
        return {"bytes": rows * case["dim"] * (BYTES[case["dtype"]] + BYTES[case["to"]])
                + 4 * case["tokens"], "flops": 0}
    if kind == "append":
        rows, dim, size = case["tokens"] * case["heads"], case["dim"], BYTES[case["dtype"]]
        # Rows in; queries, codes and scales out; codes and scales back in, float16 values out.
        b = rows * case["group"] * dim * (size + 2) + 2 * rows * (dim * size + 2 * (dim // 2 + 2) + 2 * dim)
        return {"bytes": b + 20 * case["tokens"], "flops": 0}
    if kind == "tables":
        nodes = sum(_ragged(case["requests"], case["nodes"]))
        return {"bytes": 16 * nodes + 8 * case["requests"] + 4, "flops": 0}
    if kind == "adapters":
        new, ids, ranks, widths = _adapter_tokens(case), _adapter_of(case), _adapter_ranks(case), _widths(case)
        features = len(widths) * case["k"] + sum(widths)
        with_one = [(n, ranks[i]) for n, i in zip(new, ids) if i >= 0]
        weights = 2 * sum(ranks[i] for i in set(ids) if i >= 0) * features
        return {"bytes": weights + sum(n for n, _ in with_one) * 2 * case["k"] + 8 * sum(new) * sum(widths),
                "flops": sum(2 * n * r * features for n, r in with_one)}
    hq, new = case["heads"] * case["group"], _ragged(case["requests"], case["nodes"])
    seen = _seen_cached(case)
    b = (sum(seen) + sum(new)) * case["heads"] * (case["dim"] + 4)
    b += sum(new) * (hq * (case["dim"] * (BYTES[case["dtype"]] + 2) + 4) + 8)
    # A node sees itself and the cached tokens at least.
    pairs = sum(n * (c + 1) for n, c in zip(new, seen))
    return {"bytes": b, "flops": 4 * case["dim"] * hq * pairs}


# ------------------------------------------------------------------ 64-bit results

def _exact_turned(x, weight, s):
    """float64 rows, normed and turned as complex numbers."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS) * weight.double()
    half = s["inv_freq"].numel()
    angle = s["positions"].double()[:, None, None] * s["inv_freq"].double()
    turn = torch.polar(torch.ones_like(angle), angle)
    pairs = x[..., :2 * half]
    pairs = pairs.unflatten(-1, (half, 2)) if s["interleaved"] else pairs.unflatten(-1, (2, half)).transpose(-1, -2)
    z = torch.view_as_real(torch.complex(pairs[..., 0], pairs[..., 1]) * turn)
    z = z.flatten(-2) if s["interleaved"] else z.transpose(-1, -2).flatten(-2)
    return torch.cat([z, x[..., 2 * half:]], -1)


def _exact_rows(x):
    """float64 values that the 4-bit rows of x stand for, from the format's definition."""
    x = x.double()
    finite = torch.where(torch.isfinite(x), x, torch.zeros_like(x))
    size = finite.abs().amax(-1, keepdim=True)
    # Smallest number of 8 significant bits that is at least size / 6.
    e = torch.exp2(torch.floor(torch.log2(torch.where(size > 0, size, torch.ones_like(size)) / 6)) - 7)
    scale = torch.ceil(size / 6 / e) * e
    scale = torch.where(6 * (scale - e) >= size, scale - e, scale)
    ratio = x.abs() / torch.where(scale > 0, scale, torch.ones_like(scale))
    levels = torch.tensor(MAGNITUDES, dtype=torch.float64, device=DEV)
    middle = (levels[1:] + levels[:-1]) / 2
    which = torch.bucketize(ratio, middle, right=True)
    return torch.sign(x) * levels[which] * scale


def _exact_rotate(case, seed):
    s = _prepare_rotate(case, seed)
    q = _exact_turned(s["q"], s["q_weight"], s)
    k = _exact_turned(s["k"], s["k_weight"], s)
    if case["kind"] == "rotate":
        return dict(q=q, k=k)
    keep = (s["slots"] >= 0)[:, None, None]
    return dict(q=q, k=_exact_rows(k.float()) * keep, v=_exact_rows(s["v"]) * keep)


def _exact_attention(case, seed):
    s = _prepare_attention(case, seed)
    kc, ks, vc, vs = s["cache"]
    level = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), dtype=torch.float64, device=DEV)
    page, dim, h, group = case["page"], case["dim"], case["heads"], case["group"]
    starts, lens = s["q_starts"].tolist(), s["seq_lens"].tolist()
    masks = s["masks"].cpu().numpy().view(np.uint64)
    tokens, hq = s["q"].shape[:2]
    out = torch.zeros((tokens, hq, dim), dtype=torch.float64, device=DEV)
    lse = torch.full((tokens, hq), -math.inf, dtype=torch.float64, device=DEV)
    for r, length in enumerate(lens):
        a, b = starts[r], starts[r + 1]
        cached = length - (b - a)
        hide = np.zeros((b - a, length), dtype=bool)
        for i in range(b - a):
            bits = int(masks[a + i])
            if case["window"]:
                hide[i, :max(0, cached + bin(bits).count("1") - case["window"])] = True
            hide[i, cached:] = [not bits >> j & 1 for j in range(b - a)]
        hide = torch.from_numpy(hide).to(DEV)
        ids = s["table"][r, :-(-length // page)].long()
        for j in range(h):
            k = torch.stack([level[(kc[ids, j] & 15).long()], level[(kc[ids, j] >> 4).long()]], -1)
            k = k.reshape(-1, dim) * ks[ids, j].double().reshape(-1, 1)
            c = vc[ids, j]                                        # [pages][page/8][16][8][D/32]
            v = torch.stack([level[(c & 15).long()], level[(c >> 4).long()]], -1)
            v = v.permute(0, 1, 3, 2, 4, 5).reshape(-1, dim) * vs[ids, j].double().reshape(-1, 1)
            k, v = k[:length], v[:length]
            for g in range(j * group, (j + 1) * group):
                score = s["q"][a:b, g].double() @ k.T * s["scale"]
                score = score.masked_fill(hide, -math.inf)
                total = torch.logsumexp(score, 1)
                out[a:b, g] = torch.exp(score - total[:, None]) @ v
                lse[a:b, g] = total
    return dict(out=out, lse=lse)


def _exact_adapters(case, seed):
    s = _prepare_adapters(case, seed)
    starts, ids = s["q_starts"].tolist(), s["adapter"].tolist()
    outs = [y.double() for y in s["ys"]]
    for r, i in enumerate(ids):
        rows = slice(starts[r], starts[r + 1])
        if i < 0:
            continue
        x, rank = s["x"][rows].double(), int(s["ranks"][i])
        for out, a, b in zip(outs, s["a"], s["b"]):
            delta = b[i, :, :rank].double() @ (a[i, :rank].double() @ x.T)
            out[rows] += float(s["scales"][i]) * delta.T
    return outs


def exact(case, seed):
    make = dict(rotate=_exact_rotate, append=_exact_rotate, attention=_exact_attention,
                adapters=_exact_adapters)
    return make[case["kind"]](case, seed) if case["kind"] in make else None
