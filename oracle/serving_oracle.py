"""Plain float64 definitions of a serving step's operators (test infrastructure only): the 4-bit
key/value rows, block tables and slot maps, attention over the cache, and token log probabilities.
Written from the formulas in include/logbq.h; imports nothing from the library.
"""
import math

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
THRESHOLDS = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])


def bf16_up(x: float) -> float:
    """The smallest bfloat16 number that is at least x >= 0."""
    if x == 0.0:
        return 0.0
    e = max(math.floor(math.log2(x)), -126)
    for step in (2.0 ** (e - 8), 2.0 ** (e - 7)):        # log2 may round up to the next integer
        step = max(step, 2.0 ** -133)
        n = math.ceil(x / step)
        if n * step >= x and n <= 256:
            return n * step
    raise AssertionError(x)


def kv4_quantize(x):
    """(codes uint8, one a byte, and float64 scales) of rows [...][D]."""
    x = np.asarray(x, dtype=np.float64)
    rows = x.reshape(-1, x.shape[-1])
    codes = np.zeros(rows.shape, dtype=np.uint8)
    scales = np.zeros(rows.shape[0])
    for r, row in enumerate(rows):
        finite = np.abs(row[np.isfinite(row)])
        size = float(finite.max()) if finite.size else 0.0
        if size == 0.0:
            continue
        s = bf16_up(size / 6.0)
        # size / 6 rounds in float64; the definition compares 6 s with size.
        assert 6.0 * s >= size
        a = np.abs(row)
        mag = np.zeros(row.shape, dtype=np.uint8)
        for t in THRESHOLDS:
            mag += np.where(np.isnan(row), False, a >= t * s).astype(np.uint8)
        codes[r] = mag | (((row < 0) & (mag > 0)).astype(np.uint8) << 3)
        scales[r] = s
    return codes.reshape(x.shape), scales.reshape(x.shape[:-1])


def kv4_values(codes, scales):
    """float64 values of codes, one a byte."""
    v = MAGNITUDES[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    return v * np.asarray(scales, dtype=np.float64)[..., None]


def pack_keys(codes):
    """[pages][heads][page][D] codes, one a byte -> [pages][heads][page][D/2]."""
    return np.ascontiguousarray(codes[..., 0::2] | (codes[..., 1::2] << 4))


def unpack_keys(packed):
    out = np.empty(packed.shape[:-1] + (2 * packed.shape[-1],), dtype=np.uint8)
    out[..., 0::2], out[..., 1::2] = packed & 15, packed >> 4
    return out


def pack_values(codes):
    """[pages][heads][page][D] codes, one a byte -> [pages][heads][page/8][16][8][D/32]."""
    p, h, page, d = codes.shape
    out = np.zeros((p, h, page // 8, 16, 8, d // 32), dtype=np.uint8)
    for token in range(page):
        for group in range(16):
            c = codes[:, :, token, group * (d // 16):(group + 1) * (d // 16)]
            out[:, :, token // 8, group, token % 8] = c[..., 0::2] | (c[..., 1::2] << 4)
    return out


def unpack_values(packed):
    p, h, blocks, _, _, n = packed.shape
    out = np.zeros((p, h, blocks * 8, 32 * n), dtype=np.uint8)
    for token in range(blocks * 8):
        for group in range(16):
            c = packed[:, :, token // 8, group, token % 8]
            at = group * 2 * n
            out[:, :, token, at:at + 2 * n:2] = c & 15
            out[:, :, token, at + 1:at + 2 * n:2] = c >> 4
    return out


def batch_tables(cached, new, free, table, page, tokens):
    """Block table, slots, positions, starts, lengths and info, one request after another."""
    table = np.array(table, dtype=np.int64)
    width = table.shape[1]
    slots, positions = np.full(tokens, -1, dtype=np.int64), np.zeros(tokens, dtype=np.int64)
    starts, lens = [0], []
    taken = made = flags = 0
    for r, (c, n) in enumerate(zip(cached, new)):
        c, n = max(int(c), 0), max(int(n), 0)
        have, need = -(-c // page), -(-(c + n) // page)
        flags |= 2 if need > width else 0
        for j in range(have, need):
            if j < width:
                table[r, j] = free[taken] if taken < len(free) else -1
            taken += 1
        for i in range(n):
            if made + i < tokens:
                p = c + i
                page_id = table[r, p // page] if p // page < width else -1
                slots[made + i] = page_id * page + p % page if page_id >= 0 else -1
                positions[made + i] = min(p, 2**31 - 1)
        made += n
        starts.append(min(made, tokens))
        lens.append(min(c + n, 2**31 - 1))
    flags |= (1 if taken > len(free) else 0) | (4 if made > tokens else 0)
    info = [made, min(taken, len(free)), max(lens, default=0), flags]
    return dict(table=table, slots=slots, positions=positions, q_starts=np.array(starts),
                seq_lens=np.array(lens, dtype=np.int64), info=np.array(info))


def attention(q, k, v, table, seq_lens, q_starts, page, scale, window=0):
    """(out, lse, size) of q [T][q_heads][D] over values k, v [pages][heads][page][D]; size is
    the weighted sum of |v| that error bounds go by, with the largest sum of |scale q k|."""
    q = np.asarray(q, dtype=np.float64)
    tokens, q_heads, dim = q.shape
    heads = k.shape[1]
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    lse, reach = np.full((tokens, q_heads), -np.inf), np.zeros((tokens, q_heads))
    for r in range(len(seq_lens)):
        a, b, length = int(q_starts[r]), int(q_starts[r + 1]), int(seq_lens[r])
        for t in range(a, b):
            p = length - (b - a) + (t - a)
            seen = [j for j in range(max(0, p - window + 1 if window else 0),
                                     min(p + 1, table.shape[1] * page))
                    if 0 <= table[r, j // page] < k.shape[0]]
            if not seen:
                continue
            seen = np.array(seen)
            ids, off = table[r, seen // page], seen % page
            for h in range(q_heads):
                kk, vv = k[ids, h * heads // q_heads, off], v[ids, h * heads // q_heads, off]
                s = scale * (kk @ q[t, h])
                m = s.max()
                w = np.exp(s - m)
                out[t, h], size[t, h] = w @ vv / w.sum(), w @ np.abs(vv) / w.sum()
                lse[t, h] = m + math.log(w.sum())
                reach[t, h] = abs(scale) * (np.abs(kk) @ np.abs(q[t, h])).max()
    return out, lse, size, reach


def token_logprobs(x, targets, top):
    """(logprob, entropy, top_index, top_logprob) of rows of logits."""
    x = np.asarray(x, dtype=np.float64)
    rows, vocab = x.shape
    lp, ent = np.zeros(rows), np.zeros(rows)
    index, best = np.zeros((rows, top), dtype=np.int64), np.zeros((rows, top))
    for r in range(rows):
        row = x[r]
        bad = np.isnan(row).any() or np.isposinf(row).any() or np.isneginf(row).all()
        # Differences from the maximum, as m + log s would round log s away where m is huge.
        if bad:
            d, log_s, ent[r] = np.full(vocab, np.nan), np.nan, np.nan
        else:
            d = row - row.max()
            e = np.exp(d)
            log_s = math.log(e.sum())
            keep = e > 0
            ent[r] = log_s - (e[keep] * d[keep]).sum() / e.sum()
        t = int(targets[r])
        with np.errstate(invalid="ignore"):
            lp[r] = d[t] - log_s if 0 <= t < vocab else 0.0
            # NaN first, then larger values, equal ones by index.
            order = np.lexsort((np.arange(vocab), np.where(np.isnan(row), 0.0, -row), ~np.isnan(row)))
            index[r] = order[:top]
            best[r] = d[order[:top]] - log_s
    return lp, ent, index, best


def rotate(x, weight, positions, inv_freq, interleaved=False, factor=1.0, eps=1e-6):
    """Rows [T][heads][D] with each head normed (weight not None) and turned by its token's position."""
    x = np.array(x, dtype=np.float64)
    if weight is not None:
        x = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    out = x.copy()
    pairs = len(inv_freq)
    for t, p in enumerate(positions):
        for i, f in enumerate(inv_freq):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
            angle = int(p) * float(f)
            c, s = factor * math.cos(angle), factor * math.sin(angle)
            out[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
            out[t, :, b] = x[t, :, b] * c + x[t, :, a] * s
    return out


def tree_tables(parents, q_starts, seq_lens):
    """(masks as Python numbers, positions) of every token that belongs to a request, by walking up."""
    masks, positions = {}, {}
    for r, length in enumerate(seq_lens):
        a, b = q_starts[r], q_starts[r + 1]
        for i in range(b - a):
            if i >= 64:
                masks[a + i], positions[a + i] = 0, 0
                continue
            bits, j = 0, i
            while j >= 0:
                bits |= 1 << j
                up = parents[a + j]
                j = up if 0 <= up < j else -1
            masks[a + i] = bits
            positions[a + i] = max(0, max(0, length) - (b - a) + bin(bits).count("1") - 1)
    return masks, positions


def adapters(x, y, a, b, q_starts, adapter, ranks, scales):
    """y [T][N] + scale (x A^T) B^T with each request's adapter; x [T][K], a [adapters][rank][K], b [adapters][N][rank]."""
    out = np.array(y, dtype=np.float64)
    for r, i in enumerate(adapter):
        if 0 <= i < len(a):
            rows = slice(q_starts[r], q_starts[r + 1])
            h = x[rows] @ a[i][:ranks[i]].T
            out[rows] += scales[i] * (h @ b[i][:, :ranks[i]].T)
    return out
