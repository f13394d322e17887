"""Attention over the 4-bit cache against float64, with a bound that each position enters by its own
logit: a far position whose logit is huge but whose weight is nothing adds nothing to it.

A logit s_j = scale q . k_j with R_j = |scale| sum_i |q_i k_ji|: products of float16 queries (or of two
float16 numbers, to 2^-22 of a float32 query) and codes are exact, their float32 sum has a relative error
of at most (D + 4) 2^-24 of R_j, scaling and exp2 add at most 2^-21 (R_j + 2). So it is off by at most
d_j = (D + 16) 2^-23 (R_j + 2). With weights p_j (sum 1) over N positions:
  log sum: sum p_j d_j, N 2^-24 of the sum's rounding, and 2^-22 of its own size;
  output:  each weight is off by a factor 1 +- 2 d_j, and 2^-15 for the 16 bits in which it is
           multiplied with a value, and so is the normalisation: sum p_j (2 d_j + 2^-15) (|v_j| + A) with
           A = sum p_j |v_j|, N 2^-23 A for the sums, and half an ulp of the output's type; weights
           below 2^-126 of the largest are 0 in float32: N 2^-126 of the largest |v_j|.
"""
import math

import numpy as np
import torch

from oracle import serving_oracle as S
from paper_2607_01127_amd import logbq as L

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
    return t if dtype is None else t.to(dtype)


def host(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def cache_of(k, v):
    """A Kv4Cache of rows k, v [pages][heads][page][D], and the values it stands for."""
    kc, ks = S.kv4_quantize(k)
    vc, vs = S.kv4_quantize(v)
    bf = lambda s: dev(s.astype(np.float32), torch.bfloat16)  # noqa: E731
    buffers = L.Kv4Cache(dev(S.pack_keys(kc)), bf(ks), dev(S.pack_values(vc)), bf(vs))
    return buffers, S.kv4_values(kc, ks), S.kv4_values(vc, vs)


def exact(q, k, v, table, lens, starts, page, scale, window):
    """(out, lse, bound of out before its rounding, bound of lse); lse is -inf where nothing is seen."""
    tokens, q_heads, dim = q.shape
    heads = k.shape[1]
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    lse, lse_tol = np.full((tokens, q_heads), -np.inf), np.zeros((tokens, q_heads))
    for r in range(len(lens)):
        a, b, length = int(starts[r]), int(starts[r + 1]), int(lens[r])
        for t in range(a, b):
            p = length - (b - a) + (t - a)
            j = np.arange(max(0, p - window + 1 if window else 0), min(p + 1, table.shape[1] * page))
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


def attend(q, cache, table, lens, new, page, out="f32", scale=None, window=0, max_new=None, rows=None):
    """One call on q [tokens][q_heads][D] (a device tensor), checked; `rows` (a mask of [tokens][q_heads])
    limits the check. Returns its results."""
    buffers, k, v = cache
    table = np.asarray(table, dtype=np.int32)
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    scale = q.shape[2] ** -0.5 if scale is None else scale
    lse = torch.full(q.shape[:2], 7.0, device=DEV)
    res = torch.full(q.shape, math.nan, device=DEV, dtype=TYPES[out])
    L.kv4_attention(q, buffers, dev(table), dev(np.asarray(lens, dtype=np.int32)), dev(starts),
                    max(new) if max_new is None else max_new, scale=scale, window=window, out=res, lse=lse)
    ref, ref_lse, tol, lse_tol = exact(host(q), k, v, table, lens, starts, page, scale, window)
    got, got_lse = host(res), host(lse)
    rows = np.ones(q.shape[:2], dtype=bool) if rows is None else rows
    got, got_lse, ref, ref_lse, tol, lse_tol = (x[rows] for x in (got, got_lse, ref, ref_lse, tol, lse_tol))
    empty = np.isneginf(ref_lse)
    wrong = np.flatnonzero(np.isneginf(got_lse) != empty)
    assert wrong.size == 0, (wrong.size, wrong[:5], got_lse[wrong[:5]], ref_lse[wrong[:5]])
    assert not got[empty].any() and not np.isnan(got).any()
    off = np.abs(got_lse[~empty] - ref_lse[~empty]) / lse_tol[~empty]
    assert float(np.max(off, initial=0.0)) <= 1.0, float(off.max())
    tol = tol + HALF_ULP[out] * np.abs(ref) + (2.0 ** -25 if out == "f16" else 0.0)
    off = np.abs(got - ref) / np.where(tol > 0, tol, 1e-300)
    assert float(np.max(off, initial=0.0)) <= 1.0, float(off.max())
    return res, lse
