"""Token log probabilities where the size of the logits could enter a result: rows masked with large
finite constants, rows whose largest logit is huge, and offsets common to a row. Against the float64
oracle, within bounds that do not grow with the logits.

With m the row's maximum and d = x - m, a term is exp(d): d is off by 2^-24 of itself, so a term by a
factor of at most 1 +- 2^-22 (|d| + 2), and |d| exp(d) <= 0.37, so that the sum s >= 1 of n terms and its
rounding (a chain of at most vocab / 256 + 64 additions) give at most
eps = (vocab / 256 + 64) 2^-24 + 2^-20 of log s. A log probability is d - log s: 2^-22 (|d| + log s) more.
The entropy is log s - sum d exp(d) / s, whose terms are those of the entropy itself: eps (2 + entropy).
"""
import math

import numpy as np
import pytest

from oracle import serving_oracle as S
from paper_2607_01127_amd import logbq as L

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
LOWEST = {n: torch.finfo(t).min for n, t in TYPES.items()}


def host(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def sums_bound(vocab):
    return (vocab / 256 + 64) * 2.0 ** -24 + 2.0 ** -20


def check(x, targets, top):
    got = L.token_logprobs(x, torch.tensor(targets, device=DEV), top)
    lp, ent, index, best = S.token_logprobs(host(x), targets, top)
    eps = sums_bound(x.shape[1])
    for name, want, tol in (("logprob", lp, eps + 2.0 ** -21 * np.abs(lp)),
                            ("top_logprob", best, eps + 2.0 ** -21 * np.abs(best)),
                            ("entropy", ent, eps * (2 + ent))):
        have = host(got[name])
        assert np.isfinite(have).all(), (name, have)
        assert float(np.max(np.abs(have - want) - tol, initial=-1.0)) <= 0.0, (name, have, want)
    assert np.array_equal(got["top_index"].cpu().numpy(), index)
    return got


MASKS = [-1e9, -1e10, -1e12, -1e20, -1e30, -9e37, "lowest"]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [40, 5000, 131072])
def test_finite_masks(vocab, dtype):
    """Forbidden tokens at a large finite value: all but the last 5, all but the first 5, all but a few
    in between, every other one, all but one, and all (a uniform row)."""
    print("masks", vocab, dtype, flush=True)
    g = torch.Generator(device=DEV).manual_seed(vocab)
    for mask in MASKS if dtype != "f16" else [-3e4, -6e4, "lowest"]:
        mask = LOWEST[dtype] if mask == "lowest" else mask
        x = torch.randn((6, vocab), generator=g, device=DEV)
        x[0, :-5] = mask
        x[1, 5:] = mask
        keep = x[2, vocab // 2:vocab // 2 + 7].clone()
        x[2] = mask
        x[2, vocab // 2:vocab // 2 + 7] = keep
        x[3, ::2] = mask
        x[4] = mask
        x[4, vocab // 3] = 3.0
        x[5] = mask
        x = x.to(TYPES[dtype])
        check(x, [vocab - 1, 0, vocab // 2 + 3, 1, vocab // 3, 7], 4)
        check(x, [0, vocab - 1, 0, 0, 0, 0], 0)             # masked ones


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [40, 5000, 131072])
def test_large_maxima(vocab, dtype):
    """Rows whose largest logit is huge: its log probability is 0 (never above), the others' are their
    distance; and rows in which all are huge and equal."""
    print("maxima", vocab, dtype, flush=True)
    for peak in [65504.0, 3e4] if dtype == "f16" else [65504.0, 1e6, 1e9, 1e10, 1e20, 1e30, 9e37, 3e38]:
        x = torch.zeros((4, vocab), device=DEV)
        x[0, 0] = peak
        x[1, vocab - 1] = peak
        x[2] = peak
        x[3, 3:] = -peak
        x = x.to(TYPES[dtype])
        got = check(x, [0, vocab - 1, 5, 0], 3)
        assert bool((got["logprob"] <= 0).all()) and bool((got["top_logprob"] <= 0).all())


@pytest.mark.parametrize("vocab", [40, 5000, 131072])
def test_common_offsets_change_nothing(vocab):
    """Logits on a grid of 1/8, so that the offsets are exact: only differences may enter."""
    print("offsets", vocab, flush=True)
    g = torch.Generator(device=DEV).manual_seed(vocab + 1)
    x = torch.randint(-80, 81, (3, vocab), generator=g, device=DEV) / 8
    x[2, vocab // 2] = 30.0                                 # a dominated row
    targets = [0, vocab - 1, vocab // 2]
    ref = check(x, targets, 5)
    for offset in (100.0, 1000.0, -1000.0, 60000.0, -1e6):
        got = check(x + offset, targets, 5)
        for name in ("logprob", "top_logprob", "entropy"):
            off = float((got[name] - ref[name]).abs().max())
            assert off <= 2 * sums_bound(vocab) * (2 + float(ref["entropy"].max())), (name, offset, off)
        assert torch.equal(got["top_index"], ref["top_index"])


def test_differences_past_the_range():
    """A row whose differences pass float32's range: the far ones have probability 0."""
    print("differences", flush=True)
    x = torch.randn((2, 3000), device=DEV, generator=torch.Generator(device=DEV).manual_seed(2))
    x[0, ::3] = -3.4e38
    x[0, 7] = 3e38
    x[1, ::3] = -math.inf
    x[1, 1::3] = torch.finfo(torch.float32).min
    got = L.token_logprobs(x, torch.tensor([7, 5], device=DEV), 2)
    lp, ent, index, _ = S.token_logprobs(host(x), [7, 5], 2)
    assert np.allclose(host(got["logprob"]), lp, rtol=2.0 ** -21, atol=sums_bound(3000))
    assert np.allclose(host(got["entropy"]), ent, atol=sums_bound(3000) * (2 + ent.max()))
    assert np.array_equal(got["top_index"].cpu().numpy(), index)
