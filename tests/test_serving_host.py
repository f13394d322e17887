"""Host-side checks of the serving operators (no GPU): every refusal of the entry points comes
before any HIP call, the binding refuses tensors that do not fit, and the oracle agrees with
worked values and with brute force."""
import ctypes

import numpy as np
import pytest

from oracle import serving_oracle as S
from paper_2607_01127_amd import logbq as L

torch = pytest.importorskip("torch")
A, B = 4096, 4104          # an aligned address and one that is not; never read on these paths
BAD, NO = L.ERR_INVALID_ARG, L.ERR_UNSUPPORTED


def cache(**kw):
    f = dict(k_codes=A, v_codes=A, k_scales=A, v_scales=A, pages=4, heads=2, page=64, dim=128)
    f.update(kw)
    return ctypes.byref(L.Kv4Struct(**f))


def test_empty_calls_need_nothing():
    h = L.lib()
    none = cache(k_codes=None, v_codes=None, k_scales=None, v_scales=None, pages=0)
    assert h.logbq_kv4_append(None, 0, None, 0, 0, 0, none, None, None) == L.OK
    assert h.logbq_kv4_read(none, None, 0, None, None, 1, None) == L.OK
    assert h.logbq_kv4_attention(None, 0, 1, 0, 2, none, None, 0, 0, None, None, 0, 1.0, 0, None, 1,
                                 None, None, 0, None) == L.OK
    assert h.logbq_token_logprobs(None, 0, 0, 5, 5, None, 0, None, None, None, None, None, 0,
                                  None) == L.OK


@pytest.mark.parametrize("change,status", [
    (dict(requests=-1), BAD), (dict(free_count=-1), BAD), (dict(width=-1), BAD),
    (dict(tokens=-1), BAD), (dict(page=8), NO), (dict(page=48), NO), (dict(page=2048), NO),
    (dict(requests=4097), NO), (dict(width=1 << 31), NO), (dict(tokens=1 << 31), NO),
    (dict(free_count=1 << 31), NO), (dict(cached=None), BAD), (dict(new=None), BAD),
    (dict(free=None), BAD), (dict(table=None), BAD), (dict(slots=None), BAD),
    (dict(positions=None), BAD), (dict(starts=None), BAD), (dict(lens=None), BAD),
    (dict(info=None), BAD)])
def test_batch_tables_refusals(change, status):
    f = dict(cached=A, new=A, requests=3, free=A, free_count=5, table=A, width=4, page=16, tokens=7,
             slots=A, positions=A, starts=A, lens=A, info=A)
    f.update(change)
    assert L.lib().logbq_batch_tables(*f.values(), None) == status


CACHES = [(dict(k_codes=None), BAD), (dict(v_codes=None), BAD), (dict(k_scales=None), BAD),
          (dict(v_scales=None), BAD), (dict(pages=-1), BAD), (dict(heads=0), BAD),
          (dict(dim=96), NO), (dict(page=24), NO), (dict(page=8), NO), (dict(page=2048), NO),
          (dict(heads=1025), NO), (dict(pages=1 << 26), NO), (dict(k_codes=B), NO),
          (dict(v_codes=B), NO), (dict(k_scales=B), NO), (dict(v_scales=B), NO)]


@pytest.mark.parametrize("change,status", CACHES)
def test_cache_refusals(change, status):
    h, c = L.lib(), cache(**change)
    assert h.logbq_kv4_append(A, 256, A, 256, 1, 3, c, A, None) == status
    assert h.logbq_kv4_read(c, A, 3, A, A, 1, None) == status
    assert h.logbq_kv4_attention(A, 512, 1, 3, 4, c, A, 1, 4, A, A, 3, 1.0, 0, A, 1, None, A,
                                 L.KV4_WORKSPACE_BYTES, None) == status


def test_append_and_read_refusals():
    h, c = L.lib(), cache()
    append = lambda *a: h.logbq_kv4_append(*a, None)  # noqa: E731
    assert append(A, 256, A, 256, 1, -1, c, A) == BAD
    assert append(A, 256, A, 256, 1, 3, None, A) == BAD
    assert append(None, 256, A, 256, 1, 3, c, A) == BAD
    assert append(A, 256, None, 256, 1, 3, c, A) == BAD
    assert append(A, 256, A, 256, 1, 3, c, None) == BAD
    assert append(A, 256, A, 256, 3, 3, c, A) == NO           # no such type
    assert append(A, 255, A, 256, 1, 3, c, A) == NO           # rows overlap
    assert append(A, 256, A, 260, 1, 3, c, A) == NO           # rows not 16-byte aligned
    assert append(B, 256, A, 256, 1, 3, c, A) == NO
    assert append(A, 256, B, 256, 1, 3, c, A) == NO
    assert append(A, 256, A, 256, 1, 1 << 31, c, A) == NO
    assert append(A, 1 << 60, A, 256, 1, 1 << 20, c, A) == NO
    read = lambda *a: h.logbq_kv4_read(*a, None)  # noqa: E731
    assert read(c, A, -1, A, A, 1) == BAD
    assert read(None, A, 1, A, A, 1) == BAD
    assert read(c, None, 1, A, A, 1) == BAD
    assert read(c, A, 1, None, A, 1) == BAD
    assert read(c, A, 1, A, B, 1) == NO
    assert read(c, A, 1, A, A, 7) == NO


@pytest.mark.parametrize("change,status", [
    (dict(q=None), BAD), (dict(tokens=-1), BAD), (dict(requests=-1), BAD), (dict(width=-1), BAD),
    (dict(max_new=-1), BAD), (dict(window=-1), BAD), (dict(q_heads=0), BAD), (dict(cache=None), BAD),
    (dict(scale=float("nan")), BAD), (dict(scale=float("inf")), BAD), (dict(table=None), BAD),
    (dict(lens=None), BAD), (dict(starts=None), BAD), (dict(out=None), BAD), (dict(work=None), BAD),
    (dict(work_bytes=-1), BAD), (dict(work_bytes=0), NO), (dict(work=B), NO),
    (dict(q_heads=5), NO), (dict(q_heads=34, stride=34 * 128), NO), (dict(q_dtype=3), NO),
    (dict(out_dtype=-1), NO), (dict(stride=511), NO), (dict(stride=516), NO), (dict(q=B), NO),
    (dict(out=B), NO), (dict(width=1 << 26), NO), (dict(tokens=1 << 31), NO),
    (dict(requests=1 << 31), NO)])
def test_attention_refusals(change, status):
    f = dict(q=A, stride=512, q_dtype=1, tokens=3, q_heads=4, cache=cache(), table=A, requests=2,
             width=4, lens=A, starts=A, max_new=2, scale=0.1, window=0, out=A, out_dtype=1,
             lse=None, work=A, work_bytes=L.KV4_WORKSPACE_BYTES)
    f.update(change)
    assert L.lib().logbq_kv4_attention(*f.values(), None) == status


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), BAD), (dict(vocab=0), BAD), (dict(top=-1), BAD), (dict(top=11), BAD),
    (dict(vocab=99, stride=99, top=33), NO), (dict(dtype=5), NO), (dict(stride=9), NO),
    (dict(logits=None), BAD), (dict(targets=None), BAD), (dict(logprob=None), BAD),
    (dict(entropy=None), BAD), (dict(index=None), BAD), (dict(best=None), BAD),
    (dict(work=None), BAD), (dict(work=B), NO), (dict(work_bytes=64), NO), (dict(logits=4098), NO),
    (dict(vocab=1 << 31, stride=1 << 31), NO), (dict(tokens=1 << 31), NO)])
def test_logprobs_refusals(change, status):
    f = dict(logits=A, dtype=0, tokens=2, vocab=10, stride=10, targets=A, top=3, logprob=A,
             entropy=A, index=A, best=A, work=A, work_bytes=L.LOGPROBS_WORKSPACE_BYTES)
    f.update(change)
    assert L.lib().logbq_token_logprobs(*f.values(), None) == status


def test_more_rows_than_a_launch_holds_are_refused():
    h, c = L.lib(), cache()
    most = (1 << 28) - 16
    assert h.logbq_kv4_append(A, 256, A, 256, 1, most, c, A, None) == NO
    assert h.logbq_kv4_read(c, A, most, A, A, 1, None) == NO
    assert h.logbq_token_logprobs(A, 0, 1 << 24, 10, 10, A, 0, A, A, None, None, A,
                                  L.LOGPROBS_WORKSPACE_BYTES, None) == NO


def test_binding_refuses_host_tensors_and_wrong_shapes():
    i32 = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        L.batch_tables(i32, i32, i32, torch.zeros((3, 2), dtype=torch.int32), 16, 4)
    host = L.kv4_cache(2, 2, 64, 16, device="cpu")
    with pytest.raises(ValueError):
        L.kv4_append(torch.zeros(1, 2, 64), torch.zeros(1, 2, 64), host, torch.zeros(1, dtype=torch.int64))
    with pytest.raises(ValueError):
        L.kv4_cache(2, 2, 96)
    with pytest.raises(ValueError):
        L.kv4_cache(2, 2, 64, 20)
    with pytest.raises(ValueError):
        L.token_logprobs(torch.zeros(2, 5), torch.zeros(2, dtype=torch.int64))


# ------------------------------------------------------------------ the oracle's own pins

def test_oracle_scale_is_the_smallest_that_holds():
    rng = np.random.default_rng(5)
    for x in np.concatenate([np.exp(rng.uniform(-60, 60, 500)), [2.0 ** -126, 1.0, 6.0, 1e-45]]):
        s = S.bf16_up(float(np.float32(x)) / 6.0)
        bits = np.float32(s).view(np.uint32)
        assert float(np.float32(s)) == s and bits & 0xffff == 0
        below = float(np.array(bits - 0x10000, dtype=np.uint32).view(np.float32))
        assert 6 * s >= float(np.float32(x)) > 6 * below


def test_oracle_codes_worked():
    # max 6: scale 1; each threshold belongs to the larger magnitude.
    row = np.array([6.0, 5.0, -4.99, 3.5, 2.5, -1.75, 1.25, 0.75, 0.25, -0.24, 0.0, np.nan, -np.inf])
    codes, scale = S.kv4_quantize(row)
    assert scale == 1.0
    assert codes.tolist() == [7, 7, 14, 6, 5, 12, 3, 2, 1, 0, 0, 0, 15]
    values = S.kv4_values(codes, scale)
    assert values.tolist() == [6, 6, -4, 4, 3, -2, 1.5, 1, 0.5, 0, 0, 0, -6]
    zero, scale = S.kv4_quantize(np.array([0.0, -0.0, np.nan, np.inf]))
    assert scale == 0.0 and not zero.any()


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_oracle_layouts_invert(dim):
    rng = np.random.default_rng(dim)
    codes = rng.integers(0, 16, (3, 2, 16, dim), dtype=np.uint8)
    assert np.array_equal(S.unpack_keys(S.pack_keys(codes)), codes)
    packed = S.pack_values(codes)
    assert packed.shape == (3, 2, 2, 16, 8, dim // 32)
    assert np.array_equal(S.unpack_values(packed), codes)


def test_oracle_attention_and_logprobs_by_brute_force():
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((2, 1, 16, 8)), rng.standard_normal((2, 1, 16, 8))
    q = rng.standard_normal((2, 1, 8))
    out, lse, _, _ = S.attention(q, k, v, np.array([[1, 0]]), [18], [0, 2], 16, 0.5, window=5)
    rows_k, rows_v = np.concatenate([k[1, 0], k[0, 0]]), np.concatenate([v[1, 0], v[0, 0]])
    for t, p in ((0, 16), (1, 17)):
        e = np.exp(0.5 * rows_k[p - 4:p + 1] @ q[t, 0])
        assert np.allclose(out[t, 0], e @ rows_v[p - 4:p + 1] / e.sum(), rtol=1e-12)
        assert np.isclose(lse[t, 0], np.log(e.sum()), rtol=1e-12)
    x = np.array([[1.0, 3.0, -np.inf, 3.0], [0.0, 0.0, 0.0, 0.0]])
    lp, ent, index, best = S.token_logprobs(x, [0, 7], 2)
    total = np.exp(1) + 2 * np.exp(3)
    assert np.isclose(lp[0], 1 - np.log(total)) and lp[1] == 0
    assert np.isclose(ent[1], np.log(4)) and index.tolist() == [[1, 3], [0, 1]]
    assert np.allclose(best[0], 3 - np.log(total))


def test_oracle_tables_worked():
    got = S.batch_tables([0, 20, 16], [3, 12, 1], [9, 8, 7, 6], [[-1, -1], [4, 5], [3, -1]], 16, 18)
    assert got["table"].tolist() == [[9, -1], [4, 5], [3, 8]]
    assert got["slots"].tolist() == [144, 145, 146] + list(range(84, 96)) + [128, -1, -1]
    assert got["positions"].tolist() == [0, 1, 2] + list(range(20, 32)) + [16, 0, 0]
    assert got["q_starts"].tolist() == [0, 3, 15, 16] and got["seq_lens"].tolist() == [3, 32, 17]
    assert got["info"].tolist() == [16, 2, 32, 0]
