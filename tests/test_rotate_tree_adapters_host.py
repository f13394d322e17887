"""Host-side checks (no GPU) of rotation, rotated appends, draft trees and adapters: every refusal comes
before any HIP call, the binding refuses tensors that do not fit, and the oracle agrees with worked values."""
import ctypes
import math

import numpy as np
import pytest

from oracle import serving_oracle as S
from paper_2607_01127_amd import logbq as L

torch = pytest.importorskip("torch")
# Addresses far apart, an aligned one for each buffer, and one that is not aligned; never read on these paths.
A, Q, K, V, QO, KO, W, P, C = (i << 32 for i in range(1, 10))
BAD, NO = L.ERR_INVALID_ARG, L.ERR_UNSUPPORTED


def cache(**kw):
    f = dict(k_codes=C, v_codes=C, k_scales=C, v_scales=C, pages=4, heads=2, page=64, dim=128)
    f.update(kw)
    return ctypes.byref(L.Kv4Struct(**f))


def rotation(inv_freq=W + 4096, pairs=64, interleaved=0, factor=1.0):
    return ctypes.byref(L.RotationStruct(inv_freq, pairs, interleaved, factor))


ROTATIONS = [(dict(rotation=None), BAD), (dict(rotation=rotation(pairs=-1)), BAD),
             (dict(rotation=rotation(factor=math.inf)), BAD), (dict(rotation=rotation(interleaved=2)), BAD),
             (dict(rotation=rotation(inv_freq=None)), BAD), (dict(rotation=rotation(pairs=72)), NO),
             (dict(rotation=rotation(pairs=20)), NO), (dict(eps=-1e-9), BAD), (dict(eps=math.nan), BAD),
             (dict(eps=math.inf), BAD), (dict(positions=None), BAD), (dict(q_weight=W + 4), NO),
             (dict(k_weight=W + 8), NO), (dict(dtype=3), NO), (dict(out_dtype=-1), NO), (dict(tokens=-1), BAD),
             (dict(tokens=1 << 26), NO), (dict(q_heads=-1), BAD), (dict(q_heads=16385), NO), (dict(q=None), BAD),
             (dict(k=None), BAD), (dict(q_out=None), BAD), (dict(q=Q + 8), NO), (dict(k=K + 8), NO),
             (dict(q_out=QO + 8), NO), (dict(q_stride=511), NO), (dict(q_stride=516), NO), (dict(k_stride=255), NO),
             (dict(k_stride=260), NO), (dict(q_stride=1 << 60), NO), (dict(q_out=Q + 64), BAD),
             (dict(q_out=K), BAD), (dict(q_out=W), BAD), (dict(q_out=P - 16), BAD), (dict(q_out=Q, out_dtype=0), BAD),
             (dict(q_out=Q, q_stride=520), BAD)]


@pytest.mark.parametrize("change,status", ROTATIONS + [
    (dict(dim=96), NO), (dict(k_heads=-1), BAD), (dict(k_heads=1025), NO), (dict(k_out=None), BAD),
    (dict(k_out=KO + 2), NO), (dict(k_out=QO + 512), BAD), (dict(k_out=Q), BAD), (dict(k_out=K, out_dtype=0), BAD)])
def test_qk_rotate_refusals(change, status):
    f = dict(q=Q, q_stride=512, q_heads=4, q_weight=W, k=K, k_stride=256, k_heads=2, k_weight=W, dtype=1, tokens=3,
             dim=128, eps=1e-6, positions=P, rotation=rotation(), q_out=QO, k_out=KO, out_dtype=1)
    f.update(change)
    assert L.lib().logbq_qk_rotate(*f.values(), None) == status


@pytest.mark.parametrize("change,status", ROTATIONS + [
    (dict(cache=None), BAD), (dict(cache=cache(dim=96)), NO), (dict(cache=cache(k_codes=C + 8)), NO),
    (dict(cache=cache(page=24)), NO), (dict(v=None), BAD), (dict(v=V + 8), NO), (dict(v_stride=255), NO),
    (dict(v_stride=260), NO), (dict(slots=None), BAD), (dict(q_out=V), BAD), (dict(q_out=A), BAD)])
def test_append_rotated_refusals(change, status):
    f = dict(q=Q, q_stride=512, q_heads=4, q_weight=W, k=K, k_stride=256, k_weight=W, v=V, v_stride=256, dtype=1,
             tokens=3, eps=1e-6, positions=P, rotation=rotation(), cache=cache(), slots=A, q_out=QO, out_dtype=1)
    f.update(change)
    assert L.lib().logbq_kv4_append_rotated(*f.values(), None) == status


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), BAD), (dict(requests=-1), BAD), (dict(tokens=1 << 31), NO), (dict(requests=1 << 26), NO),
    (dict(parents=None), BAD), (dict(starts=None), BAD), (dict(lens=None), BAD), (dict(masks=None), BAD),
    (dict(positions=None), BAD), (dict(masks=A), BAD), (dict(positions=A + 8), BAD), (dict(positions=Q + 8), BAD),
    (dict(positions=K + 12), BAD), (dict(masks=V), BAD)])
def test_tree_tables_refusals(change, status):
    f = dict(parents=A, tokens=7, starts=K, lens=V, requests=3, masks=Q, positions=P)
    f.update(change)
    assert L.lib().logbq_tree_tables(*f.values(), None) == status


@pytest.mark.parametrize("change,status", [
    (dict(q=None), BAD), (dict(tokens=-1), BAD), (dict(requests=-1), BAD), (dict(width=-1), BAD),
    (dict(max_new=-1), BAD), (dict(max_new=65), NO), (dict(window=-1), BAD), (dict(window=1), NO),
    (dict(window=63), NO), (dict(masks=None), BAD), (dict(masks=A + 4), NO), (dict(q_heads=0), BAD),
    (dict(cache=None), BAD), (dict(scale=math.nan), BAD), (dict(table=None), BAD), (dict(lens=None), BAD),
    (dict(starts=None), BAD), (dict(out=None), BAD), (dict(work=None), BAD), (dict(work_bytes=0), NO),
    (dict(work=A + 8), NO), (dict(q_heads=5), NO), (dict(q_heads=34, stride=34 * 128), NO), (dict(q_dtype=3), NO),
    (dict(out_dtype=3), NO), (dict(stride=511), NO), (dict(stride=516), NO), (dict(q=A + 8), NO),
    (dict(out=A + 8), NO), (dict(width=1 << 26), NO), (dict(requests=1 << 16, width=1 << 14), NO)])
def test_tree_attention_refusals(change, status):
    f = dict(q=A, stride=512, q_dtype=1, tokens=3, q_heads=4, cache=cache(), table=A, requests=2, width=4, lens=A,
             starts=A, masks=A, max_new=2, scale=0.1, window=0, out=A, out_dtype=1, lse=None, work=A,
             work_bytes=L.KV4_WORKSPACE_BYTES)
    f.update(change)
    assert L.lib().logbq_kv4_tree_attention(*f.values(), None) == status


def adapters_call(**change):
    f = dict(x=Q, tokens=5, k=64, count=2, a=[A, A], b=[K, K], n=[100, 7], dtype=1, adapters=3, rank=16, ranks=W,
             scales=W, starts=P, adapter=P, requests=2, max_new=4, y=[V, V + 4096], out=[QO, QO + 4096], work=KO,
             work_bytes=1 << 22)
    f.update(change)
    p = ctypes.c_void_p * 4
    for name in ("a", "b", "y", "out"):
        f[name] = None if f[name] is None else p(*f[name])
    f["n"] = None if f["n"] is None else (ctypes.c_int64 * 4)(*f["n"])
    return L.lib().logbq_linear_adapters(*f.values(), None)


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), BAD), (dict(k=-32), BAD), (dict(count=0), BAD), (dict(count=5), BAD), (dict(a=None), BAD),
    (dict(b=None), BAD), (dict(n=None), BAD), (dict(y=None), BAD), (dict(out=None), BAD), (dict(n=[100, -1]), BAD),
    (dict(dtype=0), NO), (dict(dtype=3), NO), (dict(adapters=-1), BAD), (dict(rank=0), BAD), (dict(rank=12), NO),
    (dict(rank=136), NO), (dict(k=48), NO), (dict(requests=-1), BAD), (dict(max_new=-1), BAD), (dict(x=None), BAD),
    (dict(starts=None), BAD), (dict(adapter=None), BAD), (dict(work=None), BAD), (dict(work_bytes=-1), BAD),
    (dict(work_bytes=5 * 16 * 2 * 16 * 4 + 6 * 16 - 1), NO), (dict(x=Q + 8), NO), (dict(work=KO + 8), NO),
    (dict(a=[A, None]), BAD), (dict(b=[None, K]), BAD), (dict(a=[A, A + 2]), NO), (dict(b=[K + 8, K]), NO),
    (dict(y=[V, V + 2]), NO), (dict(out=[QO, QO + 2]), NO), (dict(y=[None, V]), BAD), (dict(out=[QO, None]), BAD),
    (dict(out=[QO, QO + 4]), BAD), (dict(out=[Q, QO]), BAD), (dict(out=[V + 4, QO]), BAD), (dict(out=[QO, V]), BAD),
    (dict(out=[KO + 4096, QO]), BAD), (dict(out=[W, QO]), BAD), (dict(out=[P, QO]), BAD), (dict(out=[A, QO]), BAD),
    (dict(out=[K, QO]), BAD), (dict(n=[100, 1 << 31]), NO), (dict(n=[100, 65536 * 256]), NO),
    (dict(tokens=1 << 31), NO), (dict(requests=1 << 31), NO), (dict(adapters=1 << 31), NO), (dict(requests=1 << 25), NO)])
def test_adapters_refusals(change, status):
    assert adapters_call(**change) == status


def test_adapters_workspace():
    size = L.linear_adapters_workspace_bytes
    assert size(0, 1, 8) == 16 and size(1, 1, 8) == 16 * 8 * 4 + 32 and size(5, 2, 16) == 5 * 16 * 2 * 16 * 4 + 6 * 16
    assert size(100000, 4, 128) == 100000 * 4 * 128 * 4 + 16 * 103126      # no split: one part a token
    assert size(4000, 1, 8) == 32768 * 8 * 4 + 16 * 4126                   # split in eight at most
    assert size(-1, 1, 8) == size(5, 0, 8) == size(5, 5, 8) == size(5, 1, 12) == size(5, 1, 136) == 0


def test_empty_calls_need_nothing():
    h = L.lib()
    none = cache(k_codes=None, v_codes=None, k_scales=None, v_scales=None, pages=0)
    assert h.logbq_qk_rotate(None, 0, 4, None, None, 0, 2, None, 1, 0, 128, 1e-6, None, rotation(), None, None, 1,
                             None) == L.OK
    assert h.logbq_qk_rotate(None, 0, 0, None, None, 0, 0, None, 1, 9, 128, 1e-6, None, rotation(), None, None, 1,
                             None) == L.OK
    assert h.logbq_kv4_append_rotated(None, 0, 4, None, None, 0, None, None, 0, 1, 0, 1e-6, None, rotation(), none,
                                      None, None, 1, None) == L.OK
    assert h.logbq_tree_tables(None, 0, None, None, 4, None, None, None) == L.OK
    assert h.logbq_kv4_tree_attention(None, 0, 1, 0, 2, none, None, 0, 0, None, None, None, 0, 1.0, 0, None, 1, None,
                                      None, 0, None) == L.OK
    nothing = [None, None]
    assert adapters_call(tokens=0, x=None, a=nothing, b=nothing, y=nothing, out=nothing, starts=None, adapter=None,
                         work=None, work_bytes=0) == L.OK


def test_binding_refuses_host_tensors_and_wrong_shapes():
    i32, i64 = torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)
    rows = torch.zeros(3, 2, 64)
    turn = L.Rotation(torch.ones(32))
    with pytest.raises(ValueError):
        L.tree_tables(i32, torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        L.qk_rotate(rows, rows, i32, turn)
    host = L.kv4_cache(2, 2, 64, 16, device="cpu")
    with pytest.raises(ValueError):
        L.kv4_append_rotated(rows, rows, rows, host, i64, i32, turn)
    with pytest.raises(ValueError):
        L.kv4_tree_attention(rows, host, torch.zeros((1, 1), dtype=torch.int32), i32[:1], i32[:2], i64, 3)
    with pytest.raises(ValueError):
        L.linear_adapters(torch.zeros(3, 64).half(), [torch.zeros(3, 8)], [torch.zeros(1, 8, 64).half()],
                          [torch.zeros(1, 8, 8).half()], i32[:2], i32[:1], 3)


# ------------------------------------------------------------------ the oracle's own pins

def test_oracle_rotation_worked():
    # A quarter turn, once as halves and once as pairs; the norm before it has a root mean square of 5.
    x = np.array([[[3.0, 4.0, 5.0, 0.0]]]) * np.sqrt(2)
    quarter = [math.pi / 2, 0.0]
    assert np.allclose(S.rotate(x, None, [1], quarter)[0, 0] / np.sqrt(2), [-5, 4, 3, 0])
    assert np.allclose(S.rotate(x, None, [1], quarter, interleaved=True)[0, 0] / np.sqrt(2), [-4, 3, 5, 0])
    got = S.rotate(x, np.array([1.0, 2.0, 1.0, 1.0]), [0], quarter, factor=2.0, eps=0.0)[0, 0]
    assert np.allclose(got, 2 * np.sqrt(2) * np.array([3, 8, 5, 0]) / 5)
    assert np.allclose(S.rotate(x, None, [3], [0.25])[0, 0, 2:], x[0, 0, 2:])


def test_oracle_rotation_keeps_lengths_and_adds_angles():
    rng = np.random.default_rng(0)
    x, f = rng.standard_normal((3, 2, 8)), rng.uniform(0, 1, 4)
    once = S.rotate(x, None, [3, 5, 7], f)
    assert np.allclose(np.linalg.norm(once, axis=-1), np.linalg.norm(x, axis=-1))
    assert np.allclose(S.rotate(once, None, [4, 2, 0], f), S.rotate(x, None, [7, 7, 7], f))


def test_oracle_tree_tables_worked():
    # 0 - 1 - 3, 0 - 2, and a second root 4; a parent that is not before its node counts as none.
    masks, positions = S.tree_tables([-1, 0, 0, 1, 9, -1, 1], [0, 5, 7], [105, 2])
    assert masks == {0: 1, 1: 3, 2: 5, 3: 11, 4: 16, 5: 1, 6: 2}
    assert positions == {0: 100, 1: 101, 2: 101, 3: 102, 4: 100, 5: 0, 6: 0}


def test_oracle_adapters_worked():
    x, y = np.array([[1.0, 2.0], [3.0, 4.0], [5.0, 6.0]]), np.ones((3, 1))
    a, b = np.array([[[1.0, 0.0], [0.0, 9.0]], [[1.0, 1.0], [1.0, -1.0]]]), np.array([[[2.0, 9.0]], [[1.0, 3.0]]])
    got = S.adapters(x, y, a, b, [0, 1, 2, 3], [0, -1, 1], [1, 2], [10.0, 1.0])
    assert got[:, 0].tolist() == [1 + 10 * 2 * 1, 1, 1 + 11 - 3]
