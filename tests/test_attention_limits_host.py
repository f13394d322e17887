"""Attention calls with more row tiles than a launch holds are refused before anything is enqueued (no
GPU: a call that got as far as a launch would report a HIP error)."""
import ctypes

import pytest

from paper_2607_01127_amd import logbq as L

A = 4096                      # an aligned address that is never read on these paths


@pytest.mark.parametrize("tokens,requests,max_new,heads,group", [
    (16384 * 17, 16384, 17, 1024, 1),      # many requests, each one row past decode's
    (1 << 21, 1, 1 << 21, 1024, 1),        # one long prompt
    (1 << 20, 3, 1 << 19, 256, 16)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_more_row_tiles_than_a_launch_holds(tokens, requests, max_new, heads, group, dim):
    cache = ctypes.byref(L.Kv4Struct(k_codes=A, v_codes=A, k_scales=A, v_scales=A, pages=4, heads=heads,
                                     page=64, dim=dim))
    new = max_new + 64                  # an upper bound past what the decode kernels alone hold
    assert L.lib().logbq_kv4_attention(A, heads * group * dim, 1, tokens, heads * group, cache, A, requests, 4,
                                       A, A, new, 0.1, 0, A, 1, None, A, L.KV4_WORKSPACE_BYTES,
                                       None) == L.ERR_UNSUPPORTED
