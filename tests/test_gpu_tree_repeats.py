"""Full trees over contexts that many workgroups share: within the bounds of attention_check, and the same bits at each
call, whatever the workspace held."""
import numpy as np
import pytest

from attention_check import TYPES, dev
from paper_2607_01127_amd import logbq as L
from test_gpu_tree import attend, ints, step

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,dtype", [(128, "bf16"), (128, "f32"), (64, "f16"), (256, "bf16")])
def test_long_contexts_repeat_themselves(dim, dtype):
    print("repeats", dim, dtype, flush=True)
    lens, new = [9001, 6100], [64, 37]
    q, cache, table, masks = step(dim, lens, new, 2, 4, dim, 64, dtype)
    work = torch.empty(L.KV4_WORKSPACE_BYTES, dtype=torch.uint8, device=q.device)
    res, lse = attend(q, cache, table, lens, new, masks, 64, dtype, workspace=work)
    bits = dev(np.array(masks, dtype=np.uint64).view(np.int64))
    for fill in (0, 255, 0x7f, 1):
        work.fill_(fill)
        out, sums = torch.full(q.shape, 3.0, dtype=TYPES[dtype], device=q.device), torch.full_like(lse, 3.0)
        L.kv4_tree_attention(q, cache[0], dev(table), ints(lens), ints([0, 64, 101]), bits, 64, out=out, lse=sums,
                             workspace=work)
        assert torch.equal(out, res) and torch.equal(sums, lse)
