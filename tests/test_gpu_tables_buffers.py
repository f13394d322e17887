"""Block tables whose inputs and outputs are parts of one buffer, one right after the other, and inputs
that a call refuses to write to."""
import numpy as np
import pytest

from oracle import serving_oracle as S
from paper_2607_01127_amd import logbq as L

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_parts_of_one_buffer():
    print("parts of one buffer", flush=True)
    rng = np.random.default_rng(3)
    n, page, width = 70, 16, 9
    cached = rng.integers(0, 60, n).astype(np.int32)
    new = rng.integers(0, 40, n).astype(np.int32)
    tokens = int(new.sum())
    free = rng.permutation(300).astype(np.int32)
    table = rng.integers(0, 300, (n, width)).astype(np.int32)
    want = S.batch_tables(cached, new, free, table, page, tokens)
    sizes = dict(slots=2 * tokens, cached=n, seq_lens=n, new=n, q_starts=n + 1, free=300, info=4, positions=tokens,
                 table=n * width)
    buffer, at, part = torch.full((sum(sizes.values()),), -7, dtype=torch.int32, device="cuda"), 0, {}
    for name, size in sizes.items():
        part[name] = buffer[at:at + size]
        at += size
    for name, x in (("cached", cached), ("new", new), ("free", free), ("table", table.ravel())):
        part[name].copy_(torch.from_numpy(x))
    part["slots"], part["table"] = part["slots"].view(torch.int64), part["table"].view(n, width)
    out = {k: part[k] for k in ("slots", "positions", "q_starts", "seq_lens", "info")}
    L.batch_tables(part["cached"], part["new"], part["free"], part["table"], page, tokens, out=out)
    for name in out:
        assert np.array_equal(out[name].cpu().numpy(), want[name]), name
    assert np.array_equal(part["table"].cpu().numpy(), want["table"])
    for name, x in (("cached", cached), ("new", new), ("free", free)):
        assert np.array_equal(part[name].cpu().numpy(), x), name
    # Lengths that would be updated in place.
    with pytest.raises(L.LogbqError):
        L.batch_tables(part["cached"], part["new"], part["free"], part["table"], page, tokens,
                       out=dict(out, seq_lens=part["cached"]))
