"""Every form of the prompt kernel: float32 and bfloat16 queries at each head size, pages within and past a
tile, chunks beside single tokens, and tables of the largest context (positions worked on in splits)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from attention_check import TYPES, attend, cache_of, dev  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("f32", "f16"), ("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("heads,group,dim,page", [(2, 4, 128, 64), (2, 4, 128, 16), (1, 16, 64, 128), (3, 1, 64, 32),
                                                  (1, 2, 256, 64), (2, 3, 256, 16)])
def test_prompts(heads, group, dim, page, dtype, out):
    """One prompt; chunks behind a cached part; prompts beside single tokens and empty requests; whole and
    windowed, in narrow tables and in tables of 32768 positions."""
    print("prompts", heads, group, dim, page, dtype, out, flush=True)
    rng = np.random.default_rng(dim + page)
    pages = 24
    cache = cache_of(rng.standard_normal((pages, heads, page, dim)), rng.standard_normal((pages, heads, page, dim)))
    for lens, new in (([211], [211]), ([400], [67]), ([300, 1, 0, 129, 90], [70, 1, 1, 129, 1])):
        for span in (448, 32768):
            table = np.full((len(lens), -(-span // page)), -1, dtype=np.int32)
            for r, n in enumerate(lens):
                table[r, :-(-n // page)] = rng.integers(0, pages, -(-n // page))
            q = dev(rng.standard_normal((sum(new), heads * group, dim)), torch.float32).to(TYPES[dtype])
            attend(q, cache, table, lens, new, page, window=0 if span > 448 else 150, out=out)
