"""Few rows of logits, whose parts different workgroups sum and the last one to finish joins: what it
joins is what the others stored, in every call."""
import pytest

from paper_2607_01127_amd import logbq as L

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("tokens,top", [(1, 32), (16, 20), (16, 0), (170, 5)])
def test_parts_are_joined_as_stored(tokens, top):
    """Two inputs in turn through one workspace: each call's results are bit for bit those of the
    input's first call, so no part is taken before it is stored or after it is cleared. The inputs
    differ by more than any rounding, and the exact results of a uniform row are known."""
    print("parts", tokens, top, flush=True)
    vocab = 131072
    g = torch.Generator(device=DEV).manual_seed(tokens)
    a = torch.randn((tokens, vocab), generator=g, device=DEV)
    b = 3 * torch.randn((tokens, vocab), generator=g, device=DEV) + 1
    t = torch.randint(0, vocab, (tokens,), generator=g, device=DEV)
    work = torch.zeros(L.LOGPROBS_WORKSPACE_BYTES, dtype=torch.uint8, device=DEV)
    first = [L.token_logprobs(x, t, top, workspace=work) for x in (a, b)]
    uniform = torch.zeros_like(a)
    out = [{n: torch.empty_like(v) for n, v in first[0].items()} for _ in range(150)]
    for i in range(0, 150, 3):
        for k, x in enumerate((a, b, uniform)):
            L.token_logprobs(x, t, top, out=out[i + k], workspace=work)
    torch.cuda.synchronize()
    assert not work.any()
    for i in range(150):
        if i % 3 < 2:
            assert all(torch.equal(first[i % 3][n], out[i][n]) for n in out[i]), i
        else:
            # 131072 terms of 1: the sum and its logarithm to base 2 are whole numbers.
            want = torch.tensor(-17 * 0.6931471805599453, device=DEV)
            assert float((out[i]["logprob"] - want).abs().max()) <= 2.0 ** -20, i
            assert float((out[i]["entropy"] + want).abs().max()) <= 2.0 ** -20, i
            assert torch.equal(out[i]["top_index"], torch.arange(top, device=DEV, dtype=torch.int32).repeat(tokens, 1)), i
