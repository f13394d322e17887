"""The serving example: batches of one decoder that live side by side, and what its calls refuse."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_batches_of_one_decoder_do_not_share_pages():
    """Two batches in turn on one decoder give bit for bit what each gives on a decoder of its own: the
    pages are others, the positions and values are not."""
    from paper_2607_01127_amd.serve_example import Batch, Decoder, Shape
    print("two batches", flush=True)
    shape = Shape(layers=1)
    texts = [[list(range(40)), [7, 8, 9]], [list(range(100, 163)), [5]]]
    steps = [[[1], [2]], [[3], [4]], [[5, 6, 7], [8]]]

    def logits(batch, text):
        yield batch.step(text)
        for s in steps:
            yield batch.step(s)

    alone = [list(logits(Batch(Decoder(shape, pages=40, page=16, seed=6), 2, 128), t)) for t in texts]
    both = Decoder(shape, pages=40, page=16, seed=6)
    together = zip(*(logits(Batch(both, 2, 128), t) for t in texts))
    for i, pair in enumerate(together):
        for k in range(2):
            assert torch.equal(pair[k], alone[k][i]), (i, k)
    used = sum(-(-(len(t) + sum(len(s[r]) for s in steps)) // 16) for text in texts for r, t in enumerate(text))
    assert both.used == used
    with pytest.raises(ValueError):
        Batch(both, 1, 1000).step([list(range(16 * (40 - used) + 1))])


def test_empty_prompts_and_single_tokens():
    """An empty prompt has no last token whose logits could be continued (they would be the request's
    before it); texts of one token have nothing to score."""
    from paper_2607_01127_amd.serve_example import Batch, Decoder, Shape
    print("empty prompts", flush=True)
    d = Decoder(Shape(layers=1), pages=16, page=16, seed=6)
    for prompts in ([[1, 2], []], [[], [1, 2]], [[]]):
        with pytest.raises(ValueError):
            Batch(d, len(prompts), 64).generate(prompts, 2)
    with pytest.raises(ValueError):
        Batch(d, 1, 64).generate([[1, 2]], 0)
    assert d.used == 0
    assert Batch(d, 2, 64).score([[3], [4]]).shape == (0,)
    whole, part = Batch(d, 2, 64).score([[3, 4], [5]]), Batch(d, 1, 64).score([[3, 4]])
    assert whole.shape == (1,) and float((whole - part).abs()) < 1e-3
