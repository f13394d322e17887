"""Block tables whose outputs overlap what the call reads are refused (no GPU: a call that got as far as
a launch would report a HIP error)."""
import pytest

from paper_2607_01127_amd import logbq as L

SIZES = dict(cached=12, new=12, free=20, table=48, slots=56, positions=28, starts=16, lens=12, info=16)
INPUTS, OUTPUTS = ("cached", "new", "free"), ("table", "slots", "positions", "starts", "lens", "info")


def call(at):
    return L.lib().logbq_batch_tables(at["cached"], at["new"], 3, at["free"], 5, at["table"], 4, 16, 7,
                                      at["slots"], at["positions"], at["starts"], at["lens"], at["info"], None)


@pytest.mark.parametrize("read", INPUTS)
@pytest.mark.parametrize("written", OUTPUTS)
def test_outputs_over_inputs_are_refused(read, written):
    apart = {name: 4096 * (i + 1) for i, name in enumerate(SIZES)}
    for by in (0, SIZES[read] - 4, 4 - SIZES[written]):              # the same place, and by one element
        assert call(dict(apart, **{written: apart[read] + by})) == L.ERR_INVALID_ARG

