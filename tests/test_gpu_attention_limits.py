"""Attention at the ends of its arguments' ranges: sequences longer than their page
table. Against the oracle, as in
test_gpu_attention."""
import pytest

from test_gpu_attention import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [[1, 1], [3, 2], [60, 9], [300, 200]])
@pytest.mark.parametrize("window,sinks", [(0, 0), (16, 0), (16, 4), (40, 33), (70, 64), (500, 3),
                                          (16, 1000)])
@pytest.mark.parametrize("past", [1, 36, 90, 5000])
def test_sequences_longer_than_their_table(new, window, sinks, past, rng):
    """Positions past the table are not there; the window stays at the query's own."""
    c = Case(rng, new, [512, 512], 4, 2, 64, 32, "f16", window=window, sinks=sinks)
    c.lens = [512 + past, 512 + past // 2]
    c.check()
