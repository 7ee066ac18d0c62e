"""Attention at the ends of its arguments' ranges: sequences longer than their page
table, windows and sinks up to the largest int32, values up to the largest that are
said to stay finite. Against the oracle, as in test_gpu_attention."""
import numpy as np
import pytest

from test_gpu_attention import Case

pytestmark = pytest.mark.gpu
INT_MAX = 2 ** 31 - 1


@pytest.mark.parametrize("new", [[1, 1], [3, 2], [60, 9], [300, 200]])
@pytest.mark.parametrize("window,sinks", [(0, 0), (16, 0), (16, 4), (40, 33), (70, 64), (500, 3),
                                          (16, 1000)])
@pytest.mark.parametrize("past", [1, 36, 90, 5000])
def test_sequences_longer_than_their_table(new, window, sinks, past, rng):
    """Positions past the table are not there; the window stays at the query's own."""
    c = Case(rng, new, [512, 512], 4, 2, 64, 32, "f16", window=window, sinks=sinks)
    c.lens = [512 + past, 512 + past // 2]
    c.check()


@pytest.mark.parametrize("new,lens", [([1, 1], [300, 40]), ([6], [3]), ([40, 7], [20, 5]),
                                      ([300], [200]), ([300, 9], [310, 90])])
@pytest.mark.parametrize("window,sinks", [
    (INT_MAX, 0), (INT_MAX, INT_MAX), (INT_MAX - 1, 4), (INT_MAX - 40, 0), (7, INT_MAX),
    (7, INT_MAX - 30), (7, INT_MAX - 31), (33, INT_MAX - 1)])
def test_largest_windows_and_sinks(new, lens, window, sinks, rng):
    """Sequences shorter than what asks among them: their first queries' positions are
    negative, and see nothing."""
    Case(rng, new, lens, 4, 2, 64, 32, "bf16", window=window, sinks=sinks).check()


@pytest.mark.parametrize("exponent", [90, -60])
@pytest.mark.parametrize("new,heads,dim", [([1, 1], 4, 64), ([2, 1], 8, 128), ([1, 3], 12, 256),
                                           ([70, 9], 4, 128)])
@pytest.mark.parametrize("max_kv", [0, 2000])
def test_values_of_large_and_small_size(new, heads, dim, exponent, max_kv, rng):
    """Offsets and steps times a power of two; the bound grows with them."""
    c = Case(rng, new, [600, 90], heads, 2, dim, 32, "bf16", max_kv=max_kv)
    for b, of in enumerate(c.rows):
        for g, (kw, kc, vw, vc) in enumerate(of):
            held = vw.astype(np.int64)
            for at in (7, 23):                 # the exponents of the offset and of the step
                there = (held >> at & 255) > 0
                held += np.where(there, exponent << at, 0)
            of[g] = (kw, kc, held.astype(np.uint32), vc)
            for i, page in enumerate(c.table[b][:-(-len(kw) // 32)]):
                c._fill(page, g, 32 * i, *of[g])
    c.check()
