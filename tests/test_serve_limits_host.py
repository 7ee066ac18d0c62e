"""Host side of the serving operators at the ends of their arguments' ranges, on the CPU."""
import pytest

import paper_1911_08076_amd as P

INT_MAX = 2 ** 31 - 1


def workspace(window, sinks, max_q=1):
    d = P.kv_desc(4, 4 * max_q, max_q, 5000, 8, 2, 128, 64, 400, 100, P.IFQ_TYPE_BF16,
                  window=window, sinks=sinks)
    return P.ifq_kv_attention_workspace_bytes(d)


@pytest.mark.parametrize("max_q", [1, 200])
def test_workspace_with_the_largest_windows_and_sinks(max_q):
    """More sinks than the sequence has tokens are as good as all of it."""
    whole = workspace(0, 0, max_q)
    assert whole > 0
    for window, sinks in ((100, 2 ** 31 - 32), (100, 2 ** 31 - 31), (100, INT_MAX),
                          (INT_MAX, 0), (INT_MAX, INT_MAX), (INT_MAX - 31, 5)):
        assert workspace(window, sinks, max_q) == whole, (window, sinks)


@pytest.mark.parametrize("value", [1, -1, INT_MAX])
def test_product_refuses_what_is_reserved(value):
    d = P.f8_matmul_desc(64, 256, 4096, P.IFQ_TYPE_BF16)
    d.reserved = value
    with pytest.raises(P.IfqError) as e:
        P.ifq_f8_matmul(d, None, None, None, None, None, stream=0)
    assert e.value.status == -1 and "reserved" in str(e.value)
    assert P.ifq_f8_matmul_workspace_bytes(d) == 0
