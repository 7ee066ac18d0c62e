"""Which kernel the serving operators take, on the CPU: the GPU cases name every
instance that is compiled, and each case goes to the one that it names."""
import os
import re

import pytest

import paper_1911_08076_amd as P
from test_gpu_serve_instances import ATTENTIONS, PRODUCTS, attention_desc

CSRC = os.path.join(os.path.dirname(P.__file__), "csrc")


def named(source, stem):
    with open(os.path.join(CSRC, source)) as f:
        return set(re.findall(r'"(%s[a-z]+<[\d, ]+>)"' % stem, f.read()))


def test_every_instance_of_the_product_has_cases():
    names = named("ifq_f8.hip", "f8_matmul_")
    assert len(names) == 9 and {c[3] for c in PRODUCTS} == names
    for m, n, k, kernel, parts in PRODUCTS:
        d = P.f8_matmul_desc(m, n, k, P.IFQ_TYPE_BF16)
        assert P.ifq_f8_matmul_kernel_name(d) == kernel, (m, n, k)
        assert (P.ifq_f8_matmul_workspace_bytes(d) > 0) == parts, (m, n, k)
    assert any(c[4] for c in PRODUCTS)


def test_every_instance_of_the_attention_has_cases():
    names = named("ifq_attn.hip", "kv_attention_")
    assert len(names) == 11 and {c[4] for c in ATTENTIONS} == names
    for new, heads, kv_heads, dim, kernel in ATTENTIONS:
        for hint in (0, 1500):
            d = attention_desc(new, heads, kv_heads, dim, hint)
            assert P.ifq_kv_attention_kernel_name(d) == kernel, (new, heads, dim)
            assert (P.ifq_kv_attention_workspace_bytes(d) > 0) == (hint > 0), (new, heads, dim)


@pytest.mark.parametrize("m,n,k,kernel", [
    # the performance cases
    (1, 4096, 4096, "f8_matmul_few<1, 8>"), (37, 1000, 4096, "f8_matmul_few<1, 8>"),
    (515, 6144, 4096, "f8_matmul_tiled<2, 2, 2, 2, 2>"),
    (8192, 14336, 4096, "f8_matmul_tiled<2, 2, 2, 2, 1>")])
def test_product(m, n, k, kernel):
    assert P.ifq_f8_matmul_kernel_name(P.f8_matmul_desc(m, n, k, P.IFQ_TYPE_BF16)) == kernel


def test_no_kernel_for_nothing():
    assert P.ifq_f8_matmul_kernel_name(P.f8_matmul_desc(0, 64, 128, P.IFQ_TYPE_F32)) == ""
    assert P.ifq_f8_matmul_kernel_name(P.f8_matmul_desc(1, 64, 100, P.IFQ_TYPE_F32)) == ""
    assert P.ifq_kv_attention_kernel_name(attention_desc([0], 2, 1, 64, 0)) == ""
    assert P.ifq_kv_attention_kernel_name(attention_desc([1], 2, 1, 96, 0)) == ""
