"""Which kernel the products with weights in 4-bit floats take, on the CPU: the GPU
cases name every instance that is compiled, and each case goes to the one that it names."""
import os
import re

import pytest

import paper_1911_08076_amd as P
from test_gpu_f4_instances import GATED, PRODUCTS

SOURCE = os.path.join(os.path.dirname(P.__file__), "csrc", "ifq_f4.hip")


def name_of(m, n, k, activation=P.IFQ_ACT_NONE):
    d = P.f4_matmul_desc(m, n, k, P.IFQ_TYPE_BF16, activation=activation)
    return (P.ifq_f4_gated_kernel_name if activation else P.ifq_f4_matmul_kernel_name)(d)


def test_every_instance_has_cases():
    with open(SOURCE) as f:
        text = f.read()
    rows = re.findall(r"\bF\((\d+), (\d+), (\d+), (\d+), (\d+)\)", text)
    names = {"f4_matmul_few<%s>" % ", ".join(r) for r in rows}
    names |= set(re.findall(r'"(f4_matmul_tiled<[\d, ]+>)"', text))
    assert len(names) == 39
    for whole in (True, False):
        assert {c[3] for c in PRODUCTS + GATED if (c[2] % 8 == 0) == whole} == names
    for m, n, k, kernel in PRODUCTS:
        assert name_of(m, n, k) == kernel, (m, n, k)
    for m, n, k, kernel in GATED:
        assert name_of(m, n, k, P.IFQ_ACT_SILU) == kernel, (m, n, k)


@pytest.mark.parametrize("m,n,k,activation,kernel", [
    # the performance cases
    (1, 4096, 14336, 0, "f4_matmul_few<4, 1, 1, 4, 1>"),
    (24, 6144, 4096, 0, "f4_matmul_few<32, 2, 1, 2, 1>"),
    (7, 128000, 4096, 0, "f4_matmul_few<8, 2, 2, 4, 1>"),
    (2011, 4096, 14336, 0, "f4_matmul_tiled<4, 2, 4, 2, 1>"),
    (1, 14336, 4096, 1, "f4_matmul_few<4, 2, 1, 4, 2>"),
    (41, 9001, 4008, 1, "f4_matmul_few<48, 2, 3, 3, 2>"),
    (3001, 14336, 4096, 1, "f4_matmul_tiled<4, 2, 4, 1, 2>")])
def test_kernel(m, n, k, activation, kernel):
    assert name_of(m, n, k, activation) == kernel


def test_no_kernel_for_nothing():
    assert name_of(0, 64, 128) == name_of(3, 0, 128) == name_of(3, 64, 0) == ""
