"""Every instance of the product's and the attention's kernels, by name, against the
oracle: shapes that end inside a tile and go round each loop more than once, NaN scales
in each kernel, and sequences whole and in parts."""
import numpy as np
import pytest
import torch

import paper_1911_08076_amd as P
from oracle import serve as S
from test_gpu_attention import Case
from test_gpu_f8 import DEV, TYPES, dev, operands

pytestmark = pytest.mark.gpu

# m, n, k, kernel, whether k is in parts
PRODUCTS = [
    (8, 9000, 4112, "f8_matmul_few<1, 4>", False),
    (16, 4001, 4144, "f8_matmul_few<1, 8>", False),
    (13, 1000, 12304, "f8_matmul_few<1, 16>", False),
    (32, 14001, 2064, "f8_matmul_few<2, 4>", False),
    (50, 2002, 4112, "f8_matmul_few<2, 8>", False),
    (32, 2000, 4112, "f8_matmul_few<2, 16>", False),
    (67, 14331, 1040, "f8_matmul_tiled<1, 1, 2, 2, 1>", False),
    (200, 2001, 2064, "f8_matmul_tiled<1, 1, 2, 2, 1>", True),
    (515, 4002, 784, "f8_matmul_tiled<2, 2, 2, 2, 1>", False),
    (4090, 2100, 2064, "f8_matmul_tiled<2, 2, 2, 2, 1>", False),   # more tiles than CUs
    (515, 4002, 2064, "f8_matmul_tiled<2, 2, 2, 2, 2>", False),    # an odd number of blocks
    (530, 4003, 1936, "f8_matmul_tiled<2, 2, 2, 2, 2>", False)]


@pytest.mark.parametrize("m,n,k,kernel,parts", PRODUCTS)
def test_product(m, n, k, kernel, parts, rng):
    a, sa, w, sw = operands(rng, m, n, k)
    want, size = S.f8_matmul(a, sa, w, sw)
    on = dev(a, sa, w, sw)
    for kind, (dtype, code, u) in TYPES.items():
        y = torch.full((m, n), -3.0, dtype=dtype, device=DEV)
        P.ifq_f8_matmul(P.f8_matmul_desc(m, n, k, code), *on, y)
        got = y.double().cpu().numpy()
        # as in test_gpu_f8: sums in fp32, and the rounding of the output
        bound = (128 + len(sa) + 4) * 2.0 ** -23 * size + u * np.abs(want)
        fits = np.abs(want) <= 65000 if kind == "f16" else np.ones_like(want, bool)
        bound += 2.0 ** -25 if kind == "f16" else 0.0
        assert (np.abs(got - want) <= bound)[fits].all(), kind


@pytest.mark.parametrize("m,n,k,kernel,parts", PRODUCTS)
def test_product_scales_that_are_nan(m, n, k, kernel, parts, rng):
    """They reach their rows and their columns of 128, and no others."""
    a, sa, w, sw = operands(rng, m, n, k)
    sa[len(sa) - 1, m // 2] = np.nan
    sw[len(sw) // 2, sw.shape[1] - 1] = np.nan
    y = torch.empty(m, n, device=DEV)
    P.ifq_f8_matmul(P.f8_matmul_desc(m, n, k, P.IFQ_TYPE_F32), *dev(a, sa, w, sw), y)
    want = np.zeros((m, n), bool)
    want[m // 2] = True
    want[:, 128 * (sw.shape[1] - 1):] = True
    assert np.array_equal(torch.isnan(y).cpu().numpy(), want)


# new tokens, heads, kv heads, dim, kernel
ATTENTIONS = [(new, heads, kv_heads, dim, kernel % dim)
              for dim in (64, 128, 256)
              for new, heads, kv_heads, kernel in (
                  ([1, 1, 0], 8, 2, "kv_attention_few<%%d, %d>" % (2 if dim == 256 else 4)),
                  ([2, 1, 3], 2, 1, "kv_attention_few<%d, 2>"),
                  ([1, 1, 1], 24, 2, "kv_attention_few<%d, 1>"),
                  ([16, 5, 9], 2, 2, "kv_attention_few<%d, 1>"),
                  ([1, 1, 1], 17, 1, "kv_attention_many<%d>"),
                  ([70, 3, 129], 2, 1, "kv_attention_many<%d>"))]


def attention_desc(new, heads, kv_heads, dim, hint, lens=(700, 333, 41)):
    return P.kv_desc(len(new), sum(new), max(new), hint, heads, kv_heads, dim, 64, 40,
                     -(-max(lens) // 64), P.IFQ_TYPE_BF16)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("hint", [0, 1500])           # whole, and in parts
@pytest.mark.parametrize("new,heads,kv_heads,dim,kernel", ATTENTIONS)
def test_attention(new, heads, kv_heads, dim, kernel, hint, kind, rng):
    Case(rng, new, [700, 333, 41], heads, kv_heads, dim, 64, kind, max_kv=hint).check()
