"""The block-scaled product where the product of two scales leaves fp32's range and the
result does not, in each of its kernels."""
import numpy as np
import pytest
import torch

import paper_1911_08076_amd as P
from oracle import serve as S
from test_gpu_f8 import DEV, dev, operands
from test_gpu_serve_instances import PRODUCTS

pytestmark = pytest.mark.gpu
SHAPES = [c[:3] for c in PRODUCTS if c[0] < 4000]


def product(a, sa, w, sw):
    (m, k), n = a.shape, len(w)
    y = torch.empty(m, n, device=DEV)
    P.ifq_f8_matmul(P.f8_matmul_desc(m, n, k, P.IFQ_TYPE_F32), *dev(a, sa, w, sw), y)
    return y.double().cpu().numpy()


def close(got, want, size, kb):
    # sums in fp32, as in test_gpu_f8, and a unit of the smallest number for each block
    return np.abs(got - want) <= ((128 + kb + 4) * 2.0 ** -23 * size + 2.0 ** -23 * np.abs(want) +
                                  (kb + 2) * 2.0 ** -149)


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("ea,ew", [(-75, -68), (-60, -88), (-104, -40)])
def test_small_scales(m, n, k, ea, ew, rng):
    """2^-143 to 2^-148: the sums of the codes' products, up to 2^24, bring the result
    back into the range."""
    a, sa, w, sw = operands(rng, m, n, k)
    sa, sw = sa * np.float32(2.0 ** ea), sw * np.float32(2.0 ** ew)
    want, size = S.f8_matmul(a, sa, w, sw)
    assert np.abs(want).max() > 2.0 ** -126
    assert close(product(a, sa, w, sw), want, size, len(sa)).all()


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_large_scales(m, n, k, rng):
    """Around 2^129, with the smallest codes: the sums of their products are below 2^-10."""
    a, sa, w, sw = operands(rng, m, n, k)
    a, w = (c & 0x81 for c in (a, w))                        # 0 and 2^-9
    w[:, ::2] = 0
    sa, sw = sa * np.float32(2.0 ** 100), sw * np.float32(2.0 ** 29)
    want, size = S.f8_matmul(a, sa, w, sw)
    assert size.max() < 2.0 ** 127
    assert close(product(a, sa, w, sw), want, size, len(sa)).all()


def test_zeros_under_large_scales(rng):
    """Rows that share no column: 0, not infinity times 0."""
    for m, n, k in SHAPES:
        a, sa, w, sw = operands(rng, m, n, k)
        a[:, ::2] = 0
        w[:, 1::2] = 0
        sa[:], sw[:] = 2.0 ** 100, 2.0 ** 60
        assert not product(a, sa, w, sw).any(), (m, n, k)
