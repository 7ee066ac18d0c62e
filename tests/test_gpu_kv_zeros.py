"""Rows of zeros of both signs in the cache of 4-bit codes: -0 counts below 0 wherever
it stands, so that the offset's bits do not go by the order of a row's lanes."""
import numpy as np
import pytest
import torch

from test_gpu_kv import DEV, Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rot,adjacent", [(0, False), (64, False), (32, True)])
def test_zeros_of_both_signs(kind, dim, rot, adjacent, rng):
    b = Batch(rng, [9, 40], [9, 77], 2, 2, dim, 32, kind, rot, adjacent)
    x = b.rows
    x[:] = 0.0
    sign = torch.from_numpy(rng.random(x.shape) < 0.03).to(DEV)
    x[sign] = -0.0
    x[::5, :, 7] = 2.5                          # and above them, a value
    x[1::5] = 0.0
    x[2::5] = -0.0
    b.check()
    assert {0x0000, 0x8000} <= {int(w) & 0xFFFF for w in words(b)}


def words(b):
    """Offsets and steps of all rows in the expected cache."""
    cache = b.expected()[0]
    return np.unique(cache[:, :, b.page * b.dim:].copy().view(np.uint32))
