"""The oracles of weights in 4-bit floats and of log probabilities against other
statements of the same things."""
import itertools
import math

import numpy as np
import pytest
import torch

from oracle import f4 as O
from oracle import logprobs as L


def test_code_values():
    """Sign, two exponent bits with bias 1, one mantissa bit, no infinity."""
    for c in range(16):
        e, m = c >> 1 & 3, c & 1
        v = m / 2 if e == 0 else (1 + m / 2) * 2.0 ** (e - 1)
        assert O.VALUES[c] == (-v if c & 8 else v)


def test_codes_that_overflow():
    """bfloat16 and float32: 4 and more under 2^126, 2 and more under 2^127; float16: from 65536."""
    codes = np.tile(np.arange(16, dtype=np.uint8), (255, 2))
    scales = np.full((1, 255, 4), 255, np.uint8)
    scales[0, :, 0] = np.arange(255)
    held = torch.from_numpy(O.values(codes, scales, 16))
    magnitude, e = torch.from_numpy(np.tile(O.MAGNITUDES, 2)), torch.arange(255)[:, None] - 127
    for dtype in (torch.float32, torch.bfloat16):
        assert torch.equal(held.to(dtype).isinf(), (magnitude >= 4) & (e == 126) |
                           (magnitude >= 2) & (e == 127))
    assert torch.equal(held.half().isinf(), held.abs() >= 65536)


def test_codes_are_the_nearest(rng):
    v = np.concatenate([rng.uniform(-7, 7, 2000), (O.MAGNITUDES[:-1] + O.MAGNITUDES[1:]) / 2,
                        O.MAGNITUDES, [-0.0, 6.9, -7.0]])
    got = O.nearest_code(v)
    for x, c in zip(v, got):
        best = min(range(8), key=lambda i: (abs(min(abs(x), 6) - O.MAGNITUDES[i]), i % 2))
        assert c & 7 == best and bool(c & 8) == (math.copysign(1, x) < 0)


@pytest.mark.parametrize("top,e", [(7.0, 0), (7.0000005, 1), (3.5, -1), (6.0, 0), (0.0, -98),
                                   (2.0 ** -96, -98), (2.0 ** 127, 125), (3.4e38, 126)])
def test_scale(top, e):
    assert O.scale_byte(top) == e + 127


def test_scale_of_no_number():
    assert O.scale_byte(np.inf) == O.scale_byte(np.nan) == 255


def test_quantizer_is_within_half_a_step(rng):
    x = (rng.standard_normal((7, 150)) * 10.0 ** rng.integers(-6, 6, (7, 1))).astype(np.float32)
    codes, scales = O.quantize(x)
    back = O.values(codes, scales, 150)
    e = scales.transpose(1, 0, 2).reshape(7, -1).astype(np.float64) - 127
    a = np.abs(x / np.repeat(2.0 ** e, 32, 1)[:, :150])
    half = np.where(a < 2, 0.25, np.where(a < 4, 0.5, 1.0))
    assert a.max() <= 7
    assert (np.abs(back - x) <= half * np.repeat(2.0 ** e, 32, 1)[:, :150]).all()
    assert not codes[:, 150:].any()
    assert np.array_equal(O.unpack(O.pack(codes)), codes)


def test_activations(rng):
    g = np.concatenate([rng.standard_normal(200) * 5, [0.0, 20.0, -20.0]])
    t = torch.from_numpy(g)
    for kind, want in ((1, torch.nn.functional.silu(t)), (2, torch.nn.functional.gelu(t)),
                       (3, torch.nn.functional.gelu(t, approximate="tanh"))):
        assert np.allclose(O.activate(g, kind), want.numpy(), rtol=1e-9, atol=1e-14)


def test_logprobs(rng):
    x = rng.standard_normal((6, 50)) * 3
    x[1, 5:20] = -np.inf
    x[2, 7] = x[2, 30] = x[2].max() + 1            # a tie goes to the lower index
    x[3] = -np.inf
    x[4, 4] = np.nan
    tokens = [3, 0, 30, 1, 2, -1]
    (lp, h, best, at), _ = L.logprobs(x, tokens, 7, 0.5)
    for r in (0, 1, 2, 5):
        dist = torch.distributions.Categorical(logits=torch.from_numpy(0.5 * x[r]))
        p = dist.probs.numpy()
        assert np.isclose(h[r], -(p[p > 0] * np.log(p[p > 0])).sum())
        want = sorted(itertools.islice(range(50), 50), key=lambda i: (-x[r, i], i))[:7]
        assert list(at[r]) == want
        assert np.allclose(best[r], np.log(p[want]))
        if tokens[r] >= 0:
            assert np.isclose(lp[r], np.log(p[tokens[r]]))
    assert lp[5] == 0 and at[2, 0] == 7 and at[2, 1] == 30
    assert lp[3] == -np.inf and h[3] == 0 and list(at[3]) == list(range(7))
    assert np.isnan(lp[4]) and np.isnan(h[4]) and (at[4] == -1).all()
