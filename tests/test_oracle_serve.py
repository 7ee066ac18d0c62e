"""The oracle of the serving operators against other statements of the same
things: 8-bit floats as PyTorch reads them, pages put together code by code,
rotation by complex numbers, attention by explicit loops."""
import numpy as np
import pytest
import torch

from oracle import serve as S


def test_e4m3_values_and_rounding(rng):
    codes = np.arange(256, dtype=np.uint8)
    t = torch.from_numpy(codes).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(S.E4M3, t.astype(np.float64), equal_nan=True)
    x = np.concatenate([rng.standard_normal(4000) * 10.0 ** rng.integers(-4, 3, 4000),
                        (S.E4M3[:126] + S.E4M3[1:127]) / 2, S.E4M3[:127], [0.0, -0.0]])
    x = np.clip(x, -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(S.e4m3_codes(x), want)


def test_quantizer_keeps_the_largest_value_exact(rng):
    x = rng.standard_normal((5, 300)).astype(np.float32)
    codes, scales = S.f8_quantize(x)
    back = S.E4M3[codes] * scales.T[:, np.arange(300) // 128]
    assert np.abs(S.E4M3[codes]).max() == 448
    # half a step of 3 mantissa bits, or half the smallest step of the scale
    step = np.maximum(np.abs(x) * 2.0 ** -4, scales.T[:, np.arange(300) // 128] * 2.0 ** -10)
    assert (np.abs(back - x) <= step * 1.0001).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_page_round_trip(dim, rng):
    tokens = 64
    held = rng.integers(0, 256, tokens * (dim + 8), dtype=np.uint8)
    page = S.Page(held, tokens, dim)
    k = rng.integers(0, 16, (tokens, dim), dtype=np.uint8)
    v = rng.integers(0, 16, (tokens, dim), dtype=np.uint8)
    for t in rng.permutation(tokens):
        page.put(t, t, k[t], 7 * t, v[t])
    gk, gv = page.codes()
    assert np.array_equal(gk, k) and np.array_equal(gv, v)
    assert np.array_equal(page.kw, np.arange(tokens)) and page.vw[3] == 21


def test_row_codes_cover_the_row(rng):
    x = (rng.standard_normal((200, 128)) * np.exp(3 * rng.standard_normal((200, 1)))).astype(
        np.float32)
    word, code = S.row_codes(x)
    step = S._f32_of(word & np.uint32(0xFFFF0000))
    assert (np.abs(S.row_values(word, code) - x) <= step[:, None] * 0.50001).all()
    assert (code.min(1) == 0).all() and (code.max(1) == 15).mean() > 0.5
    x[3, 5], x[4, 7], x[5] = np.nan, np.inf, 2.5
    word, code = S.row_codes(x)
    got = S.row_values(word, code)
    assert np.isnan(got[3]).all() and np.isnan(got[4]).all() and (got[5] == 2.5).all()


@pytest.mark.parametrize("adjacent", [False, True])
def test_rotation_is_a_complex_product(adjacent, rng):
    x = rng.standard_normal((3, 64)).astype(np.float32)
    ang = rng.uniform(0, 7, (3, 16))
    got = S.rotate(x, np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32), adjacent)
    z = x[:, 0:32:2] + 1j * x[:, 1:32:2] if adjacent else x[:, :16] + 1j * x[:, 16:32]
    z = z * np.exp(1j * ang)
    back = got[:, 0:32:2] + 1j * got[:, 1:32:2] if adjacent else got[:, :16] + 1j * got[:, 16:32]
    assert np.abs(back - z).max() < 1e-6 and np.array_equal(got[:, 32:], x[:, 32:])


def test_attention_by_loops(rng):
    dim, n = 64, 40
    kw, kc = S.row_codes(rng.standard_normal((n, dim)))
    vw, vc = S.row_codes(rng.standard_normal((n, dim)))
    q = rng.standard_normal((2, dim)).astype(np.float32)
    out, bound = S.attention(q, kw, kc, vw, vc, np.array([20, -1]), 0.125, window=5, sinks=2)
    k, v = (S._f32_of(w << np.uint32(16)).astype(float)[:, None] +
            S._f32_of(w & np.uint32(0xFFFF0000)).astype(float)[:, None] * c
            for w, c in ((kw, kc), (vw, vc)))
    seen = [0, 1] + [16, 17, 18, 19, 20]
    p = np.array([np.exp(0.125 * sum(float(a) * float(b) for a, b in zip(q[0], k[j])))
                  for j in seen])
    want = sum(p[i] * v[j] for i, j in enumerate(seen)) / p.sum()
    assert np.abs(out[0] - want).max() < 1e-12 and not out[1].any()
    assert 0 < bound[0].max() < 2.0 ** -8      # it tells more than the rounding to bfloat16
