"""The 8-bit oracle (``oracle/fp8.py``) against torch's e4m3 and hand-worked
values."""

import numpy as np
import pytest
import torch

from oracle import fp8 as o8


def test_table_is_e4m3():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(o8.E4M3, t.astype(np.float64), equal_nan=True)


def test_rounding_is_torchs():
    rng = np.random.default_rng(1)
    v = np.concatenate([np.exp(rng.uniform(-8, 6, 20000)) * rng.choice([-1, 1], 20000),
                        (o8._POSITIVE[1:] + o8._POSITIVE[:-1]) / 2,        # every tie
                        -(o8._POSITIVE[1:] + o8._POSITIVE[:-1]) / 2, o8._POSITIVE]).astype(np.float32)
    v = v[np.abs(v) <= 448]
    want = torch.from_numpy(v).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(o8.round_e4m3(v), want.astype(np.float64))
    assert np.isnan(o8.round_e4m3(np.array([np.inf, -np.inf, np.nan]))).all()


@pytest.mark.parametrize("a,e", [(448.0, 0), (448.00001, 1), (0.0, 0), (1.0, -8), (1.75, -8),
                                 (1.7500001, -7), (2.0 ** -149, -127), (3.4e38, 120),
                                 (2.0 ** -118, -126), (1.75 * 2.0 ** -119, -127),
                                 (np.inf, 0), (np.nan, 0)])
def test_scales_by_hand(a, e):
    x = np.zeros((1, 5))
    x[0, 3] = -a
    assert o8.scale_exponents(x)[0, 0] == e
    x[0, 1] = 2.0 ** -140 if np.isfinite(a) else 0.0       # a smaller one changes nothing
    if a > 2.0 ** -140:
        assert o8.scale_exponents(x)[0, 0] == e


def test_quantize_and_back():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((5, 300)) * np.exp(3 * rng.standard_normal((1, 300)))
    v, e = o8.quantize(x)
    assert e.shape == (5, 3)
    back = o8.dequantize(v, e)
    step = np.maximum(np.abs(x) * 2.0 ** -4, 2.0 ** -10 * 2.0 ** o8.expand(e, 5, 300))
    assert np.all(np.abs(back - x) <= step)                 # half a step, or half the least number
    top = np.abs(v).reshape(5, -1)
    assert top.max() <= 448 and np.all([top[:, 128 * g:128 * g + 128].max(1) > 216 for g in range(3)])
    v2, e2 = o8.quantize(x, 128)
    assert e2.shape == (1, 3) and np.array_equal(e2[0], e.max(0))
    assert np.array_equal(o8.quantize(4 * x)[0], v)         # powers of two pass through


def test_norm_by_hand():
    y, h = o8.rmsnorm(np.array([[3.0, 0.0]]), np.array([[0.0, 4.0]]), np.array([1.0, 2.0]), 0.0)
    assert np.allclose(y, [[3 / 12.5 ** 0.5, 8 / 12.5 ** 0.5]]) and np.array_equal(h, [[3, 4]])
    y, _ = o8.rmsnorm(np.zeros((1, 4)), None, None, 1e-5)
    assert np.array_equal(y, np.zeros((1, 4)))
