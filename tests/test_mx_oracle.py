"""Pins of the 4-bit oracle: the format by enumeration, and against the 8-bit scale type that torch has."""
import math

import numpy as np
import pytest
import torch

from oracle import mx


def block(*head, fill=0.0):
    x = np.full(32, fill)
    x[:len(head)] = head
    return x


def test_every_code_and_scale():
    want = [0, .5, 1, 1.5, 2, 3, 4, 6]
    codes = np.arange(16, dtype=np.uint8) * 17  # both halves of a byte
    for byte in range(255):
        got = mx.dequantize(codes[None], np.array([[byte]], dtype=np.uint8))[0]
        ref = [(-1 if c & 8 else 1) * math.ldexp(want[c & 7], byte - 127) for c in range(16) for _ in (0, 1)]
        assert got.tolist() == ref
    assert np.isnan(mx.dequantize(codes[None], np.array([[255]], dtype=np.uint8))).all()


def test_scales_are_torchs_e8m0():
    bytes_ = torch.arange(256, dtype=torch.uint8)
    ref = bytes_.view(torch.float8_e8m0fnu).float().double().numpy()
    codes = np.full((256, 16), 2, dtype=np.uint8)  # 1.0, 0.0
    got = mx.dequantize(codes, bytes_.numpy()[:, None])[:, 0]
    assert np.array_equal(got, ref, equal_nan=True)


def test_order_of_the_halves():
    codes, scales = mx.quantize(block(1.0, -6.0, 0.5)[None])
    assert codes[0, 0] == (2 | 15 << 4) and codes[0, 1] == 1 and scales[0, 0] == 127


def test_halves_go_to_the_even_code_and_the_largest_saturates():
    x = block(4.0, .25, .75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.9, -.25, -.75, 6.5)
    got = mx.dequantize(*mx.quantize(x[None]))[0]
    assert got[:12].tolist() == [4, 0, 1, 1, 2, 2, 4, 4, 6, 0, -1, 6]
    eps = 1e-12
    near = block(4.0, .25 + eps, .75 - eps, 1.25 + eps, 1.75 - eps, 2.5 + eps, 3.5 - eps, 5 + eps)
    assert mx.dequantize(*mx.quantize(near[None]))[0][:8].tolist() == [4, .5, .5, 1.5, 1.5, 3, 3, 6]


@pytest.mark.parametrize("top,byte", [(4.0, 127), (7.999, 127), (8.0, 128), (3.999, 126), (2.0 ** -126, 0), (2.0 ** -125, 0), (2.0 ** -124, 1),
                                      (2.0 ** -140, 0), (0.0, 0), (3.4e38, 252)])
def test_scale_byte(top, byte):
    assert mx.quantize(block(top, -top / 3)[None])[1][0, 0] == byte


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_block_with_an_infinity_or_nan_is_nan_alone(bad):
    x = np.ones((1, 64))
    x[0, 40] = bad
    codes, scales = mx.quantize(x)
    assert scales.tolist() == [[125, 255]] and not codes[0, 16:].any()
    got = mx.dequantize(codes, scales)[0]
    assert (got[:32] == 1).all() and np.isnan(got[32:]).all()


def test_values_that_codes_stand_for_stay():
    rng = np.random.default_rng(1)
    codes = rng.integers(0, 256, (50, 48), dtype=np.uint8)
    scales = rng.integers(3, 252, (50, 3), dtype=np.uint8)
    codes[:, ::16] |= 7  # the largest of a block is 6 (or -6)
    x = mx.dequantize(codes, scales)
    again = mx.quantize(x)
    assert np.array_equal(again[0], codes) and np.array_equal(again[1], scales)


def test_error_is_half_a_step_of_the_codes():
    x = np.random.default_rng(2).standard_normal((200, 128)) * np.exp(np.random.default_rng(3).standard_normal((200, 1)) * 5)
    got = mx.dequantize(*mx.quantize(x))
    unit = np.repeat(np.ldexp(1.0, mx.quantize(x)[1].astype(int) - 127), 32, axis=-1)
    y, err = np.abs(x) / unit, np.abs(got - x) / unit
    step = np.where(y < 2, .5, np.where(y < 4, 1.0, 2.0))
    assert (err <= np.where(y > 6, y - 6, step / 2)).all()
