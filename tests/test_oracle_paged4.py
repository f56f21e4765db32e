"""Pins of the 4-bit rows and the rotation in the float64 oracle (oracle/paged.py)."""
import numpy as np
import pytest

from oracle import paged


def test_bf16():
    x = np.float32([1.0, 1.00390625, 1.01171875, 1.0000001, 3.0, 0.0, -1.00390625, -2.5])
    assert np.array_equal(paged.to_bf16(x), np.float32([1.0, 1.0, 1.015625, 1.0, 3.0, 0.0, -1.0, -2.5]))
    up = paged.to_bf16(np.float32([1.0, 1.0000001, 1.0078125, 0.0]), up=True)
    assert np.array_equal(up, np.float32([1.0, 1.0078125, 1.0078125, 0.0]))


@pytest.mark.parametrize("scale", [1.0, 2.0 ** -90, 2.0 ** 95, 2.0 ** 130])
def test_a_value_is_half_a_step_off_at_most(scale):
    rng = np.random.default_rng(0)
    with np.errstate(over="ignore"):
        x = ((rng.standard_normal((200, 64)) + rng.standard_normal((200, 1)) * 3) * scale).astype(np.float32)
    c, step, mid = paged.rows4(x)
    assert c.max() <= 15 and (step >= 2.0 ** -100).all() and (step <= 2.0 ** 100).all()
    assert (step >= np.abs(mid) * 2.0 ** -16).all()
    y = paged.values4(paged.pack4(c), np.stack([step, mid], -1))
    x = np.clip(x.astype(np.float64), -2.0 ** 102, 2.0 ** 102)
    # x - middle, the product with the rounded reciprocal, the sum with 7.5: each half a step of float32
    off = np.abs(y - x)
    slack = 2.0 ** -24 * (np.abs(x - mid[:, None]) + 3 * 15 * step[:, None])
    assert (off <= 0.5 * step[:, None] + slack).all()


def test_rows_without_a_range():
    x = np.zeros((4, 64), np.float32)
    x[1] = 1.0
    x[2] = -1000.25
    x[3, 5] = np.nan
    c, step, mid = paged.rows4(x)
    assert step[0] == 2.0 ** -100 and mid[0] == 0 and step[3] == 2.0 ** -100
    assert mid[1] == 1 and step[1] == 2.0 ** -16
    assert mid[2] == -1000 and step[2] >= 0.25 / 7.5
    y = paged.values4(paged.pack4(c), np.stack([step, mid], -1))
    assert np.abs(y - np.nan_to_num(x)).max(1)[2] <= step[2] / 2


def test_turning_keeps_lengths_and_relative_angles():
    rng = np.random.default_rng(1)
    half = 16
    angle = np.arange(50)[:, None] * 10000.0 ** (-np.arange(half) / half)
    cos, sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
    for pairs in (False, True):
        x, y = rng.standard_normal((2, 1, 1, 64)).astype(np.float32)
        at = lambda v, p: paged.turn(v, [p], cos, sin, 32, pairs).astype(np.float64)
        assert np.array_equal(at(x, 7)[..., 32:], x[..., 32:])
        assert abs(np.linalg.norm(at(x, 7)) / np.linalg.norm(x) - 1) < 1e-6
        # the product goes by the distance alone
        a, b = (at(x, 30) * at(y, 27)).sum(), (at(x, 10) * at(y, 7)).sum()
        assert abs(a - b) < 1e-4
        # against the complex product
        i = np.arange(16)
        i, j = (2 * i, 2 * i + 1) if pairs else (i, i + 16)
        z = (x[0, 0, i] + 1j * x[0, 0, j]) * np.exp(1j * angle[9])
        t = at(x, 9)[0, 0]
        assert np.abs(t[i] - z.real).max() < 1e-6 and np.abs(t[j] - z.imag).max() < 1e-6


def test_write4_packs_two_a_byte():
    rng = np.random.default_rng(2)
    codes, numbers = np.zeros((2, 1, 16, 32), np.uint8), np.zeros((2, 1, 16, 2), np.float32)
    x = rng.standard_normal((3, 1, 64)).astype(np.float32)
    paged.write4(codes, numbers, x, [17, -1, 40])
    c, step, mid = paged.rows4(x)
    assert np.array_equal(codes[1, 0, 1] & 15, c[0, 0, ::2]) and np.array_equal(codes[1, 0, 1] >> 4, c[0, 0, 1::2])
    assert np.array_equal(numbers[1, 0, 1], [step[0, 0], mid[0, 0]])
    assert not codes[0].any() and not codes[1, 0, 0].any() and not codes[1, 0, 2:].any()
