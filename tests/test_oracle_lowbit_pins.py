"""Pins of the low-bit oracle (no GPU): the formats' values by hand, the
rounding at every tie, the norm's gradient against differences, and the
attention's union of two key sets against one softmax over both."""

import numpy as np
import pytest

from oracle import lowbit


def test_e2m1_values():
    assert lowbit.e2m1_value(np.arange(8)).tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    assert lowbit.e2m1_value(np.arange(8, 16)).tolist() == [0, -0.5, -1, -1.5, -2, -3, -4, -6]


def test_e4m3_values():
    assert lowbit.e4m3_value(np.array([0x00, 0x01, 0x08, 0x38, 0x7e, 0xb8])).tolist() == [0, 2.0 ** -9, 2.0 ** -6, 1, 448, -1]
    assert np.isnan(lowbit.e4m3_value(0x7f))


def test_mx_rounding_ties_and_saturation():
    # a maximum in [4, 8) has scale 1: byte 127
    x = np.zeros((1, 32))
    x[0, :14] = [4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7.9, -0.25, -0.76, 0.26, 5.01, -7]
    code, byte = lowbit.mx_codes(x)
    assert byte[0, 0] == 127
    assert lowbit.e2m1_value(code[0, :14]).tolist() == [4, 0, 1, 1, 2, 2, 4, 4, 6, 0, -1, 0.5, 6, -6]


@pytest.mark.parametrize("top,byte", [(1.0, 125), (1.999, 125), (2.0, 126), (6.0, 127), (8.0, 128), (2.0 ** -126, 0),
                                      (2.0 ** -125, 0), (2.0 ** -124, 1), (2.0 ** -149, 0), (0.0, 0), (2.0 ** 127, 252),
                                      (np.inf, 255), (np.nan, 255)])
def test_mx_scale_bytes(top, byte):
    x = np.zeros((1, 40))
    x[0, 33] = top
    assert lowbit.mx_scale_byte(x).tolist() == [[0, byte]]


def test_mx_round_trip_of_representable_values():
    rng = np.random.default_rng(0)
    x = rng.choice(lowbit.e2m1_value(np.arange(16)), (5, 64)) * 2.0 ** rng.integers(-20, 20, (5, 1))
    x[:, ::32] = 6 * 2.0 ** np.floor(np.log2(np.abs(x).max(1, keepdims=True) / 4))  # the block's largest
    code, byte = lowbit.mx_codes(x)
    # every value lies on the grid of its block's scale, or below its step
    y = lowbit.mx_values(lowbit.mx_pack(code), byte)
    step = 2.0 ** (byte - 127.0).repeat(32, 1) / 2
    assert (np.abs(y - x) <= step).all()


@pytest.mark.parametrize("with_sum", [False, True])
def test_norm_gradient_against_differences(with_sum):
    rng = np.random.default_rng(1)
    s, w, dy = rng.normal(size=(4, 7)), rng.normal(size=7), rng.normal(size=(4, 7))
    ds = rng.normal(size=(4, 7)) if with_sum else None
    eps = 1e-3

    def f(s, w):
        return (dy * lowbit.norm(s, w, eps)[0]).sum() + (0 if ds is None else (ds * s).sum())

    dx, dw = lowbit.norm_grad(s, w, eps, dy, ds)
    h = 1e-6
    for i in range(4):
        for j in range(7):
            e = np.zeros((4, 7))
            e[i, j] = h
            assert abs((f(s + e, w) - f(s - e, w)) / (2 * h) - dx[i, j]) < 1e-7
    for j in range(7):
        e = np.zeros(7)
        e[j] = h
        assert abs((f(s, w + e) - f(s, w - e)) / (2 * h) - dw[j]) < 1e-7


def test_attention_union_is_one_softmax_over_both_key_sets():
    rng = np.random.default_rng(2)
    q, k, v = rng.normal(size=(2, 3, 4, 8)), rng.normal(size=(2, 9, 2, 8)), rng.normal(size=(2, 9, 2, 8))
    whole = lowbit.attention(q, k, v, 0.3, [9, 9])
    first = lowbit.attention(q, k[:, :4], v[:, :4], 0.3, [4, 4])
    both = lowbit.attention(q, k[:, 4:], v[:, 4:], 0.3, [5, 5], prior=first[:2])
    assert np.allclose(both[0], whole[0], atol=1e-12) and np.allclose(both[1], whole[1], atol=1e-12)


def test_attention_without_keys():
    q = np.ones((1, 2, 1, 8))
    out, lse, _ = lowbit.attention(q, np.ones((1, 3, 1, 8)), np.ones((1, 3, 1, 8)), 1.0, [0])
    assert (out == 0).all() and np.isneginf(lse).all()
