"""The oracle of the operators for streams served together, pinned by facts that do
not come from it: hand-worked values, invariances, the operators of other parts of
the oracle."""

import numpy as np
import pytest

from oracle import lowbit, paged

rng = np.random.default_rng(0)


def test_adapter_is_a_change_of_the_weights():
    x, w, bias = rng.normal(size=(7, 5)), rng.normal(size=(6, 5)), rng.normal(size=6)
    a, b = rng.normal(size=(2, 2, 3, 5)), rng.normal(size=(2, 6, 3))
    ys, _, _ = paged.adapter_project(x, w, bias, [1, 4, 7], [1, 0], a, b, [0.5, 2.0], 2, 3.0)
    for r in range(7):
        j = None if r < 1 else 1 if r < 4 else 0
        for p in range(2):
            m = w[3 * p:3 * p + 3]
            if j is not None:
                m = m + [0.5, 2.0][j] * b[j, 3 * p:3 * p + 3] @ a[j, p]
            want = (m @ x[r] + bias[3 * p:3 * p + 3]) * (3.0 if p == 0 else 1.0)
            assert np.allclose(ys[p][r], want, rtol=1e-12)


@pytest.mark.parametrize("halves", [False, True])
def test_rotation(halves):
    u, v = (0, 2) if halves else (0, 1)
    x = np.zeros((1, 1, 6))
    x[0, 0, u], x[0, 0, 5] = 2.0, 7.0
    y, mag = paged.rotate(x, np.array([[np.pi / 2, 0.3]]), halves)  # a quarter turn of the first pair
    want = np.zeros(6)
    want[v], want[5] = 2.0, 7.0
    assert np.allclose(y[0, 0], want, atol=1e-15) and mag[0, 0, v] == 2.0
    # scores depend on the distance of positions alone, lengths stay
    q, k, f = rng.normal(size=(1, 1, 8)), rng.normal(size=(1, 1, 8)), rng.normal(size=4)
    dots = []
    for a, b in ((3, 10), (1000, 1007)):
        turned = [paged.rotate(t, f[None] * p, halves)[0] for t, p in ((q, a), (k, b))]
        dots.append((turned[0] * turned[1]).sum())
        assert np.isclose(np.linalg.norm(turned[0]), np.linalg.norm(q))
    assert np.isclose(*dots)


def test_places():
    index, place = paged.places([1, 3, 3, 6], [5, 9, 4], [[7, 2, 0], [1, 1, 1], [3, -1, 9]], 2, 8, 7)
    assert index == [None, 3, 4, 1, 2, 3, None]
    assert place == [None, (2, 1), (0, 0), (3, 1), None, None, None]
    assert paged.places(None, [1, 4], [[0], [1]], 2, 2, 4) == ([-1, 0, 2, 3], [None, (0, 0), None, None])


def test_attention_without_mask_is_that_over_a_cache():
    q, k, v = rng.normal(size=(6, 4, 8)), rng.normal(size=(5, 3, 2, 8)), rng.normal(size=(5, 3, 2, 8))
    table = [[4, 0, 2], [1, 3, -1]]
    out, lse, mag = paged.attention(q, k, v, [0, 2, 6], [8, 5], table, 0.3)
    for b, (r, n) in enumerate(((slice(0, 2), 8), (slice(2, 6), 5))):
        flat = [t[table[b]].reshape(1, -1, 2, 8) for t in (k, v)]
        o, l, m = lowbit.attention(q[None, r], *flat, 0.3, [n])
        assert np.allclose(out[r], o[0]) and np.allclose(lse[:, r], l[0]) and np.allclose(mag[r], m[0])


def test_mask_by_hand():
    """One query dim of zeros: the output is the mean of the values that are seen."""
    v = np.arange(1.0, 9.0).reshape(4, 2, 1, 1)
    out, lse, _ = paged.attention(np.zeros((3, 1, 1)), np.zeros((4, 2, 1, 1)), v, [0, 3], [7], [[0, 1, 2, 3]], 1.0, 2)
    # indices 4, 5, 6; blocks of two: tokens 0 and 1 see six, token 2 all seven
    assert np.allclose(out[:, 0, 0], [3.5, 3.5, 4.0]) and np.allclose(lse[0], np.log([6, 6, 7]))
    out, lse, _ = paged.attention(np.zeros((3, 1, 1)), np.zeros((4, 2, 1, 1)), v, [0, 3], [2], [[0, 1, 2, 3]], 1.0, 1)
    # a cache shorter than the chunk: the first token's index is -1
    assert np.allclose(out[:, 0, 0], [0.0, 1.0, 1.5]) and np.isneginf(lse[0, 0])
    out, _, _ = paged.attention(np.zeros((1, 1, 1)), np.zeros((4, 2, 1, 1)), v, [0, 1], [6], [[0, -1, 2]], 1.0)
    assert np.allclose(out, (1 + 2 + 5 + 6) / 4)


def test_joined_result_is_the_softmax_over_both():
    q, k, v = rng.normal(size=(3, 1, 4)), rng.normal(size=(2, 5, 1, 4)), rng.normal(size=(2, 5, 1, 4))
    o, l, _ = paged.attention(q, k, v, None, [5], [[1]], 0.5)
    both, lse, _ = paged.attention(q, k, v, None, [5], [[0]], 0.5, 0, (o, l))
    whole, want, _ = paged.attention(q, k, v, None, [10], [[0, 1]], 0.5)
    assert np.allclose(both, whole) and np.allclose(lse, want)
