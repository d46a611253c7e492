"""Attention over an MXFP4 cache by the kernel of eight waves (more than 2048
query rows a key head) against the fp64 oracle, with the bounds of
test_gpu_mx_attention.py.  That these sizes reach that kernel is checked by
test_lowbit_rules.py."""

import pytest

from test_gpu_mx_attention import _run

pytestmark = pytest.mark.gpu

# (batch, n_q, q_heads, kv_heads): rows that fill blocks of 256 and that do not, grouped heads
WIDE = [(1, 2049, 1, 1), (1, 2304, 1, 1), (1, 2100, 2, 2), (1, 1100, 4, 2), (2, 700, 6, 2)]
TOKENS = [1, 64, 65, 200, 1000, 1111]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shape", WIDE)
@pytest.mark.parametrize("T", TOKENS)
def test_sizes(D, shape, T):
    B, n_q, H, KH = shape
    _run(B, n_q, H, KH, D, T, seed=D)


# One block an item, and few workers that take several items, or parts of them, in turn.
RAGGED = (5, 2061, 2, 2)
LENGTHS = {192: [0, 1, 192, 0, 65], 700: [64, 0, 700, 1, 5000], 3000: [0, 2999, 0, -3, 130]}


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", list(LENGTHS))
@pytest.mark.parametrize("prior", [False, True])
def test_ragged_lengths(D, T, prior):
    """Empty, single-token, tile-edge, full and out-of-range lengths; tokens past them hold NaN scales."""
    B, n_q, H, KH = RAGGED
    _run(B, n_q, H, KH, D, T, lens=LENGTHS[T], prior=prior, seed=1)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [150, 1500])
@pytest.mark.parametrize("alias", [False, True])
def test_joined(D, T, alias):
    """With an earlier result, in buffers of its own and in place."""
    _run(1, 2500, 2, 2, D, T, prior=True, seed=2, lse_stride=2513, alias=alias)


@pytest.mark.parametrize("amp,scale", [(0.0, 0.2), (3.0, 0.2)])
def test_flat_and_peaked_scores(amp, scale):
    _run(1, 2200, 2, 2, 64, 777, amp=amp, scale=scale, seed=5)


# (batch, n_q, q_heads, kv_heads, head_dim, tokens) of every case
CASES = ([(*s, D, T) for D in (64, 128) for s in WIDE for T in TOKENS]
         + [(*RAGGED, D, T) for D in (64, 128) for T in LENGTHS]
         + [(1, 2500, 2, 2, D, T) for D in (64, 128) for T in (150, 1500)] + [(1, 2200, 2, 2, 64, 777)])
