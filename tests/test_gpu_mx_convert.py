"""Conversion to MXFP4 and back against the oracle's formats: codes and scale
bytes equal bit for bit, values equal."""

import numpy as np
import pytest
import torch

from oracle import lowbit
from paper_2607_20940_amd import mssa

from lowbit_common import TORCH, Banded, cuda, f64

pytestmark = pytest.mark.gpu


def _round_trip(x, dtype):
    rows, cols = x.shape
    (cr, cb), (sr, sb) = mssa.mx_shapes(rows, cols)
    codes, scales = Banded((cr, cb), torch.uint8, 0x77), Banded((sr, sb), torch.uint8, 0x77)
    mssa.mssa_mx_quantize(rows, cols, dtype, x, codes.t, scales.t, x_stride=x.stride(0))
    y = Banded((rows, cols), TORCH[dtype])
    mssa.mssa_mx_dequantize(rows, cols, dtype, codes.t, scales.t, y.t)
    torch.cuda.synchronize()
    assert codes.intact() and scales.intact() and y.intact()
    return codes.t.cpu().numpy(), scales.t.cpu().numpy(), f64(y.t)


def _check(x, dtype):
    codes, scales, y = _round_trip(x, dtype)
    want, byte = lowbit.mx_codes(f64(x))
    assert np.array_equal(scales, byte)
    # a negative value that rounds to zero keeps its sign bit: compare values
    got = lowbit.mx_unpack(codes)
    assert np.array_equal(lowbit.e2m1_value(got), lowbit.e2m1_value(want))
    assert (got[:, x.shape[1]:] == 0).all()
    ref = lowbit.mx_values(codes, byte)[:, : x.shape[1]]
    keep = np.abs(ref) >= (2.0 ** -133 if dtype == "bf16" else 2.0 ** -149)
    assert np.array_equal(np.where(keep, y, 0), np.where(keep, ref, 0))


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 33), (7, 31), (5, 128), (1000, 128), (2, 5120), (300, 64),
                                       (17, 100), (65, 1000), (1, 8), (4, 9)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad", [0, 3])
def test_codes_and_values(rows, cols, dtype, pad):
    rng = np.random.default_rng(rows + cols)
    x = rng.normal(size=(rows, cols + pad)) * np.exp(2 * rng.normal(size=(rows, 1)))
    x[rng.random(x.shape) < 0.05] = 0
    _check(cuda(x, dtype)[:, pad // 2: pad // 2 + cols], dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_tie_and_neighbour_at_every_scale(dtype):
    """Ties of e2m1 and the values next to them, at exponents from the
    smallest scale to the largest."""
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 0.5, 1.5, 3.0])
    near = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -23
    rows = []
    for e in list(range(-124, -110)) + list(range(-8, 9)) + list(range(110, 126)):
        v = np.concatenate([[4.0], ties[:10], ties[:10] * (1 + near), -ties[:10] * (1 - near / 2), [-6.0]])
        rows.append(v[:32] * 2.0 ** e)
    _check(cuda(np.array(rows), dtype), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_smallest_largest_and_non_finite_blocks(dtype):
    """Blocks below the smallest scale, at the type's largest value, of zeros,
    and with an infinity or a NaN, which stay in their own block."""
    t = TORCH[dtype]
    x = torch.ones(8, 96, dtype=t, device="cuda")
    x[0, 32:64] = 0
    x[1, 32:64] = 2.0 ** -126
    x[2, 32:64] = 2.0 ** -130
    x[3, 40] = torch.finfo(t).max
    x[4, 40] = torch.finfo(t).min
    x[5, 40] = float("inf")
    x[6, 63] = float("nan")
    x[7, 32] = -float("inf")
    codes, scales, y = _round_trip(x, dtype)
    want, byte = lowbit.mx_codes(f64(x))
    assert np.array_equal(scales, byte)
    assert np.array_equal(lowbit.e2m1_value(lowbit.mx_unpack(codes)), lowbit.e2m1_value(want))
    assert np.isnan(y[5:, 32:64]).all() and np.isfinite(y[:5]).all()
    assert np.isfinite(y[:, :32]).all() and np.isfinite(y[:, 64:]).all()


def test_offsets_past_32_bits():
    """Rows far into a tensor of over 2^32 elements."""
    rows, cols = (1 << 32) // 128 + 3, 128
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(0)
    tail = cuda(rng.normal(size=(3, cols)), "bf16")
    x[-3:] = tail
    codes, scales = (torch.empty(s, dtype=torch.uint8, device="cuda") for s in mssa.mx_shapes(rows, cols))
    mssa.mssa_mx_quantize(rows, cols, "bf16", x, codes, scales)
    x.fill_(1)
    mssa.mssa_mx_dequantize(rows, cols, "bf16", codes, scales, x)
    torch.cuda.synchronize()
    want, byte = lowbit.mx_codes(f64(tail))
    assert np.array_equal(scales[-3:].cpu().numpy(), byte)
    assert np.array_equal(f64(x[-3:]), lowbit.mx_values(lowbit.mx_pack(want), byte))
    assert int((x[:-3] != 0).sum()) == 0
