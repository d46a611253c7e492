"""Every scale byte with every code, through each of the product's paths: a
contraction of one value, so that each output is one weight times one.  Exact
in both output types; below 2^-123 (where type and sums have subnormal numbers
or none) an absolute 2^-123."""

import numpy as np
import pytest
import torch

from oracle import lowbit
from paper_2607_20940_amd import mssa

from lowbit_common import TORCH, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["e4m3", "mxfp4"])
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 20, 70])
def test_product_of_one_value(fmt, out, rows):
    features = 256 * 16
    w = torch.zeros(features, 16, dtype=torch.uint8)
    w[:, 0] = torch.arange(features) % 16
    ws = (torch.arange(features) // 16).to(torch.uint8)[:, None]
    one, blocks = (0x38, 32) if fmt == "e4m3" else (2, 16)
    x = torch.zeros(rows, blocks, dtype=torch.uint8)
    x[:, 0] = one
    xs = torch.ones(rows) if fmt == "e4m3" else torch.full((rows, 1), 127, dtype=torch.uint8)
    y = torch.empty(rows, features, dtype=TORCH[out], device="cuda")
    mssa.mssa_mx_project(mssa.mx_project_desc(rows, 1, features, 1, fmt, out), x.cuda(), xs.cuda(), w.cuda(),
                         ws.contiguous().cuda(), None, [y])
    torch.cuda.synchronize()
    got = f64(y)
    want = lowbit.mx_values(w.numpy(), ws.numpy())[:, 0]
    with np.errstate(over="ignore"):
        want = want.astype(np.float32).astype(np.float64)  # past fp32's range: infinite
    want = np.broadcast_to(want, got.shape)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(np.isinf(got), np.isinf(want))
    fine = np.isfinite(want)
    assert (np.abs(got[fine] - want[fine]) <= np.where(np.abs(want[fine]) < 2.0 ** -123, 2.0 ** -123, 0)).all()
