"""Products whose contraction ends inside a stage of the tile kernels: values
against the fp64 oracle (bounds of test_gpu_mx_project.py), and NaN scales
among a row's last blocks, which reach their own row's outputs only."""

import numpy as np
import pytest
import torch

from paper_2607_20940_amd import mssa

from lowbit_common import TORCH, cuda, quantize
from test_gpu_mx_project import _project

pytestmark = pytest.mark.gpu

# Contractions of 20, 28, 36 and 44 blocks end four blocks into a stage of eight
# with scales that are moved from memory to LDS as they lie there.
SHORT = [640, 896, 1152, 1408]
# (rows, features) of a kernel with tiles of 64 x 128, and of one with 256 x 256
SMALL, LARGE = (70, 260), (4090, 4090)


@pytest.mark.parametrize("fmt", ["e4m3", "mxfp4"])
@pytest.mark.parametrize("cols", SHORT)
@pytest.mark.parametrize("rows", [33, 64, 70, 128])
def test_short_last_stage(fmt, cols, rows):
    _project(rows, cols, 258, 3, fmt, "bf16", factor=0.3)


@pytest.mark.parametrize("fmt", ["e4m3", "mxfp4"])
@pytest.mark.parametrize("cols", [640, 1152])
def test_short_last_stage_of_large_tiles(fmt, cols):
    _project(LARGE[0], cols, LARGE[1], 5, fmt, "bf16", factor=0.3)


def _nan_outputs(rows, cols, features, out, bad_tokens, bad_features, block):
    """Marks the scale of `block` of some tokens and features NaN; the outputs' NaNs have to be theirs."""
    rng = np.random.default_rng(rows + cols)
    x, xs = quantize(cuda(rng.normal(size=(rows, cols)), "f32"))
    w, ws = quantize(cuda(rng.normal(size=(features, cols)), "f32"))
    xs[bad_tokens, block] = 255
    ws[bad_features, block] = 255
    y = torch.empty(rows, features, dtype=TORCH[out], device="cuda")
    mssa.mssa_mx_project(mssa.mx_project_desc(rows, cols, features, 1, "mxfp4", out), x, xs, w, ws, None, [y])
    want = torch.zeros(rows, features, dtype=torch.bool, device="cuda")
    want[bad_tokens] = True
    want[:, bad_features] = True
    assert torch.equal(torch.isnan(y), want)


@pytest.mark.parametrize("cols", SHORT)
@pytest.mark.parametrize("from_end", [16, 15, 14, 13, 5, 4, 1])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_nan_blocks_of_small_tiles(cols, from_end, out):
    """Rows in the middle of a tile, first and last ones of tiles: the row before each stays finite."""
    _nan_outputs(SMALL[0], cols, SMALL[1], out, [10, 63, 64, 69], [0, 50, 127, 128, 259], cols // 32 - from_end)


@pytest.mark.parametrize("cols", [640, 1152])
@pytest.mark.parametrize("from_end", [16, 13, 1])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_nan_blocks_of_large_tiles(cols, from_end, out):
    _nan_outputs(LARGE[0], cols, LARGE[1], out, [10, 255, 256, 4089], [0, 50, 255, 256, 4089], cols // 32 - from_end)


def test_no_nan_where_no_scale_is():
    """The same sizes without a NaN scale: nothing next to the operands' last bytes shows."""
    for cols in SHORT:
        _nan_outputs(SMALL[0], cols, SMALL[1], "f32", [], [], 0)
