"""Product with MXFP4 weights against the fp64 oracle, tokens as 8-bit rows
and as MXFP4, over the kernels that few, ordinary and many tokens reach.

Bounds.  An output is off by its own rounding (bf16: 2^-8 of itself at most,
2^-8 / sqrt(3) rms) and by the sum's error: 1e-6 of the sum of magnitudes
where products are exact and sums fp32 (MXFP4 tokens, and 8-bit tokens with
fp32 outputs); 2^-12 of it where 8-bit tokens go to bf16 outputs, because the
matrix core aligns a step's e4m3 products to the largest of them."""

import numpy as np
import pytest
import torch

from oracle import lowbit
from paper_2607_20940_amd import mssa

from lowbit_common import HALF_ULP, TORCH, Banded, cuda, f64, quantize

pytestmark = pytest.mark.gpu


def _tokens(rng, rows, cols, fmt):
    """(x, x_scales, values) of random tokens in 8-bit rows or MXFP4."""
    v = rng.normal(size=(rows, cols)) * np.exp(0.5 * rng.normal(size=(1, cols)))
    if fmt == "mxfp4":
        codes, scales = quantize(cuda(v, "f32"))
        return codes, scales, lowbit.mx_values(codes.cpu().numpy(), scales.cpu().numpy())[:, :cols]
    code = np.zeros((rows, lowbit.padded(cols)), np.uint8)
    code[:, :cols] = rng.integers(0, 127, (rows, cols)) | (rng.integers(0, 2, (rows, cols)) << 7)  # every finite value
    scale = np.exp(rng.normal(size=rows) - 6).astype(np.float32)
    return (torch.from_numpy(code).cuda(), torch.from_numpy(scale).cuda(),
            lowbit.e4m3_value(code[:, :cols]) * scale[:, None].astype(np.float64))


def _project(rows, cols, features, parts, fmt, out, bias=True, factor=1.0, seed=0):
    rng = np.random.default_rng(seed + rows + cols + features)
    x, xs, xv = _tokens(rng, rows, cols, fmt)
    w, ws = quantize(cuda(rng.normal(size=(features, cols)) / np.sqrt(cols), "f32"))
    wv = lowbit.mx_values(w.cpu().numpy(), ws.cpu().numpy())[:, :cols]
    b = cuda(rng.normal(size=features), out) if bias else None
    ys = [Banded((rows, features // parts), TORCH[out]) for _ in range(parts)]
    d = mssa.mx_project_desc(rows, cols, features, parts, fmt, out, factor)
    mssa.mssa_mx_project(d, x, xs, w, ws, b, [y.t for y in ys])
    torch.cuda.synchronize()
    ref = lowbit.project(xv, wv, f64(b) if bias else None, parts, factor)
    size = lowbit.project(np.abs(xv), np.abs(wv), None, parts, abs(factor))
    for p, y in enumerate(ys):
        assert y.intact()
        err = np.abs(f64(y.t) - ref[p])
        summed = 2.0 ** -12 if fmt == "e4m3" and out == "bf16" else 1e-6
        assert (err <= HALF_ULP[out] * 1.01 * np.abs(ref[p]) + summed * size[p] + 1e-30).all(), (p, err.max())
        if out == "bf16" and err.size >= 1000:
            assert np.sqrt((err ** 2).mean()) <= 2.0 ** -8 / np.sqrt(3) * 1.05 * np.sqrt((ref[p] ** 2).mean())
    return ys


@pytest.mark.parametrize("fmt", ["e4m3", "mxfp4"])
@pytest.mark.parametrize("rows", [1, 2, 16, 17, 32, 33, 100, 128, 129, 300])
@pytest.mark.parametrize("cols,features,parts", [(1536, 384, 3), (32, 16, 1), (100, 60, 3), (64, 7, 1), (520, 129, 3),
                                                 (1000, 96, 8)])
def test_product(fmt, rows, cols, features, parts):
    _project(rows, cols, features, parts, fmt, "bf16", factor=0.3 if parts == 3 else 1.0)


@pytest.mark.parametrize("fmt", ["e4m3", "mxfp4"])
@pytest.mark.parametrize("rows,cols,features,parts", [(4, 128, 48, 2), (200, 1536, 512, 2), (70, 33, 5, 5), (40, 1, 3, 1)])
def test_fp32_outputs(fmt, rows, cols, features, parts):
    _project(rows, cols, features, parts, fmt, "f32", bias=rows != 70)


@pytest.mark.parametrize("fmt", ["e4m3", "mxfp4"])
@pytest.mark.parametrize("rows,cols,features", [(4099, 288, 4104), (4096, 1536, 4608), (2050, 1120, 8001)])
def test_large_tiles(fmt, rows, cols, features):
    """Enough tiles for the large-tile kernel, at its edges and on odd sizes."""
    _project(rows, cols, features, 3, fmt, "bf16", factor=0.1275)


@pytest.mark.parametrize("fmt", ["e4m3", "mxfp4"])
@pytest.mark.parametrize("rows", [1, 60])
def test_nan_scales_reach_their_rows_only(fmt, rows):
    """A NaN block of a weight row makes that feature NaN, one of a token that
    token; blocks past the row's end and rows past the tile's do neither."""
    rng = np.random.default_rng(0)
    cols, features = 96, 40
    x, xs, _ = _tokens(rng, rows, cols, fmt)
    w, ws = quantize(cuda(rng.normal(size=(features, cols)), "f32"))
    ws[5, 1] = 255
    if fmt == "mxfp4":
        xs[0, 2] = 255
    else:
        xs[0] = float("nan")
    y = torch.empty(rows, features, device="cuda")
    mssa.mssa_mx_project(mssa.mx_project_desc(rows, cols, features, 1, fmt, "f32"), x, xs, w, ws, None, [y])
    torch.cuda.synchronize()
    bad = np.isnan(f64(y))
    want = np.zeros_like(bad)
    want[:, 5] = True
    want[0] = True
    assert np.array_equal(bad, want)


def test_reproducible_and_replayed():
    rng = np.random.default_rng(1)
    x, xs, _ = _tokens(rng, 700, 512, "e4m3")
    w, ws = quantize(cuda(rng.normal(size=(768, 512)), "f32"))
    d = mssa.mx_project_desc(700, 512, 768, 3)
    a, b = ([torch.empty(700, 256, dtype=torch.bfloat16, device="cuda") for _ in range(3)] for _ in range(2))
    mssa.mssa_mx_project(d, x, xs, w, ws, None, a)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mssa.mssa_mx_project(d, x, xs, w, ws, None, b)
    for _ in range(3):
        for t in b:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(s, t) for s, t in zip(a, b))
