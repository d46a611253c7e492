"""Root-mean-square norm with the residual's addition, and its backward,
against the fp64 oracle.

Bounds, from the arithmetic: s is one rounding of x + r (equal bit for bit);
y is fp32 arithmetic (a sum of squares in a tree over at most 2^15 values and
five roundings: below 2e-6 relative) rounded once; an 8-bit code is the value
nearest to y / scale, half a step of 2^-4 relative or 2^-10 absolute.  dx
subtracts two terms, each held to 4e-6 of its own size, and is rounded once;
dweight is an fp32 sum over the rows, held to 2e-6 of the sum of magnitudes."""

import numpy as np
import pytest
import torch

from oracle import lowbit
from paper_2607_20940_amd import mssa

from lowbit_common import HALF_ULP, TORCH, Banded, cuda, f64

pytestmark = pytest.mark.gpu

EPS = 1e-6
SHAPES = [(1, 1), (3, 7), (2, 31), (5, 64), (1, 1536), (9, 1536), (4, 511), (4, 513), (3, 2048), (3, 2049), (2, 5120),
          (3, 4097), (2, 8192), (2, 8199), (1, 16385), (1, 32768), (2, 32763)]


def _rows(rng, rows, cols, dtype, pad, scale=1.0):
    wide = cuda(rng.normal(size=(rows, cols + pad)) * np.exp(rng.normal(size=(rows, 1))) * scale, dtype)
    return wide[:, pad // 2: pad // 2 + cols]


def _sum(x, r):
    return x if r is None else (x.float() + r.float()).to(x.dtype)


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("out", ["same", "e4m3"])
@pytest.mark.parametrize("residual,pad", [(True, 0), (False, 3), (True, 6)])
def test_norm(rows, cols, dtype, out, residual, pad):
    rng = np.random.default_rng(rows * 100003 + cols)
    x = _rows(rng, rows, cols, dtype, pad)
    r = _rows(rng, rows, cols, dtype, pad, 3.0) if residual else None
    w = cuda(1 + 0.3 * rng.normal(size=cols), dtype)
    s = Banded((rows, cols), TORCH[dtype])
    rstd = Banded((rows,), torch.float32)
    e4 = out == "e4m3"
    y = Banded((rows, lowbit.padded(cols)), torch.uint8) if e4 else Banded((rows, cols), TORCH[dtype])
    ys = Banded((rows,), torch.float32)
    d = mssa.norm_desc(rows, cols, dtype, "e4m3" if e4 else dtype, EPS, x_stride=cols + pad,
                       residual_stride=cols + pad if residual else 0)
    mssa.mssa_add_rms_norm(d, x, r, w, s.t if residual else None, y.t, ys.t if e4 else None, rstd.t)
    torch.cuda.synchronize()
    want_s = _sum(x, r)
    if residual:
        assert torch.equal(s.t, want_s)
    ref, ref_rstd = lowbit.norm(f64(want_s), f64(w), EPS)
    assert np.abs(f64(rstd.t) / ref_rstd - 1).max() < 2e-6
    if e4:
        scale = np.maximum(np.abs(ref).max(1), lowbit.TINY) / 448
        assert np.abs(f64(ys.t) / scale - 1).max() < 2e-6
        got = lowbit.e4m3_value(y.t.cpu().numpy())
        assert (got[:, cols:] == 0).all()
        v = ref / scale[:, None]
        bound = np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10) * (1 + 1e-5)
        assert (np.abs(got[:, :cols] - v) <= bound).all()
        assert np.abs(got).max() == 448
    else:
        assert (np.abs(f64(y.t) - ref) <= (HALF_ULP[dtype] * 1.001 + 2e-6) * np.abs(ref) + 1e-38).all()
    assert s.intact() and y.intact() and ys.intact() and rstd.intact()


@pytest.mark.parametrize("alias", ["x", "residual"])
def test_norm_sum_in_place(alias):
    rng = np.random.default_rng(3)
    x, r = (cuda(rng.normal(size=(37, 1536)), "bf16") for _ in range(2))
    w = cuda(np.ones(1536), "bf16")
    want = _sum(x, r)
    y = torch.empty_like(x)
    dst = x if alias == "x" else r
    mssa.mssa_add_rms_norm(mssa.norm_desc(37, 1536, eps=EPS), x, r, w, dst, y)
    torch.cuda.synchronize()
    assert torch.equal(dst, want)


def test_norm_zero_tiny_and_non_finite_rows():
    """A zero row gives zeros; a row whose largest output lies below 2^-100
    keeps the scale of 2^-100; a NaN or an infinity stays in its own row and
    shows in its scale."""
    x = torch.ones(6, 96, device="cuda")
    x[0] = 0
    x[1] = 2.0 ** -125
    x[2, 5] = float("nan")
    x[3, 95] = float("inf")
    x[4] = 3e38  # squares pass fp32's range: 1 / rms is 0, as the fp32 formula says
    w = torch.ones(96, device="cuda")
    y = torch.empty(6, 96, dtype=torch.uint8, device="cuda")
    ys = torch.empty(6, device="cuda")
    mssa.mssa_add_rms_norm(mssa.norm_desc(6, 96, "f32", "e4m3", 1.0), x, None, w, None, y, ys)
    torch.cuda.synchronize()
    v, s = lowbit.e4m3_value(y.cpu().numpy()), f64(ys)
    tiny = 2.0 ** -100 / 448
    assert (v[0] == 0).all() and abs(s[0] / tiny - 1) < 1e-6 and abs(s[1] / tiny - 1) < 1e-6
    assert (np.abs(v[1] - 448 * 2.0 ** -25) <= 2.0 ** -10).all()
    assert np.isnan(s[2]) and np.isnan(s[3]) and (v[4] == 0).all()
    assert (v[5] == 448).all() and abs(s[5] * 448 - np.sqrt(0.5)) < 1e-6


def test_norm_on_another_stream_and_replayed():
    """The library takes the caller's stream; a recorded call gives the same
    bytes on every replay."""
    rng = np.random.default_rng(4)
    x, r = (cuda(rng.normal(size=(300, 1536)), "bf16") for _ in range(2))
    w = cuda(1 + rng.normal(size=1536), "bf16")
    d = mssa.norm_desc(300, 1536, out="e4m3", eps=EPS)
    bufs = [[torch.empty_like(x), torch.empty(300, 1536, dtype=torch.uint8, device="cuda"),
             torch.empty(300, device="cuda")] for _ in range(2)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    mssa.mssa_add_rms_norm(d, x, r, w, *bufs[0], stream=side)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mssa.mssa_add_rms_norm(d, x, r, w, *bufs[1])
    for _ in range(3):
        for b in bufs[1]:
            b.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*bufs))


@pytest.mark.parametrize("rows,cols", [(0, 40)] + SHAPES + [(700, 96), (1500, 1536), (1100, 2056)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("with_sum", [False, True])
def test_norm_backward(rows, cols, dtype, with_sum):
    rng = np.random.default_rng(rows * 7 + cols)
    s = _rows(rng, rows, cols, dtype, 5)
    w = cuda(1 + 0.3 * rng.normal(size=cols), dtype)
    dy, ds = (cuda(rng.normal(size=(rows, cols)), dtype) for _ in range(2))
    d = mssa.norm_desc(rows, cols, dtype, eps=EPS, sum_stride=cols + 5)
    size = mssa.mssa_add_rms_norm_workspace_size(d)
    ws = Banded((size,), torch.uint8, 0xff)
    rstd = torch.rsqrt(s.float().square().mean(-1) + EPS) if rows else torch.empty(0, device="cuda")
    dx, dw = Banded((rows, cols), TORCH[dtype]), Banded((cols,), torch.float32)
    mssa.mssa_add_rms_norm_backward(d, s, w, rstd, dy, ds if with_sum else None, ws.t, dx.t, dw.t)
    torch.cuda.synchronize()
    assert dx.intact() and dw.intact() and ws.intact()
    S, W, DY = f64(s), f64(w), f64(dy)
    if rows == 0:
        assert (f64(dw.t) == 0).all()
        return
    DS = f64(ds) if with_sum else None
    ref, ref_w = lowbit.norm_grad(S, W, EPS, DY, DS)
    n = 1 / np.sqrt((S * S).mean(1, keepdims=True) + EPS)
    size_x = n * np.abs(W * DY) + np.abs(S) * n ** 3 * np.abs(W * DY * S).mean(1, keepdims=True)
    if with_sum:
        size_x = size_x + np.abs(DS)
    assert (np.abs(f64(dx.t) - ref) <= HALF_ULP[dtype] * 1.001 * np.abs(ref) + 4e-6 * size_x).all()
    assert (np.abs(f64(dw.t) - ref_w) <= 2e-6 * np.abs(DY * S * n).sum(0) + 1e-30).all()


def test_norm_backward_in_place_and_reproducible():
    rng = np.random.default_rng(6)
    s, dy, ds = (cuda(rng.normal(size=(3000, 384)), "bf16") for _ in range(3))
    w = cuda(1 + rng.normal(size=384), "bf16")
    rstd = torch.rsqrt(s.float().square().mean(-1) + EPS)
    d = mssa.norm_desc(3000, 384, eps=EPS)
    ws = torch.empty(mssa.mssa_add_rms_norm_workspace_size(d), dtype=torch.uint8, device="cuda")
    got = []
    for alias in (None, None, "dy", "dsum"):
        a, b = dy.clone(), ds.clone()
        dx = {None: torch.empty_like(dy), "dy": a, "dsum": b}[alias]
        dw = torch.empty(384, device="cuda")
        mssa.mssa_add_rms_norm_backward(d, s, w, rstd, a, b, ws, dx, dw)
        got.append((dx.clone(), dw))
    torch.cuda.synchronize()
    assert all(torch.equal(g[0], got[0][0]) and torch.equal(g[1], got[0][1]) for g in got)


def test_norm_gradient_against_differences_of_the_kernel():
    """The kernel's own forward, differenced in fp32 along random directions.
    A central difference with h = 1e-2 of a sum of 12 x 40 terms of size one:
    its third-order term is below 1e-4 and fp32's rounding of the sum below
    1e-3 over 2 h, so 2e-3 of the gradient's size holds."""
    rng = np.random.default_rng(8)
    x, dy = (cuda(rng.normal(size=(12, 40)), "f32") for _ in range(2))
    w = cuda(1 + 0.2 * rng.normal(size=40), "f32")
    d = mssa.norm_desc(12, 40, "f32", eps=EPS)

    def y_of(x, w):
        y, rstd = torch.empty_like(x), torch.empty(12, device="cuda")
        mssa.mssa_add_rms_norm(d, x, None, w, None, y, None, rstd)
        return y, rstd

    rstd = y_of(x, w)[1]
    dx, dw = torch.empty_like(x), torch.empty(40, device="cuda")
    ws = torch.empty(max(16, mssa.mssa_add_rms_norm_workspace_size(d)), dtype=torch.uint8, device="cuda")
    mssa.mssa_add_rms_norm_backward(d, x, w, rstd, dy, None, ws, dx, dw)
    h = 1e-2
    for k in range(4):
        ux, uw = cuda(rng.normal(size=(12, 40)), "f32"), cuda(rng.normal(size=40), "f32")
        fx = ((y_of(x + h * ux, w)[0] - y_of(x - h * ux, w)[0]).double() * dy.double()).sum() / (2 * h)
        fw = ((y_of(x, w + h * uw)[0] - y_of(x, w - h * uw)[0]).double() * dy.double()).sum() / (2 * h)
        gx, gw = (dx.double() * ux.double()), (dw.double() * uw.double())
        assert abs(fx - gx.sum()) <= 2e-3 * gx.abs().sum()
        assert abs(fw - gw.sum()) <= 2e-3 * gw.abs().sum()
