"""Calls of more rows than one launch has threads for (2^32 along a grid's
axis): the rows repeat a short stretch, whose own call gives the bytes that
every stretch has to have."""

import pytest
import torch

from paper_2607_20940_amd import mssa

pytestmark = pytest.mark.gpu

STRETCH = 1 << 20


def _repeated(short, rows):
    """`rows` rows that repeat the rows of `short`."""
    n = -(-rows // short.shape[0])
    return short.repeat(n, *([1] * (short.dim() - 1)))[:rows]


def _same(got, short):
    """Whether every stretch of got's rows is short's."""
    n, rest = divmod(got.shape[0], short.shape[0])
    whole = got[: n * short.shape[0]].view(n, *short.shape)
    return all(torch.equal(w, short) for w in whole) and torch.equal(got[got.shape[0] - rest:], short[:rest])


@pytest.mark.parametrize("out", ["bf16", "e4m3"])
def test_norm(out):
    rows, cols = (1 << 26) + 5, 3  # a wave a row: 2^32 threads and more
    g = torch.Generator(device="cuda").manual_seed(0)
    x, r = (torch.randn(STRETCH, cols, generator=g, device="cuda").bfloat16() for _ in range(2))
    w = torch.tensor([1.0, -2.0, 0.5], device="cuda").bfloat16()

    def run(x, r):
        n = x.shape[0]
        s = torch.empty_like(x)
        y = torch.empty((n, 32), dtype=torch.uint8, device="cuda") if out == "e4m3" else torch.empty_like(x)
        ys, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        mssa.mssa_add_rms_norm(mssa.norm_desc(n, cols, "bf16", out), x, r, w, s, y, ys if out == "e4m3" else None, rstd)
        return (s, y, ys, rstd) if out == "e4m3" else (s, y, rstd)

    short = run(x, r)
    for got, want in zip(run(_repeated(x, rows), _repeated(r, rows)), short):
        assert _same(got, want)


def test_conversion():
    """Single values, a block each: 2^32 threads and more there and back."""
    rows = (1 << 30) + 5
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(STRETCH, 1, generator=g, device="cuda").bfloat16()

    def run(x):
        n = x.shape[0]
        codes, scales = (torch.empty(s, dtype=torch.uint8, device="cuda") for s in mssa.mx_shapes(n, 1))
        mssa.mssa_mx_quantize(n, 1, "bf16", x, codes, scales)
        y = torch.empty_like(x)
        mssa.mssa_mx_dequantize(n, 1, "bf16", codes, scales, y)
        return codes, scales, y

    short = run(x)
    for got, want in zip(run(_repeated(x, rows)), short):
        assert _same(got, want)


def test_product():
    """Tiles of 64 tokens would be 2^24 blocks of 256 threads."""
    rows = 1 << 30
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randint(0, 127, (STRETCH, 32), generator=g, device="cuda", dtype=torch.uint8)
    xs = torch.rand(STRETCH, generator=g, device="cuda")
    w = torch.randint(0, 256, (2, 16), generator=g, device="cuda", dtype=torch.uint8)
    ws = torch.full((2, 1), 127, dtype=torch.uint8, device="cuda")

    def run(x, xs):
        y = torch.empty(x.shape[0], 2, dtype=torch.bfloat16, device="cuda")
        mssa.mssa_mx_project(mssa.mx_project_desc(x.shape[0], 32, 2), x, xs, w, ws, None, [y])
        return y

    short = run(x, xs)
    assert _same(run(_repeated(x, rows), _repeated(xs, rows)), short)
