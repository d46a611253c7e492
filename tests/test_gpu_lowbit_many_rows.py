"""Calls of more rows than one launch has threads for (2^32 along a grid's
axis): the rows repeat a short stretch, whose own call gives the bytes that
every stretch has to have."""

import numpy as np
import pytest
import torch

from oracle import lowbit
from paper_2607_20940_amd import mssa

from lowbit_common import f64

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


def test_attention_of_many_queries():
    """2^24 query rows of a few rows each, whose joining launch takes a block a row; 16 sequences, again and again.
    The bounds are those of test_gpu_mx_attention.py."""
    few, times, n_q, heads, D, T = 16, 256, 32, 128, 64, 192
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randn(few, n_q, heads, D, generator=g, device="cuda").bfloat16()
    (kc, ks), (vc, vs) = ((torch.randint(0, 256, (few, T, heads, D // 2), generator=g, device="cuda", dtype=torch.uint8),
                           torch.randint(124, 127, (few, T, heads, D // 32), generator=g, device="cuda", dtype=torch.uint8))
                          for _ in range(2))
    d = mssa.mx_attention_desc(few * times, n_q, heads, heads, D, T)
    size = mssa.mssa_mx_attention_workspace_size(d)
    assert size > 0  # shared items: there is a joining launch
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    out = torch.empty(few * times, n_q, heads, D, dtype=torch.bfloat16, device="cuda")
    many = [t.repeat(times, 1, 1, 1) for t in (q, kc, ks, vc, vs)]
    mssa.mssa_mx_attention(d, *many, None, None, None, ws, out)
    torch.cuda.synchronize()

    def values(c, s):
        return lowbit.mx_values(c.cpu().numpy().reshape(-1, D // 2), s.cpu().numpy().reshape(-1, D // 32)).reshape(few, T, heads, D)

    ref, _, mag = lowbit.attention(f64(q), values(kc, ks), values(vc, vs), D ** -0.5, [T] * few)
    bound = 2.0 ** -8 * 1.02 * np.abs(ref) + (2.0 ** -8 * 1.02 + 1e-4) * mag + 1e-30
    ref, bound = (torch.from_numpy(t).cuda() for t in (ref, bound))
    for got in out.view(times, few, n_q, heads, D):
        assert bool(((got.double() - ref).abs() <= bound).all())
