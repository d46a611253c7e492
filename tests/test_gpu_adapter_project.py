"""Projection with an adapter per segment against the fp64 oracle.

Bounds: bf16 products exact, fp32 sums of K terms (K 2^-23 of the sum of
magnitudes covers any order and the matrix cores' alignment), the low-rank
factor rounded once (2^-8 of the adapter's magnitudes), the output once (2^-8
of itself)."""

import numpy as np
import pytest
import torch

from oracle import paged
from paper_2607_20940_amd import mssa

from lowbit_common import Banded, cuda, f64
from paged_common import ints

pytestmark = pytest.mark.gpu


def _inputs(rng, M, K, N, parts, J, R, pad=0, bias=True):
    x = cuda(rng.normal(size=(M, K + pad)), "bf16")[:, :K]
    w = cuda(rng.normal(size=(N, K)) * K ** -0.5, "bf16")
    b0 = cuda(rng.normal(size=N), "bf16") if bias else None
    a = cuda(rng.normal(size=(J, parts, R, K)) * K ** -0.5, "bf16")
    b = cuda(rng.normal(size=(J, N, R)), "bf16")
    return x, w, b0, a, b


def _run(M, K, N, parts, J, R, begin, which, pad=0, bias=True, scaled=True, factor=1.0, seed=0, edit=None, check=True):
    rng = np.random.default_rng(seed + M + K + N + R)
    x, w, b0, a, b = _inputs(rng, M, K, N, parts, J, R, pad, bias)
    scale = rng.normal(size=J).astype(np.float32) if scaled else None
    if edit:
        edit(x, w, a, b)
    ys = [Banded((M, N // parts), torch.bfloat16, 3.0) for _ in range(parts)]
    d = mssa.adapter_project_desc(M, K, N, len(which), J, R, parts=parts, part0_scale=factor, x_stride=K + pad)
    ws = Banded((mssa.mssa_adapter_project_workspace_size(d),), torch.uint8, 0xff)  # NaN until written
    mssa.mssa_adapter_project(d, x, w, b0, ints(begin), ints(which), a, b, None if scale is None else torch.from_numpy(scale).cuda(),
                              ws.t, [y.t for y in ys])
    torch.cuda.synchronize()
    assert ws.intact() and all(y.intact() for y in ys)
    if not check:
        return [f64(y.t) for y in ys]
    ref, mag, low = paged.adapter_project(f64(x), f64(w), None if b0 is None else f64(b0), begin, which, f64(a), f64(b),
                                          None if scale is None else scale.astype(np.float64), parts, factor)
    for y, r, m, u in zip(ys, ref, mag, low):
        got = f64(y.t)
        tol = 2.0 ** -8 * 1.01 * np.abs(r) + (K + R + 8) * 2.0 ** -23 * (m + u) + 2.0 ** -8 * u
        assert (np.abs(got - r) <= tol).all(), (np.abs(got - r) / tol).max()


def _cuts(rng, M, S):
    return np.concatenate(([0], np.sort(rng.integers(0, M + 1, size=S - 1)), [M])) if S else np.zeros(1, dtype=int)


SIZES = [(1, 64, 96, 3), (5, 8, 9, 1), (16, 128, 384, 3), (33, 100, 77, 1), (64, 256, 192, 2), (65, 192, 520, 1), (130, 72, 300, 3),
         (300, 64, 1032, 1), (611, 608, 1000, 1), (700, 320, 768, 3), (520, 128, 2304, 3)]


@pytest.mark.parametrize("M,K,N,parts", SIZES)
@pytest.mark.parametrize("R", [1, 8, 12, 16, 40, 64, 200])
@pytest.mark.parametrize("S", [1, 3, 20])
def test_sizes(M, K, N, parts, R, S):
    rng = np.random.default_rng(S)
    _run(M, K, N, parts, 3, R, _cuts(rng, M, S), rng.integers(-1, 3, size=S), factor=0.3)


@pytest.mark.parametrize("M", [1, 7, 16, 17, 32, 33, 50, 64, 200])
@pytest.mark.parametrize("K,N,R", [(512, 768, 16), (1536, 1024, 8), (100, 90, 5)])
def test_a_request_a_row(M, K, N, R):
    _run(M, K, N, 3 if N % 3 == 0 else 1, 5, R, np.arange(M + 1), (np.arange(M) * 3) % 6 - 1)


@pytest.mark.parametrize("M", [4, 40, 300])
def test_rows_outside_all_segments_have_no_adapter(M):
    _run(M, 128, 256, 2, 2, 16, [M // 4, M // 2, M // 2, M - 1], [0, 1, 1])
    _run(M, 128, 256, 2, 2, 16, [0, M], [2])  # there is no such adapter
    _run(M, 128, 256, 2, 2, 16, [0], [])
    _run(M, 128, 256, 2, 2, 16, [0, M], [-(1 << 31)], bias=False, scaled=False)


@pytest.mark.parametrize("pad,shift", [(3, 0), (8, 0), (0, 1)])
@pytest.mark.parametrize("M", [20, 300])
def test_strides_and_alignments(pad, shift, M):
    rng = np.random.default_rng(0)
    K, N, R = 128, 256, 16
    if not shift:
        return _run(M, K, N, 2, 2, R, [0, M // 2, M], [1, 0], pad=pad)
    x, w, b0, a, b = _inputs(rng, M, K, N, 1, 2, R)

    def moved(t):
        raw = torch.empty(t.numel() + shift, dtype=t.dtype, device="cuda")
        raw[shift:].copy_(t.flatten())
        return raw[shift:].view(t.shape)

    d = mssa.adapter_project_desc(M, K, N, 2, 2, R)
    ws = torch.empty(mssa.mssa_adapter_project_workspace_size(d), dtype=torch.uint8, device="cuda")
    seg, which = ints([0, M // 2, M]), ints([1, 0])
    outs = []
    for f in (lambda t: t, moved):
        y = f(torch.empty(M, N, dtype=torch.bfloat16, device="cuda"))
        mssa.mssa_adapter_project(d, x, w, f(b0), seg, which, a, f(b), None, ws, [y])
        outs.append(f64(y))
    ref, mag, low = paged.adapter_project(f64(x), f64(w), f64(b0), [0, M // 2, M], [1, 0], f64(a), f64(b), None, 1, 1.0)
    for got in outs:
        assert (np.abs(got - ref[0]) <= 2.0 ** -8 * 1.01 * np.abs(ref[0]) + (K + R) * 2.0 ** -23 * (mag[0] + low[0]) + 2.0 ** -8 * low[0]).all()


@pytest.mark.parametrize("M", [1, 20, 33, 64, 70])
@pytest.mark.parametrize("K", [1, 3, 7, 8, 9, 15, 16, 23, 31, 33, 63, 65, 95, 577, 1537])
@pytest.mark.parametrize("pad", [0, 1, 2, 9])
def test_rows_of_odd_lengths(M, K, pad):
    """Rows end anywhere and begin at any value; what stands between them is not used."""
    def between(x, w, a, b):
        if pad:
            x._base[:, K:] = float("nan")

    _run(M, K, 50, 2, 3, 12, [0, M // 3, M // 3, M], [2, 1, 0], pad=pad, edit=between)


@pytest.mark.parametrize("bad", [np.inf, np.nan])
@pytest.mark.parametrize("M,K,N,R", [(12, 128, 192, 16), (300, 128, 768, 16), (300, 100, 90, 5), (600, 128, 768, 8)])
def test_an_adapters_infinities_stay_with_its_rows(bad, M, K, N, R):
    begin, which = [0, M // 3, M // 2, M], [0, 1, 2]

    def edit(x, w, a, b):
        a[1, 0, 0, 0] = bad
        b[1, :, R - 1] = bad

    got = np.concatenate(_run(M, K, N, 3, 3, R, begin, which, edit=edit, check=False), 1)
    rows = np.isfinite(got).all(1)
    assert rows[: M // 3].all() and rows[M // 2:].all() and not rows[M // 3: M // 2].any()

    def one_part(x, w, a, b):
        a[1, 1] = bad

    ys = _run(M, K, N, 3, 3, R, begin, which, edit=one_part, check=False)
    assert np.isfinite(ys[0]).all() and np.isfinite(ys[2]).all() and np.isfinite(ys[1][: M // 3]).all()
    assert not np.isfinite(ys[1][M // 3: M // 2]).any()


@pytest.mark.parametrize("M", [9, 300])
def test_repeatable_on_another_stream_and_in_a_graph(M):
    rng = np.random.default_rng(4)
    K, N, R, J = 256, 768, 16, 3
    x, w, b0, a, b = _inputs(rng, M, K, N, 3, J, R)
    d = mssa.adapter_project_desc(M, K, N, 3, J, R, parts=3)
    begin, which = ints([0, M // 3, M // 2, M]), ints([2, 0, 1])

    def buffers():
        return (torch.empty(mssa.mssa_adapter_project_workspace_size(d), dtype=torch.uint8, device="cuda"),
                [torch.empty(M, N // 3, dtype=torch.bfloat16, device="cuda") for _ in range(3)])

    one, two = buffers(), buffers()
    call = lambda s, **kw: mssa.mssa_adapter_project(d, x, w, b0, begin, which, a, b, None, *s, **kw)  # noqa: E731
    call(one)
    torch.cuda.synchronize()
    call(two, stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(one[1], two[1]))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(two)
    for step in range(3):
        which.copy_(ints([[2, 0, 1], [1, -1, 0], [0, 0, 2]][step]))
        g.replay()
        call(one)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(one[1], two[1]))


@pytest.mark.parametrize("K", [8, 40, 64, 72, 128, 136, 200, 333])
@pytest.mark.parametrize("M,N,parts,R,S", [(90, 200, 1, 8, 2), (300, 1029, 3, 20, 9), (1300, 1728, 3, 72, 3), (1290, 1730, 1, 12, 30)])
def test_waves_that_share_out_the_contraction(M, K, N, parts, R, S):
    """Odd and even numbers of stages, one group without any; tiles of both small sizes."""
    rng = np.random.default_rng(K)
    _run(M, K, N, parts, 3, R, _cuts(rng, M, S), rng.integers(-1, 3, size=S))


@pytest.mark.parametrize("M,K,N,parts,R,S", [(4200, 72, 4104, 1, 8, 3), (4097, 136, 4608, 3, 40, 2), (5000, 64, 3700, 2, 12, 5),
                                             (4500, 192, 3900, 3, 70, 4), (4300, 8, 4096, 1, 24, 40), (4200, 100, 2000, 1, 8, 3), (4500, 97, 4100, 2, 16, 3), (9000, 131, 768, 3, 40, 2),
                                             (9000, 456, 768, 3, 100, 2), (2100, 328, 2050, 1, 16, 700)])
def test_large_tiles(M, K, N, parts, R, S):
    rng = np.random.default_rng(M)
    _run(M, K, N, parts, 3, R, _cuts(rng, M, S), rng.integers(-1, 3, size=S), factor=1.7)
