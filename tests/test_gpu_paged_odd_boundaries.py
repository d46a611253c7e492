"""Boundaries of chunks and segments that are negative, past the rows or decrease: they are clamped, a decreasing one is an
empty chunk, and nothing outside is touched.  Rows of chunks that no other chunk overlaps come out as ever; of rows that
stand in two chunks only the last one's is looked at where it is defined (the append).  The look-ups with such values are
walked on the host by tests/test_paged_odd_boundaries.py.  Bounds as in the operators' own tests."""

import numpy as np
import pytest
import torch

from oracle import paged
from paper_2607_20940_amd import mssa

from lowbit_common import Banded, cuda, f64
from paged_common import Cache, ints

pytestmark = pytest.mark.gpu

# Of n rows: (boundaries, the chunks that they are, rows in two chunks).
ODD = {
    "ends": lambda n: ([-7, n // 3, n // 2, n + 300], [(0, n // 3), (n // 3, n // 2), (n // 2, n)], (0, 0)),
    "far ends": lambda n: ([-(1 << 31), n // 3, n // 2, (1 << 31) - 1], [(0, n // 3), (n // 3, n // 2), (n // 2, n)], (0, 0)),
    "decreasing": lambda n: ([0, n // 2, n // 2 - 3, n], [(0, n // 2), (0, 0), (n // 2 - 3, n)], (n // 2 - 3, n // 2)),
    "decreasing at the end": lambda n: ([2, n // 2, n, -9], [(2, n // 2), (n // 2, n), (0, 0)], (0, 0)),
    "all past the rows": lambda n: ([n + 1, n + 2, 1 << 30, 5], [(0, 0)] * 3, (0, 0)),
}


@pytest.mark.parametrize("kind", sorted(set(ODD) - {"decreasing at the end"}))
@pytest.mark.parametrize("M,K,N,R", [(14, 64, 96, 8), (14, 67, 96, 5), (60, 128, 96, 16), (150, 64, 200, 12), (700, 64, 512, 16)])
def test_segments(kind, M, K, N, R):
    begin, segments, twice = ODD[kind](M)
    rng = np.random.default_rng(M + K)
    x, w = cuda(rng.normal(size=(M, K)), "bf16"), cuda(rng.normal(size=(N, K)) * K ** -0.5, "bf16")
    a, b = cuda(rng.normal(size=(3, 1, R, K)) * K ** -0.5, "bf16"), cuda(rng.normal(size=(3, N, R)), "bf16")
    y = Banded((M, N), torch.bfloat16, 3.0)
    d = mssa.adapter_project_desc(M, K, N, 3, 3, R)
    ws = Banded((mssa.mssa_adapter_project_workspace_size(d),), torch.uint8, 0xff)
    mssa.mssa_adapter_project(d, x, w, None, ints(begin), ints([1, 2, 0]), a, b, None, ws.t, [y.t])
    torch.cuda.synchronize()
    assert ws.intact() and y.intact()
    ref, mag, low = (np.zeros((M, N)) for _ in range(3))
    for (r0, r1), j in zip([(0, M), *segments], (-1, 1, 2, 0)):
        (t,), (m,), (u,) = paged.adapter_project(f64(x)[r0:r1], f64(w), None, [0, r1 - r0], [j], f64(a), f64(b), None, 1, 1.0)
        ref[r0:r1], mag[r0:r1], low[r0:r1] = t, m, u
    once = np.ones(M, dtype=bool)
    once[twice[0]:twice[1]] = False
    tol = 2.0 ** -8 * 1.01 * np.abs(ref) + (K + R + 8) * 2.0 ** -23 * (mag + low) + 2.0 ** -8 * low
    assert (np.abs(f64(y.t) - ref) <= tol)[once].all()


@pytest.mark.parametrize("kind", sorted(ODD))
@pytest.mark.parametrize("n", [13, 90])
def test_append(kind, n):
    H, KH, D, page, pages = 2, 1, 32, 8, 60
    begin, chunks, _ = ODD[kind](n)
    rng = np.random.default_rng(n)
    lens = [100, 60, 95]
    table = rng.permutation(pages)[:45].reshape(3, 15)
    q, k, v = (cuda(rng.normal(size=(n, h, D)), "bf16") for h in (H, KH, KH))
    kp, vp = (Banded((pages, page, KH, D), torch.bfloat16, 3.0) for _ in range(2))
    q_out = Banded((n, H, D), torch.bfloat16, 7.0)
    d = mssa.paged_append_desc(n, 3, H, KH, D, page, pages, 15, rotate_dims=0)
    mssa.mssa_paged_append(d, q, k, v, ints(begin), ints(lens), ints(table), None, None, q_out.t, kp.t, vp.t)
    torch.cuda.synchronize()
    assert kp.intact() and vp.intact() and q_out.intact()
    want_q, want = np.full((n, H, D), 7.0), [np.full((pages, page, KH, D), 3.0) for _ in range(2)]
    owner = {r: b for b, (r0, r1) in enumerate(chunks) for r in range(r0, r1)}  # the last chunk that holds a row
    for r, b in owner.items():
        want_q[r] = f64(q)[r]
        c = lens[b] - (chunks[b][1] - r)
        if 0 <= c < 15 * page:
            for t, src in zip(want, (k, v)):
                t[table[b, c // page], c % page] = f64(src)[r]
    assert np.array_equal(f64(q_out.t), want_q)
    assert np.array_equal(f64(kp.t), want[0]) and np.array_equal(f64(vp.t), want[1])


@pytest.mark.parametrize("kind", sorted(ODD))
@pytest.mark.parametrize("n,H,KH,D,history", [(13, 4, 2, 64, 300), (40, 2, 2, 128, 40), (90, 4, 1, 64, 700), (90, 2, 1, 128, 0)])
@pytest.mark.parametrize("mask", [0, 1, 5])
def test_attention(kind, n, H, KH, D, history, mask):
    begin, chunks, twice = ODD[kind](n)
    rng = np.random.default_rng(n + D)
    lens = [history + (r1 - r0) for r0, r1 in chunks]
    cache = Cache(rng, lens, 16, KH, D).device()
    q = cuda(rng.normal(size=(n, H, D)), "bf16")
    out, lse = Banded((n, H, D), torch.bfloat16, 7.0), Banded((H, n), torch.float32, -7.0)
    d = mssa.paged_attention_desc(n, 3, n, H, KH, D, 16, cache.pages, cache.table_pages, mask_block=mask)
    ws = Banded((mssa.mssa_paged_attention_workspace_size(d),), torch.uint8, 0xff)
    mssa.mssa_paged_attention(d, q, cache.dk, cache.dv, ints(begin), ints(lens), cache.dt, None, None, ws.t, out.t, lse.t)
    torch.cuda.synchronize()
    assert out.intact() and lse.intact() and ws.intact()
    got, got_lse = f64(out.t), f64(lse.t)
    none = np.ones(n, dtype=bool)
    for b, (r0, r1) in enumerate(chunks):
        none[r0:r1] = False
        rows = np.array([r for r in range(r0, r1) if not twice[0] <= r < twice[1]], dtype=int)
        if len(rows) == 0:
            continue
        ref, ref_lse, mag = paged.attention(f64(q)[r0:r1], cache.k, cache.v, [0, r1 - r0], [lens[b]], cache.table[b:b + 1], D ** -0.5, mask)
        at = rows - r0
        tol = 2.0 ** -8 * 1.02 * np.abs(ref[at]) + (2.0 ** -8 * 1.02 + 1e-4) * mag[at] + 1e-30
        assert (np.abs(got[rows] - ref[at]) <= tol).all(), b
        assert (np.abs(got_lse[:, rows] - ref_lse[:, at]) <= 1e-4).all()
    assert (got[none] == 7.0).all() and (got_lse[:, none] == -7.0).all()
