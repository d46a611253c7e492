"""Append to a paged cache with rotation, against the fp64 oracle.

Bounds: cosine and sine in fp32 of an angle whose fraction of a turn is exact to
2^-25 (2 pi 2^-25 + 2 units of 2^-24), two products and a sum in fp32: below 1e-6
of |u| + |v|; then one rounding to bf16 (2^-8).  Values are copied: exact."""

import numpy as np
import pytest
import torch

from oracle import paged
from paper_2607_20940_amd import mssa

from lowbit_common import Banded, cuda, f64
from paged_common import begins, ints

pytestmark = pytest.mark.gpu


def _run(new, kv, H, KH, D, page, axis_pairs=None, turned=None, halves=False, first=0, behind=0, pad=0, positions=None, edit=None,
         even=False, in_place=False, theta=10000.0, stream=None, spare=1):
    rng = np.random.default_rng(sum(new) + D + page)
    turned = D if turned is None else turned
    split = [turned // 2] if axis_pairs is None else axis_pairs
    begin = begins(new, first)
    tokens = int(begin[-1]) + behind
    used = [-(-max(0, n) // page) for n in kv]
    pages = sum(used) + spare
    table = np.full((len(new), max(1, *used)), -1, dtype=np.int64)
    order, at = rng.permutation(pages), 0
    for b, u in enumerate(used):
        table[b, :u] = order[at:at + u]
        at += u
    if edit:
        edit(table, pages)
    mk = lambda h: cuda(rng.normal(size=(tokens, h * D + pad)), "bf16")[:, : h * D]  # noqa: E731
    q, k, v = mk(H) if H else None, mk(KH), mk(KH)
    freqs = np.concatenate([theta ** (-np.arange(p) / max(1, p)) for p in split]).astype(np.float32)
    pos = None if positions is None else positions(tokens, len(split))
    kp, vp = (Banded((pages, page, KH, D), torch.bfloat16, 3.0) for _ in range(2))
    q_out = Banded((tokens, max(1, H), D), torch.bfloat16, 7.0)
    if in_place:
        q_out.t.copy_(q.reshape(tokens, H, D))
        q0, q = q, q_out.t
    d = mssa.paged_append_desc(tokens, len(new), H, KH, D, page, pages, table.shape[1], rotate_dims=turned, halves=halves,
                               axis_pairs=axis_pairs, q_stride=0 if in_place else H * D + pad, k_stride=KH * D + pad,
                               v_stride=KH * D + pad)
    mssa.mssa_paged_append(d, q, k, v, None if even else ints(begin), ints(kv), ints(table), None if pos is None else ints(pos),
                           torch.from_numpy(freqs).cuda(), q_out.t if H else None, kp.t, vp.t, stream=stream)
    torch.cuda.synchronize()
    assert kp.intact() and vp.intact() and q_out.intact()
    if in_place:
        q = q0
    index, place = paged.places(None if even else begin, kv, table, page, pages, tokens)
    axis = np.repeat(np.arange(len(split)), split)
    at = np.array([0 if i is None else i for i in index])
    where = np.repeat(at[:, None], len(axis), 1) if pos is None else pos.T[:, axis]
    angle = where.astype(np.float64) * freqs.astype(np.float64)
    mine = np.array([i is not None for i in index], dtype=bool)

    def near(got, x, rows):
        ref, mag = paged.rotate(x, angle, halves)
        assert (np.abs(got - ref[rows]) <= 2.0 ** -8 * np.abs(ref[rows]) * 1.001 + 1e-6 * mag[rows] + 1e-38).all()

    if H:
        got = f64(q_out.t)
        near(got[mine], f64(q).reshape(tokens, H, D), mine)
        if not in_place:
            assert (got[~mine] == 7.0).all()
    gk, gv = f64(kp.t), f64(vp.t)
    stored = np.array([p is not None for p in place], dtype=bool)
    if stored.any():
        pg, off = np.array([p for p in place if p is not None]).T
        near(gk[pg, off], f64(k).reshape(tokens, KH, D), stored)
        assert np.array_equal(gv[pg, off], f64(v).reshape(tokens, KH, D)[stored])
        gk[pg, off] = gv[pg, off] = 3.0
    assert (gk == 3.0).all() and (gv == 3.0).all()


def _grid(tokens, axes):
    t = np.arange(tokens)
    return np.stack((t // 50, t // 10 % 5, t % 10))[:axes]


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("D", [16, 64, 112, 128, 256])
@pytest.mark.parametrize("new,kv,H,KH", [([1], [1], 1, 1), ([1, 1, 1], [5, 64, 700], 10, 2), ([37, 0, 90], [37, 40, 200], 4, 4),
                                         ([700], [1000], 3, 1), ([5, 6], [5, 6], 0, 2)])
def test_sizes(halves, D, new, kv, H, KH):
    _run(new, kv, H, KH, D, 16, halves=halves, first=2, behind=3, pad=8)


@pytest.mark.parametrize("page", [1, 7, 64, 1560])
def test_pages(page):
    _run([130, 3], [1700, 900], 4, 2, 64, page)


@pytest.mark.parametrize("halves,turned", [(False, 0), (False, 2), (False, 30), (False, 64), (True, 0), (True, 16), (True, 48), (True, 96)])
def test_part_of_a_head_is_turned(halves, turned):
    _run([9, 40], [50, 40], 4, 2, 128, 16, turned=turned, halves=halves)


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("split", [[22, 21, 21], [40, 24], [0, 64, 0], [64, 0, 0]])
def test_axes(halves, split):
    _run([60, 7], [80, 7], 4, 2, 128, 16, axis_pairs=split, halves=halves, positions=_grid)


@pytest.mark.parametrize("top", [1 << 20, (1 << 31) - 1, -(1 << 31)])
def test_far_positions(top):
    _run([40], [40], 2, 1, 128, 16, axis_pairs=[64], positions=lambda t, x: top - np.sign(top) * np.arange(t)[None] * 12345)


def test_many_sequences_and_tokens():
    rng = np.random.default_rng(3)
    for n in (150, 5000):
        new = rng.integers(0, 3, size=n)
        _run(new.tolist(), (new + rng.integers(0, 9, size=n)).tolist(), 2, 1, 64, 4, first=1)
    _run([20000], [20000], 2, 1, 16, 64)


def test_even_chunks_in_place():
    _run([4, 4, 4], [10, 4, 100], 6, 2, 64, 16, even=True)
    _run([4, 4, 4], [10, 4, 100], 6, 2, 64, 16, in_place=True)


def test_tokens_without_a_place_are_not_stored():
    def edit(table, pages):
        table[0, 1], table[1, 0] = -1, pages

    _run([60, 30], [80, 40], 4, 2, 64, 16, edit=edit)
    _run([10, 10, 4], [6, -3, 0], 4, 2, 64, 16)  # caches shorter than their chunks

    def cut(table, pages):
        table[:, 2:] = -7

    _run([60, 30], [80, 40], 4, 2, 64, 16, edit=cut)


def test_past_the_table():
    """Cache indices that the table has no entries for."""
    T, D = 40, 64
    x = cuda(np.random.default_rng(0).normal(size=(T, D)), "bf16")
    kp, vp = (Banded((2, 16, 1, D), torch.bfloat16, 3.0) for _ in range(2))
    d = mssa.paged_append_desc(T, 1, 0, 1, D, 16, 2, 2, rotate_dims=0)
    mssa.mssa_paged_append(d, None, x, x, None, ints([T]), ints([[1, 0]]), None, None, None, kp.t, vp.t)
    torch.cuda.synchronize()
    assert kp.intact() and vp.intact()
    assert torch.equal(kp.t[1, :, 0], x[:16]) and torch.equal(vp.t[0, :, 0], x[16:32])


def test_infinities_stay_in_their_pair():
    D = 64
    x = torch.ones(1, D, device="cuda", dtype=torch.bfloat16)
    x[0, 6] = float("inf")
    kp, vp = (torch.zeros(1, 1, 1, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    d = mssa.paged_append_desc(1, 1, 0, 1, D, 1, 1, 1)
    mssa.mssa_paged_append(d, None, x, x, None, ints([1]), ints([[0]]), ints([[3]]), torch.rand(D // 2, device="cuda"), None, kp, vp)
    bad = ~torch.isfinite(kp[0, 0, 0])
    assert set(bad.nonzero().flatten().tolist()) <= {6, 7} and bool(bad[6])
    assert torch.equal(vp[0, 0], x)


def test_graph_with_moving_lengths():
    rng = np.random.default_rng(0)
    D, B = 128, 3
    q, k, v = (cuda(rng.normal(size=(B, h * D)), "bf16") for h in (4, 2, 2))
    freqs = torch.rand(D // 2, device="cuda")
    table, lens = ints(rng.permutation(12).reshape(3, 4)), ints([1, 20, 60])
    d = mssa.paged_append_desc(B, B, 4, 2, D, 16, 12, 4)
    sets = [[torch.zeros(B, 4, D, dtype=torch.bfloat16, device="cuda")] +
            [torch.zeros(12, 16, 2, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2)]
    call = lambda s: mssa.mssa_paged_append(d, q, k, v, None, lens, table, None, freqs, *s)  # noqa: E731
    g = torch.cuda.CUDAGraph()
    call(sets[1])
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        call(sets[0])
    for step in range(3):
        g.replay()
        call(sets[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*sets))
        lens += 1
