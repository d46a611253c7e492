"""Attention over a paged cache against the fp64 oracle.

Bounds: bf16 products are exact, sums fp32; P is rounded to bf16 (2^-8 of each
term, so 2^-8 of the softmax mean of |v|) and the output once more (2^-8 of
itself), the scores' fp32 rounding adds below 1e-4 of that mean.  The log sum is
fp32: scores of size up to 30 to 2e-6 relative, 1e-4 absolute."""

import numpy as np
import pytest
import torch

from oracle import paged
from paper_2607_20940_amd import mssa

from lowbit_common import Banded, cuda, f64
from paged_common import Cache, begins, ints

pytestmark = pytest.mark.gpu


def _run(new, before, H, KH, D, page, mask=0, prior=False, first=0, behind=0, pad=0, lse_pad=0, amp=1.0, seed=0, scale=0.0,
         even=False, alias=False, edit=None, max_chunk=None, lens=None, table_pages=None, check=True):
    """Chunks of new[b] tokens whose sequences hold before[b] tokens before them."""
    rng = np.random.default_rng(seed + sum(new) * 7 + sum(before) + D)
    kv = [n + p for n, p in zip(new, before)] if lens is None else lens
    cache = Cache(rng, kv, page, KH, D, amp=amp, table_pages=table_pages)
    if edit:
        edit(cache)
    cache.device()
    begin = begins(new, first)
    tokens = int(begin[-1]) + behind
    wide = cuda(rng.normal(size=(tokens, H * D + pad)) * amp, "bf16")
    q = wide[:, : H * D]
    st = tokens + lse_pad
    out, lse = Banded((tokens, H, D), torch.bfloat16, 7.0), Banded((H, st), torch.float32, -7.0)
    po = pl = pr = None
    if prior:
        po = cuda(rng.normal(size=(tokens, H, D)), "bf16")
        pl_np = np.full((H, st), -5.0, dtype=np.float32)
        pl_np[:, :tokens] = rng.normal(size=(H, tokens)) + np.log(max(kv) + 1)
        pl_np[0, first] = -np.inf
        pl = torch.from_numpy(pl_np).cuda()
        pr = (f64(po), pl_np.astype(np.float64))
        if alias:
            out.t.copy_(po)
            lse.t.copy_(pl)
            po, pl = out.t, lse.t
    d = mssa.paged_attention_desc(tokens, len(new), max_chunk or max(1, *new), H, KH, D, page, cache.pages, cache.table_pages,
                                  mask_block=mask, softmax_scale=scale, q_stride=H * D + pad, lse_stride=st)
    ws = Banded((mssa.mssa_paged_attention_workspace_size(d),), torch.uint8, 0xff)
    mssa.mssa_paged_attention(d, q, cache.dk, cache.dv, None if even else ints(begin), ints(kv), cache.dt, po, pl, ws.t, out.t,
                              lse.t)
    torch.cuda.synchronize()
    assert out.intact() and lse.intact() and ws.intact()
    if not check:
        return out.t, lse.t, cache, q.reshape(tokens, H, D), begin, kv
    ref, ref_lse, mag = paged.attention(f64(q).reshape(tokens, H, D), cache.k, cache.v, None if even else begin, kv, cache.table,
                                        scale if scale > 0 else D ** -0.5, mask, pr)
    got, got_lse = f64(out.t), f64(lse.t)
    mine = ~np.isnan(ref_lse)
    rows = np.zeros(tokens, dtype=bool)
    rows[int(begin[0]):int(begin[-1])] = True
    if not prior or not alias:
        assert (got[~rows] == 7.0).all() and (got_lse[:, :tokens][:, ~rows] == -7.0).all()
    assert (got_lse[:, tokens:] == (-5.0 if alias else -7.0)).all()
    got, ref, mag = got[rows], ref[rows], mag[rows]
    err = np.abs(got - ref)
    assert (err <= 2.0 ** -8 * 1.02 * np.abs(ref) + (2.0 ** -8 * 1.02 + 1e-4) * mag + 1e-30).all(), err.max()
    got_lse, ref_lse = got_lse[:, :tokens][mine], ref_lse[mine]
    gone = np.isneginf(ref_lse)
    assert np.array_equal(np.isneginf(got_lse), gone)
    assert (np.abs(got_lse[~gone] - ref_lse[~gone]) <= 1e-4).all()
    return out.t, lse.t


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,H,KH", [(1, 1, 1), (1, 10, 2), (3, 8, 8), (11, 6, 2), (33, 2, 2), (70, 3, 1), (129, 4, 2), (300, 2, 1)])
@pytest.mark.parametrize("before", [0, 1, 63, 200, 1000])
@pytest.mark.parametrize("mask", [0, 1, 40])
def test_sizes(D, n, H, KH, before, mask):
    _run([n], [before], H, KH, D, 16, mask)


@pytest.mark.parametrize("n,group", [(1, 5), (20, 2), (200, 2), (1100, 2)])
@pytest.mark.parametrize("page", [1, 3, 16, 64, 100, 129, 1000])
def test_pages_end_anywhere(page, n, group):
    _run([n], [517], 2 * group if n < 1000 else group, 2 if n < 1000 else 1, 64, page, mask=7)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("mask", [0, 1, 13])
@pytest.mark.parametrize("new,before", [
    ([1] * 9, [0, 1, 63, 64, 65, 700, 5, 2000, 0]), ([3, 0, 1, 17, 0], [10, 20, 0, 900, 0]),
    ([40, 1, 0, 130, 7], [0, 500, 30, 64, 1300]), ([300, 1, 700, 2], [100, 3000, 0, 0]), ([0, 0], [5, 0])])
def test_ragged_batches(D, mask, new, before):
    _run(new, before, 4, 2, D, 16, mask, first=3, behind=5, pad=8, lse_pad=3)


@pytest.mark.parametrize("D,H,mask", [(64, 8, 0), (128, 8, 1), (64, 24, 1)])
def test_many_items_of_few_rows(D, H, mask):
    """1024 items and more: blocks of two waves."""
    rng = np.random.default_rng(D)
    new = rng.integers(0, 4, size=140).tolist()
    _run(new, rng.integers(0, 500, size=140).tolist(), H, 8, D, 32, mask, first=2)


def test_many_sequences():
    rng = np.random.default_rng(5)
    new = rng.integers(0, 3, size=150).tolist()
    _run(new, rng.integers(0, 300, size=150).tolist(), 2, 1, 64, 16, mask=1, first=1)
    new = rng.integers(0, 60, size=70).tolist()
    _run(new, rng.integers(0, 300, size=70).tolist(), 2, 1, 64, 32, mask=2)


@pytest.mark.parametrize("new,before,group", [([1, 1, 1], [5, 900, 64], 3), ([50, 50], [700, 3], 2), ([600], [900], 4)])
def test_even_chunks_without_begins(new, before, group):
    _run(new, before, 2 * group, 2, 128, 64, mask=1, even=True)


@pytest.mark.parametrize("alias", [False, True])
@pytest.mark.parametrize("new,before,KH", [([1, 1], [0, 900], 2), ([90, 20], [1000, 0], 2), ([1200], [2000], 1), ([2, 3], [4000, 60], 2)])
def test_joined_with_an_earlier_result(alias, new, before, KH):
    _run(new, before, 2 * KH, KH, 128, 16, prior=True, alias=alias, lse_pad=2)


@pytest.mark.parametrize("lens", [[0, 3], [-4, 2], [10, 1 << 30], [2, -(1 << 31)]])
@pytest.mark.parametrize("mask", [0, 1, 4])
@pytest.mark.parametrize("n", [5, 60, 1100])
def test_lengths_shorter_than_the_chunk_and_past_the_table(lens, mask, n):
    """A cache shorter than its chunk leaves rows without keys; longer than its table it ends there."""
    rng = np.random.default_rng(1)
    held = [min(max(x, 0), 640) for x in lens]
    cache = Cache(rng, held, 64, 1, 64, table_pages=10).device()
    begin = begins([n, n])
    q = cuda(rng.normal(size=(2 * n, 2, 64)), "bf16")
    out, lse = torch.empty_like(q), torch.empty(2, 2 * n, device="cuda")
    d = mssa.paged_attention_desc(2 * n, 2, n, 2, 1, 64, 64, cache.pages, 10, mask_block=mask)
    ws = torch.empty(mssa.mssa_paged_attention_workspace_size(d) + 16, dtype=torch.uint8, device="cuda")
    mssa.mssa_paged_attention(d, q, cache.dk, cache.dv, ints(begin), ints(lens), cache.dt, None, None, ws, out, lse)
    ref, ref_lse, mag = paged.attention(f64(q), cache.k, cache.v, begin, lens, cache.table, 0.125, mask)
    gone = np.isneginf(ref_lse)
    assert np.array_equal(np.isneginf(f64(lse)), gone) and (f64(out).transpose(1, 0, 2)[gone] == 0).all()
    assert (np.abs(f64(out) - ref) <= 2.0 ** -8 * 1.02 * (np.abs(ref) + mag) + 1e-4 * mag).all()


@pytest.mark.parametrize("n", [1, 40, 300])
def test_entries_that_name_no_page_are_not_there(n):
    def edit(cache):
        cache.table[0, 1], cache.table[0, 3], cache.table[1, 0] = -1, cache.pages, 1 << 30

    _run([n, n], [400, 200], 4, 2, 64, 32, mask=1, edit=edit)


@pytest.mark.parametrize("n", [1, 40, 300])
def test_shared_pages(n):
    def edit(cache):
        cache.table[1, :3] = cache.table[0, :3]

    _run([n, n], [400, 200], 4, 2, 128, 32, edit=edit)


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("D,H", [(64, 2), (128, 2), (128, 6)])
@pytest.mark.parametrize("n,mask", [(9, 1), (30, 4), (70, 1), (300, 1), (300, 50), (1200, 1)])
def test_values_that_a_row_does_not_see_never_reach_it(bad, D, H, n, mask):
    """Infinities and NaN in tokens of the chunk: the rows before them are as if they were not there."""
    KH = 2 if n < 1000 else 1
    H = H if n < 1000 else 2
    late = n - max(2, n // 3)  # chunk token from which on keys and values are bad
    late = late // mask * mask

    def edit(cache):
        for c in range(100 + late, 100 + n, 3):
            p = cache.table[0, c // 16], c % 16
            cache.v[p] = bad
            cache.k[p] = bad if c % 2 else cache.k[p]

    out, lse, cache, q, begin, kv = _run([n], [100], H, KH, D, 16, mask, edit=edit, check=False)
    ref, ref_lse, mag = paged.attention(f64(q)[:late], cache.k, cache.v, [0, late], [100 + late], cache.table, D ** -0.5, mask)
    got = f64(out)
    assert (np.abs(got[:late] - ref) <= 2.0 ** -8 * 1.02 * (np.abs(ref) + mag) + 1e-4 * mag).all()
    assert (np.abs(f64(lse)[:, :late] - ref_lse) <= 1e-4).all()
    if late < n:  # the last row sees a bad value
        assert not np.isfinite(got[n - 1]).all()


def test_single_bad_value_in_one_dim():
    """An infinity in one dim of one token: that dim alone is infinite, for the rows that see it."""
    def edit(cache):
        p = cache.table[0, 150 // 16], 150 % 16
        cache.v[p][0, 5] = np.inf

    for n in (60, 20):
        out, lse, cache, q, *_ = _run([n], [100 + 60 - n], 1, 1, 64, 16, 1, edit=edit, check=False)
        got = f64(out)[:, 0]
        first = 150 - (160 - n)
        assert np.isfinite(got[:first]).all() and np.isposinf(got[first:, 5]).all()
        assert np.isfinite(np.delete(got, 5, 1)).all()


@pytest.mark.parametrize("n,KH", [(1, 2), (50, 2), (1100, 1)])
def test_large_scores_and_scale(n, KH):
    _run([n], [300], 2 * KH, KH, 128, 16, 1, amp=6.0, scale=0.05)


def test_longer_chunks_than_announced():
    out, lse, *_ = _run([9, 3], [50, 60], 2, 1, 64, 16, max_chunk=4, check=False)
    got = f64(out)
    assert (got[4:9] == 7.0).all() and (f64(lse)[:, 4:9] == -7.0).all()
    assert np.isfinite(got).all() and not (got[:4] == 7.0).any() and not (got[9:] == 7.0).any()


@pytest.mark.parametrize("new,before,KH", [([1] * 5, [3000, 10, 700, 0, 65], 8), ([700, 90], [1000, 300], 1), ([1100], [3000], 2)])
def test_repeatable_on_another_stream_and_in_a_graph(new, before, KH):
    rng = np.random.default_rng(2)
    D, H, page = 128, KH * 2, 48
    kv = [n + p for n, p in zip(new, before)]
    cache = Cache(rng, kv, page, KH, D).device()
    T = sum(new)
    q = cuda(rng.normal(size=(T, H, D)), "bf16")
    d = mssa.paged_attention_desc(T, len(new), max(new), H, KH, D, page, cache.pages, cache.table_pages, mask_block=1)
    begin, lens = ints(begins(new)), ints(kv)

    def buffers():
        return (torch.empty(mssa.mssa_paged_attention_workspace_size(d) + 16, dtype=torch.uint8, device="cuda"),
                torch.empty_like(q), torch.empty(H, T, device="cuda"))

    def call(bufs, **kw):
        ws, out, lse = bufs
        mssa.mssa_paged_attention(d, q, cache.dk, cache.dv, begin, lens, cache.dt, None, None, ws, out, lse, **kw)

    a, b, c = buffers(), buffers(), buffers()
    call(a)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(b)
    call(c, stream=side)
    torch.cuda.synchronize()
    for x in (b, c):
        assert torch.equal(a[1], x[1]) and torch.equal(a[2], x[2])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(b)
    for step in range(3):  # lengths change between the replays
        lens.copy_(ints([max(0, n - 17 * step) for n in kv]))
        b[1].fill_(5.0)
        g.replay()
        call(a)
        torch.cuda.synchronize()
        assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])


@pytest.mark.parametrize("n", [1, 300])
def test_pools_whose_offsets_pass_32_bits(n):
    """Pages at the far end of a pool of 5 GiB, which the append fills and the attention reads."""
    rng = np.random.default_rng(n)
    KH, D, page, before = 8, 128, 256, 200
    pages = (5 << 30) // (page * KH * D * 2)
    held = n + before
    used = -(-held // page)
    table = np.arange(pages - used, pages)[None]
    x = [cuda(rng.normal(size=(held, KH * D)), "bf16") for _ in range(2)]
    k_pages, v_pages = (torch.empty(pages, page, KH, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    d = mssa.paged_append_desc(held, 1, 0, KH, D, page, pages, used, rotate_dims=0)
    mssa.mssa_paged_append(d, None, *x, None, ints([held]), ints(table), None, None, None, k_pages, v_pages)
    assert torch.equal(k_pages[pages - used:].view(-1, KH * D)[:held], x[0])
    assert torch.equal(v_pages[pages - used:].view(-1, KH * D)[:held], x[1])
    q = cuda(rng.normal(size=(n, KH, D)), "bf16")
    out, lse = torch.empty_like(q), torch.empty(KH, n, device="cuda")
    d = mssa.paged_attention_desc(n, 1, n, KH, KH, D, page, pages, used, mask_block=1)
    ws = torch.empty(mssa.mssa_paged_attention_workspace_size(d) + 16, dtype=torch.uint8, device="cuda")
    mssa.mssa_paged_attention(d, q, k_pages, v_pages, None, ints([held]), ints(table), None, None, ws, out, lse)
    k, v = (f64(t).reshape(1, held, KH, D) for t in x)
    ref, ref_lse, mag = paged.attention(f64(q), k, v, None, [held], [[0]], D ** -0.5, 1)
    assert (np.abs(f64(out) - ref) <= 2.0 ** -8 * 1.02 * (np.abs(ref) + mag) + 1e-4 * mag).all()
    assert (np.abs(f64(lse) - ref_lse) <= 1e-4).all()
