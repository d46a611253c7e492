"""Refusals and sizes of the entry points for streams served together (no GPU):
every bad call is rejected with its status before anything is enqueued."""

import ctypes

import pytest

from paper_2607_20940_amd import mssa

P = 1 << 20  # a 16-byte aligned address that no accepted call here reads: refusals come first
INV, UNS, WS = mssa.MSSA_ERR_INVALID_ARG, mssa.MSSA_ERR_UNSUPPORTED, mssa.MSSA_ERR_WORKSPACE


def _refused(status, call):
    with pytest.raises(mssa.MssaError) as e:
        call()
    assert e.value.status == status, str(e.value)


PROJECT = dict(rows=100, in_features=64, out_features=96, segments=2, adapters=3, rank=8, parts=3)


@pytest.mark.parametrize("status,desc,args", [
    (INV, dict(rows=-1), {}), (INV, dict(rows=(1 << 30) + 1), {}), (INV, dict(in_features=0), {}),
    (INV, dict(in_features=(1 << 20) + 1), {}), (INV, dict(out_features=0), {}), (INV, dict(parts=0), {}),
    (INV, dict(parts=9, out_features=9), {}), (INV, dict(parts=5), {}), (INV, dict(segments=-1), {}),
    (INV, dict(segments=(1 << 20) + 1), {}), (INV, dict(adapters=-1), {}), (INV, dict(rank=0), {}), (INV, dict(rank=-2), {}),
    (UNS, dict(rank=257), {}), (INV, dict(part0_scale=float("nan")), {}), (INV, dict(x_stride=63), {}),
    (INV, dict(x_stride=-64), {}), (INV, dict(x_stride=1 << 40), {}),
    (INV, {}, dict(x=None)), (INV, {}, dict(w=None)), (INV, {}, dict(begin=None)), (INV, {}, dict(which=None)),
    (INV, {}, dict(a=None)), (INV, {}, dict(b=None)), (INV, {}, dict(y=[None] * 3)), (INV, {}, dict(x=P + 8)), (INV, {}, dict(w=P + 2)),
    (INV, {}, dict(a=P * 6 + 4)), (INV, {}, dict(b=P * 7 + 1)), (INV, {}, dict(bias=P + 1)), (INV, {}, dict(begin=P + 2)), (INV, {}, dict(which=P + 1)), (INV, {}, dict(scale=P + 2)),
    (INV, {}, dict(y=[P * 20, P * 21, P * 22 + 1])), (INV, {}, dict(y=[P * 20, P, P * 22])),
    (INV, {}, dict(y=[P * 20, P * 6, P * 22])), (WS, {}, dict(workspace=None)), (WS, {}, dict(workspace_bytes=16)),
    (INV, {}, dict(workspace=P * 9 + 4)),
])
def test_project_refusals(status, desc, args):
    d = dict(PROJECT, **desc)
    a = dict(dict(x=P, w=P * 2, bias=P * 3, begin=P * 4, which=P * 5, a=P * 6, b=P * 7, scale=P * 8, workspace=P * 9,
                  workspace_bytes=1 << 40, y=[P * 20, P * 21, P * 22]), **args)
    y = (a["y"] * 3)[: max(0, d["parts"])]
    _refused(status, lambda: mssa.mssa_adapter_project(
        mssa.adapter_project_desc(**d), a["x"], a["w"], a["bias"], a["begin"], a["which"], a["a"], a["b"], a["scale"],
        a["workspace"], y, workspace_bytes=a["workspace_bytes"], stream=0))


def test_project_wants_one_output_per_part():
    with pytest.raises(ValueError):
        mssa.mssa_adapter_project(mssa.adapter_project_desc(**PROJECT), P, P, None, P, P, P, P, None, P, [P * 6], stream=0)


def test_project_wants_outputs_of_their_own():
    for y in ([P * 20, P * 20, P * 22], [P * 20, P * 21, P * 20]):
        _refused(INV, lambda: mssa.mssa_adapter_project(
            mssa.adapter_project_desc(**PROJECT), P, P * 2, P * 3, P * 4, P * 5, P * 6, P * 7, P * 8, P * 9, y,
            workspace_bytes=1 << 40, stream=0))


APPEND = dict(tokens=12, batch=3, q_heads=4, kv_heads=2, head_dim=64, page_tokens=16, pages=9, table_pages=4)


@pytest.mark.parametrize("status,desc,args", [
    (INV, dict(tokens=-1), {}), (INV, dict(tokens=(1 << 30) + 1), {}), (INV, dict(batch=0), {}), (INV, dict(batch=1 << 21), {}),
    (INV, dict(kv_heads=0), {}), (INV, dict(q_heads=-1), {}), (INV, dict(kv_heads=1 << 17), {}), (INV, dict(page_tokens=0), {}),
    (INV, dict(page_tokens=(1 << 20) + 1), {}), (INV, dict(table_pages=0), {}), (INV, dict(pages=0), {}),
    (UNS, dict(table_pages=1 << 27), {}), (UNS, dict(pages=1 << 27), {}), (UNS, dict(head_dim=24), {}), (UNS, dict(head_dim=0), {}),
    (UNS, dict(head_dim=272), {}), (INV, dict(rotate_dims=66), {}), (INV, dict(rotate_dims=-2), {}), (INV, dict(rotate_dims=3), {}),
    (UNS, dict(rotate_dims=24, halves=True), {}), (INV, dict(halves=2), {}), (INV, dict(axis_pairs=[16, 15]), {}),
    (INV, dict(axis_pairs=[33, -1]), {}), (INV, dict(q_stride=255), {}), (INV, dict(q_stride=260), {}), (INV, dict(k_stride=120), {}),
    (INV, dict(v_stride=-128), {}), (INV, dict(v_stride=1 << 30), {}), (INV, dict(tokens=13), {}),
    (INV, {}, dict(q=None)), (INV, {}, dict(q_out=None)), (INV, dict(q_heads=0), {}), (INV, {}, dict(k=None)), (INV, {}, dict(v=None)),
    (INV, {}, dict(kv_len=None)), (INV, {}, dict(table=None)), (INV, {}, dict(freqs=None)), (INV, {}, dict(kp=None)),
    (INV, {}, dict(vp=None)), (INV, dict(axis_pairs=[16, 16]), {}), (INV, {}, dict(q=P + 8)), (INV, {}, dict(vp=P * 10 + 2)),
    (INV, {}, dict(kv_len=P + 2)), (INV, {}, dict(positions=P + 1)), (INV, dict(q_stride=264), dict(q_out=P)),
    (INV, {}, dict(q_out=P * 2)), (INV, {}, dict(vp=P * 9)), (INV, {}, dict(kp=P)), (INV, {}, dict(vp=P * 8)),
])
def test_append_refusals(status, desc, args):
    a = dict(dict(q=P, k=P * 2, v=P * 3, begin=None, kv_len=P * 4, table=P * 5, positions=None, freqs=P * 7, q_out=P * 8, kp=P * 9,
                  vp=P * 10), **args)
    d = mssa.paged_append_desc(**dict(APPEND, **desc))
    _refused(status, lambda: mssa.mssa_paged_append(
        d, a["q"], a["k"], a["v"], a["begin"], a["kv_len"], a["table"], a["positions"], a["freqs"], a["q_out"], a["kp"],
        a["vp"], stream=0))


def test_append_wants_one_to_three_axes():
    for split in ([], [8, 8, 8, 8]):
        with pytest.raises(ValueError):
            mssa.paged_append_desc(**dict(APPEND, axis_pairs=split))


ATTEND = dict(tokens=12, batch=3, max_chunk=4, q_heads=4, kv_heads=2, head_dim=128, page_tokens=16, pages=900, table_pages=256)


@pytest.mark.parametrize("status,desc,args", [
    (INV, dict(tokens=-1), {}), (INV, dict(batch=0), {}), (INV, dict(max_chunk=0), {}), (INV, dict(max_chunk=(1 << 30) + 1), {}),
    (INV, dict(q_heads=0), {}), (INV, dict(q_heads=3), {}), (INV, dict(kv_heads=0), {}), (UNS, dict(head_dim=96), {}),
    (INV, dict(page_tokens=0), {}), (INV, dict(table_pages=0), {}), (INV, dict(pages=-1), {}), (UNS, dict(table_pages=1 << 27), {}),
    (UNS, dict(pages=1 << 27), {}), (INV, dict(mask_block=-1), {}), (INV, dict(q_stride=511), {}), (INV, dict(q_stride=516), {}),
    (INV, dict(lse_stride=11), {}), (INV, dict(softmax_scale=float("inf")), {}), (INV, dict(tokens=13), {}),
    (UNS, dict(tokens=3 << 28, max_chunk=1 << 30, q_heads=8), {}),
    (INV, {}, dict(q=None)), (INV, {}, dict(kp=None)), (INV, {}, dict(vp=None)), (INV, {}, dict(kv_len=None)),
    (INV, {}, dict(table=None)), (INV, {}, dict(out=None)), (INV, {}, dict(prior_out=P * 7)), (INV, {}, dict(prior_lse=P * 7)),
    (INV, {}, dict(q=P + 4)), (INV, {}, dict(kp=P + 8)), (INV, {}, dict(table=P + 1)), (INV, {}, dict(lse=P + 2)),
    (INV, {}, dict(out=P)), (INV, {}, dict(out=P * 2)), (INV, {}, dict(out=P * 3)), (WS, {}, dict(workspace=None)),
    (WS, {}, dict(workspace_bytes=16)), (INV, {}, dict(workspace=P * 8 + 4)),
])
def test_attention_refusals(status, desc, args):
    a = dict(dict(q=P, kp=P * 2, vp=P * 3, begin=None, kv_len=P * 4, table=P * 5, prior_out=None, prior_lse=None, workspace=P * 8,
                  out=P * 9, lse=None, workspace_bytes=1 << 40), **args)
    d = mssa.paged_attention_desc(**dict(ATTEND, **desc))
    _refused(status, lambda: mssa.mssa_paged_attention(
        d, a["q"], a["kp"], a["vp"], a["begin"], a["kv_len"], a["table"], a["prior_out"], a["prior_lse"], a["workspace"], a["out"],
        a["lse"], workspace_bytes=a["workspace_bytes"], stream=0))


def test_null_descriptors():
    n = ctypes.c_int64()
    assert mssa.lib.mssa_adapter_project(*[None] * 10, 0, None, None) == INV
    assert mssa.lib.mssa_adapter_project_workspace_size(None, ctypes.byref(n)) == INV
    assert mssa.lib.mssa_adapter_project_workspace_size(ctypes.byref(mssa.adapter_project_desc(**PROJECT)), None) == INV
    assert mssa.lib.mssa_paged_append(*[None] * 13) == INV
    assert mssa.lib.mssa_paged_attention(*[None] * 10, 0, None, None, None) == INV
    assert mssa.lib.mssa_paged_attention_workspace_size(None, ctypes.byref(n)) == INV
    assert mssa.lib.mssa_paged_attention_workspace_size(ctypes.byref(mssa.paged_attention_desc(**ATTEND)), None) == INV


def test_calls_without_tokens_enqueue_nothing():
    mssa.mssa_adapter_project(mssa.adapter_project_desc(**dict(PROJECT, rows=0)), *[None] * 9, [None] * 3, stream=0)
    mssa.mssa_paged_append(mssa.paged_append_desc(**dict(APPEND, tokens=0)), *[None] * 11, stream=0)
    mssa.mssa_paged_attention(mssa.paged_attention_desc(**dict(ATTEND, tokens=0)), *[None] * 10, stream=0)


@pytest.mark.parametrize("tokens,max_chunk,table_pages", [(1, 1, 1), (16, 1, 600), (9360, 9360, 600), (40000, 20000, 100),
                                                          (1 << 20, 1 << 10, 1 << 11)])
def test_workspaces_are_bounded(tokens, max_chunk, table_pages):
    d = mssa.paged_attention_desc(tokens, 1, max_chunk, 12, 12, 128, 64, 1000, table_pages)
    assert 0 <= mssa.mssa_paged_attention_workspace_size(d) <= 2 * 512 * 256 * 130 * 4
    d = mssa.adapter_project_desc(tokens, 128, 384, 4, 4, 100, parts=3)
    assert 0 < mssa.mssa_adapter_project_workspace_size(d) <= tokens * 3 * 112 * 2 + 256
    assert mssa.mssa_adapter_project_workspace_size(mssa.adapter_project_desc(tokens, 128, 384, 0, 4, 100)) == 0


def test_workspace_of_odd_rows_holds_their_copies():
    even, odd, apart = (mssa.mssa_adapter_project_workspace_size(mssa.adapter_project_desc(300, k, 200, 2, 3, 8, x_stride=x))
                        for k, x in ((104, 0), (97, 0), (104, 107)))
    assert odd - even == (300 + 200 + 3 * 8) * 104 * 2 and apart - even == 300 * 104 * 2
    for rows, size in ((16, 16 * 16 * 2), (17, 768 + (17 + 200 + 3 * 8) * 104 * 2)):  # few are read where they lie
        assert mssa.mssa_adapter_project_workspace_size(mssa.adapter_project_desc(rows, 97, 200, 2, 3, 8)) == size
