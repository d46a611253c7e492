"""Refusals and sizes of the low-bit entry points (no GPU): every bad call is
rejected with its status before anything is enqueued, with the binding's
exception, and leaves no message behind for good calls to trip over."""

import ctypes

import pytest

from paper_2607_20940_amd import mssa

P = 1 << 20  # a 16-byte aligned address that no accepted call here reads: refusals come first


def _refused(status, call):
    with pytest.raises(mssa.MssaError) as e:
        call()
    assert e.value.status == status, str(e.value)


NORM = dict(rows=4, cols=64, dtype="bf16", out="bf16")
NORM_ARGS = dict(x=P, residual=P * 2, weight=P * 3, sum_out=P * 4, y=P * 5, y_scale=None, rstd=None)


def _norm(desc=None, **args):
    a = dict(NORM_ARGS, **args)
    d = mssa.norm_desc(**dict(NORM, **(desc or {})))
    return lambda: mssa.mssa_add_rms_norm(d, a["x"], a["residual"], a["weight"], a["sum_out"], a["y"], a["y_scale"],
                                          a["rstd"], stream=0)


INV, UNS, WS = mssa.MSSA_ERR_INVALID_ARG, mssa.MSSA_ERR_UNSUPPORTED, mssa.MSSA_ERR_WORKSPACE


@pytest.mark.parametrize("status,desc,args", [
    (INV, dict(rows=-1), {}), (INV, dict(cols=0), {}), (UNS, dict(cols=32769), {}), (INV, dict(dtype="e4m3"), {}),
    (INV, dict(out="f32"), {}), (INV, dict(out="mxfp4"), {}), (INV, dict(eps=-1.0), {}), (INV, dict(eps=float("nan")), {}),
    (INV, dict(x_stride=63), {}), (INV, dict(residual_stride=-64), {}), (INV, dict(sum_stride=1 << 60), {}),
    (INV, {}, dict(x=None)), (INV, {}, dict(weight=None)), (INV, {}, dict(y=None)), (INV, {}, dict(sum_out=None)),
    (INV, {}, dict(residual=None)), (INV, {}, dict(y_scale=P * 6)), (INV, dict(out="e4m3"), {}),
    (INV, dict(out="e4m3"), dict(y=P * 5 + 8, y_scale=P * 6)), (INV, {}, dict(x=P + 1)), (INV, {}, dict(rstd=P + 2)),
    (INV, {}, dict(y=P)), (INV, {}, dict(y=P * 4)), (INV, dict(x_stride=72), dict(sum_out=P)),
    (INV, dict(residual_stride=72), dict(sum_out=P * 2)),
])
def test_norm_refusals(status, desc, args):
    _refused(status, _norm(desc, **args))


@pytest.mark.parametrize("status,desc,args", [
    (INV, dict(cols=0), {}), (INV, {}, dict(sum_in=None)), (INV, {}, dict(dx=None)), (INV, {}, dict(rstd=None)),
    (INV, {}, dict(dweight=None)), (INV, {}, dict(dx=P)), (INV, {}, dict(dy=P * 4 + 1)),
    (WS, dict(rows=4000), dict(workspace_bytes=16)), (WS, dict(rows=4000), dict(workspace=None)),
    (INV, dict(rows=4000), dict(workspace=P * 7 + 8)),
])
def test_norm_backward_refusals(status, desc, args):
    a = dict(dict(sum_in=P, weight=P * 2, rstd=P * 3, dy=P * 4, dsum=P * 5, workspace=P * 7, dx=P * 8, dweight=P * 9,
                  workspace_bytes=1 << 30), **args)
    d = mssa.norm_desc(**dict(NORM, **desc))
    _refused(status, lambda: mssa.mssa_add_rms_norm_backward(
        d, a["sum_in"], a["weight"], a["rstd"], a["dy"], a["dsum"], a["workspace"], a["dx"], a["dweight"],
        workspace_bytes=a["workspace_bytes"], stream=0))


@pytest.mark.parametrize("fn", [mssa.mssa_mx_quantize, mssa.mssa_mx_dequantize])
@pytest.mark.parametrize("status,args", [
    (INV, dict(rows=-1)), (INV, dict(cols=0)), (INV, dict(cols=(1 << 20) + 1)), (INV, dict(dtype="e4m3")),
    (INV, dict(values=None)), (INV, dict(codes=None)), (INV, dict(scales=None)), (INV, dict(values=P + 1)),
    (INV, dict(codes=P + 2)), (INV, dict(stride=63)), (UNS, dict(rows=1 << 36)),
])
def test_mx_conversion_refusals(fn, status, args):
    a = dict(dict(rows=4, cols=64, dtype="bf16", values=P, codes=P * 2, scales=P * 3, stride=0), **args)
    tensors = ((a["values"], a["codes"], a["scales"]) if fn is mssa.mssa_mx_quantize
               else (a["codes"], a["scales"], a["values"]))
    _refused(status, lambda: fn(a["rows"], a["cols"], a["dtype"], *tensors, a["stride"], stream=0))


@pytest.mark.parametrize("status,desc,args", [
    (INV, dict(rows=-1), {}), (INV, dict(rows=(1 << 30) + 1), {}), (INV, dict(in_features=0), {}),
    (INV, dict(out_features=0), {}), (INV, dict(out_features=(1 << 20) + 1), {}), (INV, dict(parts=0), {}),
    (INV, dict(parts=9, out_features=9), {}), (INV, dict(parts=5), {}), (INV, dict(x_format="bf16"), {}),
    (INV, dict(out="e4m3"), {}), (INV, dict(part0_scale=float("inf")), {}), (INV, {}, dict(x=None)),
    (INV, {}, dict(x_scales=None)), (INV, {}, dict(w=None)), (INV, {}, dict(w_scales=P * 4 + 4)),
    (INV, {}, dict(bias=P * 5 + 2)), (INV, {}, dict(y=[None] * 3)), (INV, {}, dict(y=[P * 6, P * 7, P * 8 + 4])),
    (INV, {}, dict(y=[P * 6, P, P * 8])),
])
def test_project_refusals(status, desc, args):
    d = dict(dict(rows=4, in_features=64, out_features=96, parts=3, x_format="e4m3", out="bf16"), **desc)
    a = dict(dict(x=P, x_scales=P * 2, w=P * 3, w_scales=P * 4, bias=P * 5, y=[P * 6, P * 7, P * 8]), **args)
    pd = mssa.mx_project_desc(**d)
    y = (a["y"] * 3)[: max(0, d["parts"])]
    _refused(status, lambda: mssa.mssa_mx_project(pd, a["x"], a["x_scales"], a["w"], a["w_scales"], a["bias"], y, stream=0))


def test_project_wants_one_output_per_part():
    with pytest.raises(ValueError):
        mssa.mssa_mx_project(mssa.mx_project_desc(4, 64, 96, parts=3), P, P, P, P, None, [P * 6], stream=0)


ATT = dict(batch=2, n_q=1, q_heads=4, kv_heads=2, head_dim=128, cache_tokens=4096)


@pytest.mark.parametrize("status,desc,args", [
    (INV, dict(batch=0), {}), (INV, dict(n_q=0), {}), (INV, dict(kv_heads=0), {}), (INV, dict(kv_heads=3), {}),
    (UNS, dict(head_dim=96), {}), (INV, dict(cache_tokens=0), {}), (INV, dict(cache_tokens=1 << 31), {}),
    (INV, dict(n_q=8, lse_stride=7), {}), (INV, dict(softmax_scale=float("nan")), {}),
    (UNS, dict(n_q=1 << 30, q_heads=2, kv_heads=1), {}), (UNS, dict(batch=1 << 30), {}),
    (INV, {}, dict(q=None)), (INV, {}, dict(k_codes=None)), (INV, {}, dict(v_scales=None)), (INV, {}, dict(out=None)),
    (INV, {}, dict(prior_out=P * 6)), (INV, {}, dict(prior_lse=P * 6)), (INV, {}, dict(v_codes=P * 4 + 8)),
    (INV, {}, dict(kv_len=P + 2)), (INV, {}, dict(lse=P + 1)), (INV, {}, dict(out=P)),
    (WS, {}, dict(workspace=None)), (WS, {}, dict(workspace_bytes=16)), (INV, {}, dict(workspace=P * 8 + 4)),
])
def test_attention_refusals(status, desc, args):
    a = dict(dict(q=P, k_codes=P * 2, k_scales=P * 3, v_codes=P * 4, v_scales=P * 5, kv_len=None, prior_out=None,
                  prior_lse=None, workspace=P * 8, out=P * 9, lse=None, workspace_bytes=1 << 40), **args)
    d = mssa.mx_attention_desc(**dict(ATT, **desc))
    _refused(status, lambda: mssa.mssa_mx_attention(
        d, a["q"], a["k_codes"], a["k_scales"], a["v_codes"], a["v_scales"], a["kv_len"], a["prior_out"],
        a["prior_lse"], a["workspace"], a["out"], a["lse"], workspace_bytes=a["workspace_bytes"], stream=0))


def test_null_descriptors():
    n = ctypes.c_int64()
    assert mssa.lib.mssa_add_rms_norm(*[None] * 9) == INV
    assert mssa.lib.mssa_add_rms_norm_workspace_size(None, ctypes.byref(n)) == INV
    assert mssa.lib.mssa_add_rms_norm_workspace_size(ctypes.byref(mssa.norm_desc(4, 64)), None) == INV
    assert mssa.lib.mssa_mx_project(*[None] * 8) == INV
    assert mssa.lib.mssa_mx_attention_workspace_size(None, ctypes.byref(n)) == INV
    assert mssa.lib.mssa_mx_attention_workspace_size(ctypes.byref(mssa.mx_attention_desc(**ATT)), None) == INV


def test_unknown_type_names():
    with pytest.raises(ValueError):
        mssa.norm_desc(1, 1, dtype="fp16")


def test_calls_without_rows_enqueue_nothing():
    mssa.mssa_add_rms_norm(mssa.norm_desc(0, 64), None, None, None, None, None, stream=0)
    mssa.mssa_mx_quantize(0, 64, "bf16", None, None, None, stream=0)
    mssa.mssa_mx_dequantize(0, 64, "f32", None, None, None, stream=0)
    mssa.mssa_mx_project(mssa.mx_project_desc(0, 64, 64), None, None, None, None, None, [None], stream=0)


@pytest.mark.parametrize("rows,cols", [(0, 64), (1, 1), (4, 64), (100, 1536), (27840, 5120), (1 << 40, 32768)])
def test_norm_workspace_is_bounded(rows, cols):
    n = mssa.mssa_add_rms_norm_workspace_size(mssa.norm_desc(rows, cols))
    assert 0 <= n <= 2048 * cols * 4


@pytest.mark.parametrize("n_q,tokens", [(1, 1), (1, 32760), (33, 2000), (9360, 32760), (1, (1 << 31) - 1)])
def test_attention_workspace_is_bounded(n_q, tokens):
    n = mssa.mssa_mx_attention_workspace_size(mssa.mx_attention_desc(2, n_q, 12, 12, 128, tokens))
    rows = 2 * 12 * n_q
    assert 0 <= n <= 256 * rows * 130 * 4
    assert mssa.mx_shapes(7, 33) == ((7, 32), (7, 2))


@pytest.mark.parametrize("kv_heads,ok", [(1 << 16, True), ((1 << 16) + 1, False), (1 << 26, False)])
def test_key_heads_whose_tiles_pass_32_bit_offsets_are_refused(kv_heads, ok):
    desc = mssa.mx_attention_desc(1, 1, kv_heads, kv_heads, 128, 64)
    if ok:
        assert mssa.mssa_mx_attention_workspace_size(desc) >= 0
    else:
        with pytest.raises(mssa.MssaError, match="key heads"):
            mssa.mssa_mx_attention_workspace_size(desc)
