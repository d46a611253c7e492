"""LowBitStreamingMSSA's checks of its tensors (no GPU: library calls are
recorded, not made): a tensor of another type is never read as bf16."""

import pytest
import torch

from paper_2607_20940_amd import lowbit, mssa

DESC = dict(num_states=2, scales=[1, 2], grid_h=3, grid_w=4, frames_per_state=1, sink_frames=1, num_heads=2, head_dim=64)
HIDDEN, W, TOK = 96, 128, 12


@pytest.fixture
def layer(monkeypatch):
    calls = []
    for name in ("mssa_mx_quantize", "mssa_pool_hist_ring", "mssa_add_rms_norm", "mssa_mx_project", "mssa_pool_kv",
                 "mssa_forward_lse", "mssa_mx_attention"):
        monkeypatch.setattr(mssa, name, lambda *a, _n=name, **k: calls.append((_n, a)))
    st = lowbit.LowBitStreamingMSSA(DESC, 1, 4, hidden=HIDDEN, device="cpu")
    return st, calls


def _tensors(**other):
    t = dict(norm_weight=torch.ones(HIDDEN), w_qkv=torch.ones(3 * W, HIDDEN), b_qkv=torch.ones(3 * W),
             k_sink=torch.ones(TOK, 2, 64), v_sink=torch.ones(TOK, 2, 64), k_hist=torch.ones(2 * TOK, 2, 64),
             v_hist=torch.ones(2 * TOK, 2, 64))
    return {**{k: v.bfloat16() for k, v in t.items()}, **other}


def test_bf16_tensors_and_absent_ones_are_taken(layer):
    st, calls = layer
    st.init_layer(0, **_tensors())
    assert calls[0][1][2] == "bf16" and st.state[0].count == 2
    st.init_layer(0, **_tensors(b_qkv=None, k_sink=None, v_sink=None, k_hist=None, v_hist=None))
    assert st.state[0].count == 0


def test_fp32_product_weights_are_quantised_as_fp32(layer):
    st, calls = layer
    w = torch.randn(3 * W, HIDDEN)
    st.init_layer(0, **_tensors(w_qkv=w))
    name, args = calls[0]
    assert name == "mssa_mx_quantize" and args[:3] == (3 * W, HIDDEN, "f32") and args[3] is w


# fp32 product weights are taken, and a history that ends inside a frame counts its whole frames
@pytest.mark.parametrize("name,how", [
    (n, h) for n in ("norm_weight", "w_qkv", "b_qkv", "k_sink", "v_sink", "k_hist", "v_hist")
    for h in ("f32", "f16", "strided", "short") if (n, h) not in (("w_qkv", "f32"), ("k_hist", "short"))])
def test_init_refuses_what_it_would_misread(layer, name, how):
    st, calls = layer
    good = _tensors()[name]
    bad = {"f32": good.float(), "f16": good.half(), "short": good[: len(good) - 1].contiguous(),
           "strided": torch.ones((*good.shape[:-1], 2 * good.shape[-1]), dtype=torch.bfloat16)[..., ::2]}[how]
    with pytest.raises(ValueError, match=name):
        st.init_layer(0, **_tensors(**{name: bad}))
    assert not calls and st.weights[0] is None


@pytest.mark.parametrize("name", ["x", "residual", "out"])
@pytest.mark.parametrize("how", ["f32", "strided", "short"])
def test_pass_refuses_what_it_would_misread(layer, name, how):
    st, calls = layer
    st.init_layer(0, **_tensors())
    del calls[:]
    t = dict(x=torch.ones(st.n_q, HIDDEN), residual=torch.ones(st.n_q, HIDDEN), out=torch.ones(st.n_q, 2, 64))
    t = {k: v.bfloat16() for k, v in t.items()}
    good = t[name]
    t[name] = {"f32": good.float(), "short": good[1:],
               "strided": torch.ones((*good.shape[:-1], 2 * good.shape[-1]), dtype=torch.bfloat16)[..., ::2]}[how]
    with pytest.raises(ValueError, match=name):
        st.layer_pass(0, **t, stream=0)
    assert not calls and st.state[0].count == 2


def test_pass_takes_bf16_tensors(layer):
    st, calls = layer
    st.init_layer(0, **_tensors())
    st.layer_pass(0, torch.ones(st.n_q, HIDDEN).bfloat16(), torch.ones(st.n_q, HIDDEN).bfloat16(),
                  torch.ones(st.n_q, 2, 64).bfloat16(), stream=0)
    assert st.state[0].count == 3
