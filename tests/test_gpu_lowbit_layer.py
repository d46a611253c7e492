"""The streaming layer in low bits, pass by pass over ring wraps: every step
against the fp64 oracle on the step's own inputs, so that each bound is that
step's alone."""

import numpy as np
import pytest
import torch

from oracle import lowbit
from paper_2607_20940_amd import mssa
from paper_2607_20940_amd.lowbit import LowBitStreamingMSSA

from lowbit_common import cuda, f64

pytestmark = pytest.mark.gpu

DESC = dict(num_states=3, scales=[1, 2, 4], grid_h=7, grid_w=9, frames_per_state=2, sink_frames=1, num_heads=2,
            head_dim=64)


def _codes(t):
    return t.cpu().numpy()


def _ring_values(ring, frames):
    n = frames * ring.tokens * ring.heads
    k, v = (lowbit.mx_values(_codes(c)[:n], _codes(s)[:n]).reshape(frames * ring.tokens, ring.heads, ring.head_dim)
            for c, s in (ring.k, ring.v))
    return k, v


@pytest.mark.parametrize("desc,cap,start", [
    (DESC, 5, 3), (DESC, 4, 0), (dict(DESC, head_dim=128, scales=[1, 1, 2], num_heads=3), 6, 6),
    (dict(DESC, resample="stride", frames_per_state=1, sink_frames=0), 2, 1)])
def test_passes(desc, cap, start):
    rng = np.random.default_rng(cap)
    st = LowBitStreamingMSSA(desc, 2, cap, hidden=96)
    W = st.width
    tok1 = desc["grid_h"] * desc["grid_w"]
    S = desc["sink_frames"] * tok1
    layers = []
    for layer in range(2):
        w_norm = cuda(1 + 0.2 * rng.normal(size=96), "bf16")
        w, b = cuda(rng.normal(size=(3 * W, 96)) / np.sqrt(96), "bf16"), cuda(0.1 * rng.normal(size=3 * W), "bf16")
        sink = [cuda(rng.normal(size=(S, st.heads, st.head_dim)), "bf16") if S else None for _ in range(2)]
        hist = [cuda(rng.normal(size=(start * tok1, st.heads, st.head_dim)), "bf16") if start else None for _ in range(2)]
        st.init_layer(layer, w_norm, w, b, *sink, *hist)
        layers.append((w_norm, w, b, sink))
    filled = start
    for p in range(4):
        for layer, (w_norm, w, b, sink) in enumerate(layers):
            x, res = (cuda(rng.normal(size=(st.n_q, 96)), "bf16") for _ in range(2))
            want_sum = (x.float() + res.float()).to(torch.bfloat16)
            out = torch.empty(st.n_q, st.heads, st.head_dim, dtype=torch.bfloat16, device="cuda")
            rings = [_ring_values(r, filled) for r in st.rings[layer]]
            head = st.state[layer].head
            st.layer_pass(layer, x, res, out)
            torch.cuda.synchronize()
            # 1: residual stream and 8-bit rows
            assert torch.equal(res, want_sum)
            y, _ = lowbit.norm(f64(res), f64(w_norm), 1e-6)
            x8 = lowbit.e4m3_value(_codes(st.x8))[:, :96] * f64(st.x8_scale)[:, None]
            top = np.abs(y).max(1, keepdims=True)
            assert (np.abs(x8 - y) <= np.maximum(2.0 ** -4 * np.abs(y), top / 448 * 2.0 ** -10) * (1 + 1e-4)).all()
            # 2: the projection with the weights' MXFP4 values
            wv = lowbit.mx_values(_codes(st.weights[layer][1]), _codes(st.weights[layer][2]))[:, :96]
            assert np.array_equal(wv, lowbit.mx_values(lowbit.mx_pack(lowbit.mx_codes(f64(w))[0]),
                                                       lowbit.mx_codes(f64(w))[1])[:, :96])
            ref = lowbit.project(x8, wv, f64(b), 3, 1.0)
            size = lowbit.project(np.abs(x8), np.abs(wv), None, 3, 1.0)
            for got, r, s in zip((st.q, st.k, st.v), ref, size):
                assert (np.abs(f64(got).reshape(st.n_q, W) - r) <= 2.0 ** -8 * 1.01 * np.abs(r) + 2.0 ** -12 * s).all()
            # 3 and 4: sink and window (the library's result, tested on its own) joined with the rings
            part, lse = torch.empty_like(out), torch.empty_like(st.lse)
            ws = torch.empty_like(st.workspace)
            mssa.mssa_pool_kv(st.plan, None, None, st.k, st.v, ws)
            mssa.mssa_forward_lse(st.plan, st.q, *sink, None, None, st.k, st.v, ws, part, lse)
            torch.cuda.synchronize()
            for g, (k, v) in enumerate(rings):
                a, e = st.info["q_begin"][g], st.info["q_end"][g]
                o, _, mag = lowbit.attention(f64(st.q[a:e])[None], k[None], v[None], st.head_dim ** -0.5, [len(k)],
                                             prior=(f64(part[a:e])[None], f64(lse[:, a:e])[None]))
                assert (np.abs(f64(out[a:e]) - o[0]) <= 2.0 ** -8 * 1.02 * np.abs(o[0]) + (2.0 ** -8 * 1.02 + 1e-4) * mag[0]).all()
            # 5: the head state's frames, native and pooled, in their slots
            for g, r in enumerate(st.rings[layer]):
                s, n = st.info["group_scale"][g], r.tokens * r.heads
                for (codes, scales), native, off in ((r.k, st.k, "pooled_k_offset"), (r.v, st.v, "pooled_v_offset")):
                    raw = (native[: st.F * tok1] if s == 1
                           else ws[st.info[off][g]: st.info[off][g] + st.F * n * st.head_dim * 2].view(torch.bfloat16))
                    want, byte = lowbit.mx_codes(f64(raw).reshape(st.F * n, st.head_dim))
                    for f in range(st.F):
                        at = (head + f) % cap * n
                        if any((head + later) % cap == (head + f) % cap for later in range(f + 1, st.F)):
                            continue  # a ring shorter than the state's frames keeps the last ones
                        assert np.array_equal(_codes(scales)[at: at + n], byte[f * n: (f + 1) * n])
                        got = lowbit.e2m1_value(lowbit.mx_unpack(_codes(codes)[at: at + n]))
                        assert np.array_equal(got, lowbit.e2m1_value(want[f * n: (f + 1) * n]))
        filled = min(cap, filled + st.F)
        assert all(s.count == filled for s in st.state)


def test_wan13b_layer_runs_on_another_stream():
    """The Wan-1.3B layer at its size, on a stream of the caller's, twice with
    the same bytes."""
    from paper_2607_20940_amd.workloads import STREAMING

    desc = STREAMING["layer"]
    outs = []
    for _ in range(2):
        g = torch.Generator(device="cuda").manual_seed(3)

        def rand(*shape, std=1.0):
            return (torch.randn(shape, generator=g, device="cuda") * std).bfloat16()

        st = LowBitStreamingMSSA(desc, 1, 21)
        tok, W = 1560, st.width
        st.init_layer(0, rand(W), rand(3 * W, W, std=W ** -0.5), rand(3 * W, std=0.1), rand(3 * tok, 12, 128), rand(3 * tok, 12, 128),
                      rand(6 * tok, 12, 128), rand(6 * tok, 12, 128))
        x, res = rand(st.n_q, W), rand(st.n_q, W)
        out = torch.empty(st.n_q, 12, 128, dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        for _ in range(2):
            st.layer_pass(0, x, res, out, stream=side)
        side.synchronize()
        assert torch.isfinite(out.float()).all() and float(out.float().square().mean()) > 0
        assert st.state[0].count == 12
        outs.append((out, res, st.rings[0][0].k[0].clone()))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_refusals():
    with pytest.raises(ValueError):
        LowBitStreamingMSSA(dict(DESC, scales=[2, 2, 4]), 1, 4)
    with pytest.raises(ValueError):
        LowBitStreamingMSSA(DESC, 1, 1)
