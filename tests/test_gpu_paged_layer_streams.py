"""Layers over a paged cache on a stream other than the one their buffers were made on, and beside another attention."""

import numpy as np
import pytest
import torch

from oracle import mssa_oracle, paged
from paper_2607_20940_amd import mssa
from paper_2607_20940_amd.paged import PagedStreams

from lowbit_common import cuda, f64
from paged_common import Cache, ints

pytestmark = pytest.mark.gpu
HIDDEN, H, KH, D, PAGE = 192, 4, 2, 64, 16


def _layers(rng):
    p = PagedStreams(2, HIDDEN, H, KH, D, 40, PAGE, 20, 64, 4, adapters=2, rank=16,
                     freqs=cuda(rng.uniform(size=D // 2), "f32"))
    width = (H + 2 * KH) * D
    for layer in range(2):
        p.init_layer(layer, cuda(rng.normal(size=(width, HIDDEN)) * 0.05, "bf16"), cuda(rng.normal(size=width) * 0.1, "bf16"),
                     cuda(rng.normal(size=(2, 16, HIDDEN)) * 0.1, "bf16"), cuda(rng.normal(size=(2, width, 16)) * 0.1, "bf16"),
                     cuda(rng.uniform(0.5, 1.5, size=2), "f32"))
    for s in range(3):
        p.open(s, s - 1)
    return p


def test_buffers_outlive_the_object_until_another_stream_is_done():
    """The layers, given up while another stream has their passes still to run: no new tensor takes their memory before."""
    x = cuda(np.random.default_rng(1).normal(size=(63, HIDDEN)), "bf16")
    outs = []
    for other in (False, True):
        p = _layers(np.random.default_rng(2))
        p.begin([(0, 40), (1, 3), (2, 20)])
        out = torch.zeros(2, 63, H, D, dtype=torch.bfloat16, device="cuda")
        sizes = [t.numel() * t.element_size() for t in (p.qkv, p.q, p.freqs, *p.k_pages, *p.v_pages, *p.weights[0], *p.weights[1])]
        side = torch.cuda.Stream() if other else torch.cuda.current_stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            if other:
                torch.cuda._sleep(200_000_000)
            for layer in range(2):
                p.layer_pass(layer, x, out[layer])
        del p
        if other:
            taken = [torch.full((n,), 0x7f, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(3)]
        torch.cuda.synchronize()
        outs.append(out)
    assert len(taken) > 0 and torch.equal(outs[0], outs[1])


@pytest.mark.parametrize("page", [16, 60, 100])
def test_history_in_pages_joined_with_a_plans_sink_and_window(page):
    """mssa_forward_lse's result over sink and window as the prior of the attention over the pages, in place: the attention
    over all three.  The prior's bits are taken as they are, so the bounds are those of the attention over pages alone; the
    whole is within the plan's own tolerance for bf16 (2e-2, 2e-3 in the mean)."""
    rng = np.random.default_rng(page)
    desc = dict(num_states=2, scales=[1, 1], grid_h=6, grid_w=10, frames_per_state=1, sink_frames=1, hist_frames=0, num_heads=H,
                head_dim=D, dtype="bf16")
    plan = mssa.mssa_plan_create(desc)
    n, held = 120, 3 * 60
    q, kw, vw, ks, vs, kh, vh = (cuda(rng.normal(size=(m, H, D)), "bf16") for m in (n, n, n, 60, 60, held, held))
    out, lse = torch.empty(n, H, D, dtype=torch.bfloat16, device="cuda"), torch.empty(H, n, device="cuda")
    ws = torch.empty(max(256, plan.info()["workspace_bytes"]), dtype=torch.uint8, device="cuda")
    mssa.mssa_pool_kv(plan, None, None, kw, vw, ws)
    mssa.mssa_forward_lse(plan, q, ks, vs, None, None, kw, vw, ws, out, lse)
    torch.cuda.synchronize()
    prior = f64(out), f64(lse)
    cache = Cache(rng, [held], page, H, D)
    for c in range(held):
        cache.k[cache.table[0, c // page], c % page], cache.v[cache.table[0, c // page], c % page] = f64(kh)[c], f64(vh)[c]
    cache.device()
    d = mssa.paged_attention_desc(n, 1, n, H, H, D, page, cache.pages, cache.table_pages)
    pws = torch.empty(max(256, mssa.mssa_paged_attention_workspace_size(d)), dtype=torch.uint8, device="cuda")
    mssa.mssa_paged_attention(d, q, cache.dk, cache.dv, None, ints([held]), cache.dt, out, lse, pws, out, lse)
    torch.cuda.synchronize()
    ref, ref_lse, mag = paged.attention(f64(q), cache.k, cache.v, None, [held], cache.table, D ** -0.5, 0, prior)
    assert (np.abs(f64(out) - ref) <= 2.0 ** -8 * 1.02 * np.abs(ref) + (2.0 ** -8 * 1.02 + 1e-4) * mag).all()
    assert np.abs(f64(lse) - ref_lse).max() <= 1e-4
    whole = mssa_oracle.mssa_attention(dict(desc, hist_frames=3), *(f64(t) for t in (q, ks, vs, kh, vh, kw, vw)))
    err = np.abs(f64(out) - whole)
    assert err.max() <= 2e-2 and err.mean() <= 2e-3


def test_another_current_device_is_refused(monkeypatch):
    """Kernels go to the current device: the layers' tensors have to be on it."""
    p = _layers(np.random.default_rng(3))
    p.begin([(0, 5)])
    x, out = cuda(np.ones((5, HIDDEN)), "bf16"), torch.full((5, H, D), 7.0, dtype=torch.bfloat16, device="cuda")
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_device", lambda: 1)
        for stream in (None, torch.cuda.default_stream(0)):
            with pytest.raises(ValueError):
                p.layer_pass(0, x, out, stream=stream)
    torch.cuda.synchronize()
    assert (out == 7).all() and all((t == 0).all() for t in (*p.k_pages, *p.v_pages))
    p.layer_pass(0, x, out)
    torch.cuda.synchronize()
    assert not (out == 7).all()
