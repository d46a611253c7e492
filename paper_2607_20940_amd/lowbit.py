"""A streaming MSSA layer in low bits: activations go through the QKV product
in 8 bits, its weights and the K/V history are held in MXFP4 (4.25 bits a
value), sink and window stay bf16.

One layer pass (``layer_pass``), all on the caller's stream:

1. ``mssa_add_rms_norm``: the previous block's output joins the residual
   stream and the normalised tokens leave as 8-bit rows;
2. ``mssa_mx_project``: q, k, v from the 8-bit tokens and MXFP4 weights;
3. ``mssa_pool_kv`` and ``mssa_forward_lse`` of a plan without history: the
   attention over sink and window, with its log sum;
4. ``mssa_mx_attention`` per query scale: the attention over that scale's
   history ring, joined with step 3's result in place;
5. ``mssa_mx_quantize``: the head state's frames (native, and pooled to each
   coarser scale by step 3) become the newest frames of the rings.

A history frame is quantised once, when it is emitted, at every scale that
reads it; the rings of a Wan-1.3B layer stack (30 layers, 21 frames of 1560
tokens and their 2x2 means) are 2.0 GB instead of 7.5.  The gain is memory: one
of these layers over full rings takes 3.12 ms on an MI355X, 1.91 of it the
history's attention, where the bf16 layer's pass takes 2.70 and its QKV product
0.17.

This module only sequences library calls and owns device buffers (torch
allocations); all arithmetic runs in the library.
"""

from . import mssa


def _bf16(name, t, values):
    """The layer's calls read `values` consecutive bf16 values from t (a tensor; None and addresses pass)."""
    import torch

    if t is None or isinstance(t, int):
        return
    if t.dtype != torch.bfloat16 or not t.is_contiguous() or t.numel() < values:
        raise ValueError(f"{name} must be contiguous bf16 with {values} values at least, not {t.dtype} {tuple(t.shape)}")


class _Ring:
    """K and V of one query scale's history: codes and scales of cap frames."""

    def __init__(self, cap, tokens, heads, head_dim, device):
        import torch

        rows = cap * tokens * heads
        code_shape, scale_shape = mssa.mx_shapes(rows, head_dim)
        self.tokens, self.heads, self.head_dim = tokens, heads, head_dim
        self.k, self.v = ([torch.zeros(s, dtype=torch.uint8, device=device) for s in (code_shape, scale_shape)]
                          for _ in range(2))

    def put(self, slot, frames, k, v, stream):
        """bf16 K and V of `frames` frames (token-major) into slots slot, slot + 1, .."""
        n = self.tokens * self.heads
        for (codes, scales), x in ((self.k, k), (self.v, v)):
            mssa.mssa_mx_quantize(frames * n, self.head_dim, "bf16", x, codes[slot * n:], scales[slot * n:], stream=stream)


class LowBitStreamingMSSA:
    def __init__(self, layer_desc, layers, hist_cap_frames, hidden=None, eps=1e-6, device="cuda"):
        import torch

        self.layers, self.cap, self.device = int(layers), int(hist_cap_frames), device
        self.F = int(layer_desc["frames_per_state"])
        if int(layer_desc["scales"][0]) != 1:
            raise ValueError("the head state must be native: scales[0] == 1")
        if self.cap < self.F:
            raise ValueError("the ring must hold at least one state's frames")
        # the history's attention takes the queries unscaled, and its rings are not the plan's
        flags = int(layer_desc.get("flags", 0) or 0) & mssa.MSSA_PLAN_STRIDED_SUBSAMPLE
        self.desc = dict(layer_desc, hist_frames=0, dtype="bf16", flags=flags, q_prescaled=False)
        self.plan = mssa.mssa_plan_create(self.desc)
        self.info = info = self.plan.info()
        self.heads, self.head_dim = int(layer_desc["num_heads"]), int(layer_desc["head_dim"])
        self.width = self.heads * self.head_dim
        self.hidden = int(hidden or self.width)
        self.n_q = info["n_q"]
        gh, gw = int(layer_desc["grid_h"]), int(layer_desc["grid_w"])
        self.tokens = [-(-gh // s) * -(-gw // s) for s in info["group_scale"]]  # of a frame, per query scale
        self.scale = float(layer_desc.get("softmax_scale", 0.0) or 0.0)

        def buf(*shape, dtype=torch.bfloat16):
            return torch.empty(shape, dtype=dtype, device=device)

        self.norm = mssa.norm_desc(self.n_q, self.hidden, dtype="bf16", out="e4m3", eps=eps)
        self.project = mssa.mx_project_desc(self.n_q, self.hidden, 3 * self.width, parts=3)
        self.x8 = buf(self.n_q, -(-self.hidden // 32) * 32, dtype=torch.uint8)
        self.x8_scale = buf(self.n_q, dtype=torch.float32)
        self.q, self.k, self.v = (buf(self.n_q, self.heads, self.head_dim) for _ in range(3))
        self.lse = buf(self.heads, self.n_q, dtype=torch.float32)
        self.workspace = buf(max(256, info["workspace_bytes"]), dtype=torch.uint8)
        self.attend = [mssa.mx_attention_desc(1, info["q_end"][g] - info["q_begin"][g], self.heads, self.heads,
                                              self.head_dim, self.cap * t, softmax_scale=self.scale,
                                              lse_stride=self.n_q) for g, t in enumerate(self.tokens)]
        size = max(mssa.mssa_mx_attention_workspace_size(d) for d in self.attend)
        self.attend_workspace = buf(max(256, size), dtype=torch.uint8)
        self.rings = [[_Ring(self.cap, t, self.heads, self.head_dim, device) for t in self.tokens]
                      for _ in range(self.layers)]
        self.state = [mssa.Ring(self.cap) for _ in range(self.layers)]
        # tokens that a scale's ring holds with so many frames in it: [frames, scale]
        self.kv_len = torch.tensor([[f * t for t in self.tokens] for f in range(self.cap + 1)], dtype=torch.int32,
                                   device=device)
        self.weights = [None] * self.layers
        self.sink = [(None, None)] * self.layers

    def ring_bytes(self):
        return sum(t.numel() for layer in self.rings for r in layer for t in (*r.k, *r.v))

    def init_layer(self, layer, norm_weight, w_qkv, b_qkv, k_sink=None, v_sink=None, k_hist=None, v_hist=None):
        """Weights (norm_weight [hidden] and b_qkv [3 width] in bf16; w_qkv [3 width, hidden] in bf16 or fp32, quantised
        here, once), sink K/V and initial history (bf16, oldest first) of one layer."""
        import torch

        _bf16("norm_weight", norm_weight, self.hidden)
        _bf16("b_qkv", b_qkv, 3 * self.width)
        for name, t in (("k_sink", k_sink), ("v_sink", v_sink)):
            _bf16(name, t, self.info["n_sink_tok"] * self.width)
        for name, t in (("k_hist", k_hist), ("v_hist", v_hist)):
            _bf16(name, t, 0 if k_hist is None else k_hist.shape[0] * self.width)
        w_type = "bf16"
        if not isinstance(w_qkv, int):
            w_type = {torch.bfloat16: "bf16", torch.float32: "f32"}.get(w_qkv.dtype)
            if w_type is None or not w_qkv.is_contiguous() or w_qkv.numel() < 3 * self.width * self.hidden:
                raise ValueError(f"w_qkv must be contiguous bf16 or fp32 [{3 * self.width}, {self.hidden}], not "
                                 f"{w_qkv.dtype} {tuple(w_qkv.shape)}")
        codes, scales = (torch.empty(s, dtype=torch.uint8, device=self.device)
                         for s in mssa.mx_shapes(3 * self.width, self.hidden))
        mssa.mssa_mx_quantize(3 * self.width, self.hidden, w_type, w_qkv, codes, scales)
        self.weights[layer] = (norm_weight, codes, scales, b_qkv)
        self.sink[layer] = (k_sink, v_sink)
        n = 0 if k_hist is None else k_hist.shape[0] // self.tokens[self.info["group_scale"].index(1)]
        if n > self.cap:
            raise ValueError("initial history longer than the ring")
        if n:
            plan = mssa.mssa_plan_create(dict(self.desc, hist_frames=n,
                                              flags=self.desc["flags"] | mssa.MSSA_PLAN_POOLED_HIST_RING))
            pooled = [[None if s == 1 else torch.empty(n * t, self.heads, self.head_dim, dtype=torch.bfloat16,
                                                       device=self.device)
                       for s, t in zip(self.info["group_scale"], self.tokens)] for _ in range(2)]
            mssa.mssa_pool_hist_ring(plan, k_hist, v_hist, *pooled)
            for g, s in enumerate(self.info["group_scale"]):
                k, v = (k_hist, v_hist) if s == 1 else (pooled[0][g], pooled[1][g])
                self.rings[layer][g].put(0, n, k, v, None)
        self.state[layer] = mssa.Ring(self.cap, count=n, head=n % self.cap)

    def _head_frames(self, g, frame, n):
        """K and V of frames frame .. frame + n - 1 of the head state at group g's scale."""
        if self.info["group_scale"][g] == 1:
            a, b = frame * self.tokens[g], (frame + n) * self.tokens[g]
            return self.k[a:b], self.v[a:b]
        row = self.tokens[g] * self.width * 2
        return [self.workspace[self.info[o][g] + frame * row:] for o in ("pooled_k_offset", "pooled_v_offset")]

    def layer_pass(self, layer, x, residual, out, stream=None):
        """x [n_q, hidden] (the previous block's output) joins residual [n_q, hidden], in place; out [n_q, heads,
        head_dim] is the attention of the pass, all bf16.  The emitted frames enter the rings."""
        for name, t, values in (("x", x, self.hidden), ("residual", residual, self.hidden), ("out", out, self.width)):
            _bf16(name, t, self.n_q * values)
        w_norm, w, w_scales, bias = self.weights[layer]
        mssa.mssa_add_rms_norm(self.norm, x, residual, w_norm, residual, self.x8, self.x8_scale, stream=stream)
        mssa.mssa_mx_project(self.project, self.x8, self.x8_scale, w, w_scales, bias, [self.q, self.k, self.v],
                             stream=stream)
        mssa.mssa_pool_kv(self.plan, None, None, self.k, self.v, self.workspace, stream=stream)
        k_sink, v_sink = self.sink[layer]
        mssa.mssa_forward_lse(self.plan, self.q, k_sink, v_sink, None, None, self.k, self.v, self.workspace, out,
                              self.lse, stream=stream)
        state = self.state[layer]
        if state.count:
            for g, d in enumerate(self.attend):
                a, b = self.info["q_begin"][g], self.info["q_end"][g]
                r, o, lse = self.rings[layer][g], out[a:b], self.lse[:, a:]
                mssa.mssa_mx_attention(d, self.q[a:b], *r.k, *r.v, self.kv_len[state.count, g:], o, lse, self.attend_workspace,
                                       o, lse, stream=stream)
        # the head state's frames to slots head, head + 1, .. (in runs up to the ring's end)
        frame = 0
        while frame < self.F:
            slot = (state.head + frame) % self.cap
            n = min(self.F - frame, self.cap - slot)
            for g, r in enumerate(self.rings[layer]):
                r.put(slot, n, *self._head_frames(g, frame, n), stream)
            frame += n
        state.head = (state.head + self.F) % self.cap
        state.count = min(self.cap, state.count + self.F)
