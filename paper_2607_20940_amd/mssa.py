"""ctypes binding of libmssa (include/libmssa.h): argument marshalling only.

Every step of the path runs in the library's HIP kernels; this module turns
tensors into device pointers and the current torch stream into a hipStream_t.
Importing it loads ``libmssa.so`` from this package directory and raises
ImportError if it has not been built (``python -m paper_2607_20940_amd.build``).
There is no fallback implementation.
"""

import ctypes
import os

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmssa.so")

MSSA_MAX_STATES = 8
MSSA_OK, MSSA_ERR_INVALID_ARG, MSSA_ERR_UNSUPPORTED = 0, 1, 2
MSSA_ERR_WORKSPACE, MSSA_ERR_DEVICE, MSSA_ERR_NO_MEMORY = 3, 4, 5
MSSA_BF16, MSSA_F32 = 0, 1
MSSA_E4M3, MSSA_MXFP4 = 2, 3
MSSA_PLAN_POOLED_HIST_RING = 1
MSSA_PLAN_STRIDED_SUBSAMPLE = 2
MSSA_PLAN_HEAD_IN_RING = 4
MSSA_PLAN_Q_PRESCALED = 8

# Every symbol include/libmssa.h declares.
EXPORTS = ("mssa_plan_create", "mssa_plan_create_ex", "mssa_plan_destroy", "mssa_plan_query", "mssa_plan_tables",
           "mssa_pool_kv", "mssa_forward", "mssa_hist_append", "mssa_pool_hist_ring",
           "mssa_forward_ring", "mssa_hist_append_ring", "mssa_forward_lse", "mssa_backward_workspace_size",
           "mssa_backward", "mssa_tier_workspace_size", "mssa_patch_embed", "mssa_patch_unembed",
           "mssa_qkv_project", "mssa_qkv_project_scaled", "mssa_attention_noalloc", "mssa_pool_kv_head_ring", "mssa_forward_head_ring",
           "mssa_head_ring_roll", "mssa_add_rms_norm", "mssa_add_rms_norm_workspace_size",
           "mssa_add_rms_norm_backward", "mssa_mx_quantize", "mssa_mx_dequantize", "mssa_mx_project",
           "mssa_mx_attention_workspace_size", "mssa_mx_attention", "mssa_adapter_project_workspace_size",
           "mssa_adapter_project", "mssa_paged_append", "mssa_paged_attention_workspace_size", "mssa_paged_attention",
           "mssa_status_string", "mssa_last_error")

MSSA_NOALLOC_SCRATCH_BYTES = 256 << 20


class mssa_tier_desc(ctypes.Structure):
    _fields_ = [("latent_channels", ctypes.c_int32), ("patch", ctypes.c_int32), ("hidden", ctypes.c_int32)]


class mssa_norm_desc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("out_dtype", ctypes.c_int32), ("eps", ctypes.c_float), ("x_stride", ctypes.c_int64),
                ("residual_stride", ctypes.c_int64), ("sum_stride", ctypes.c_int64)]


class mssa_mx_project_desc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("in_features", ctypes.c_int32), ("out_features", ctypes.c_int32),
                ("parts", ctypes.c_int32), ("x_format", ctypes.c_int32), ("out_dtype", ctypes.c_int32),
                ("part0_scale", ctypes.c_float)]


class mssa_mx_attention_desc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q", ctypes.c_int32), ("q_heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("cache_tokens", ctypes.c_int64),
                ("lse_stride", ctypes.c_int64), ("softmax_scale", ctypes.c_float)]


class mssa_adapter_project_desc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("in_features", ctypes.c_int32), ("out_features", ctypes.c_int32),
                ("parts", ctypes.c_int32), ("segments", ctypes.c_int32), ("adapters", ctypes.c_int32),
                ("rank", ctypes.c_int32), ("part0_scale", ctypes.c_float), ("x_stride", ctypes.c_int64)]


class mssa_paged_append_desc(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("batch", ctypes.c_int32), ("q_heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("page_tokens", ctypes.c_int32),
                ("table_pages", ctypes.c_int32), ("pages", ctypes.c_int64), ("rotate_dims", ctypes.c_int32),
                ("halves", ctypes.c_int32), ("axes", ctypes.c_int32), ("axis_pairs", ctypes.c_int32 * 3),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64)]


class mssa_paged_attention_desc(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("batch", ctypes.c_int32), ("max_chunk", ctypes.c_int32),
                ("q_heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_tokens", ctypes.c_int32), ("table_pages", ctypes.c_int32), ("pages", ctypes.c_int64),
                ("mask_block", ctypes.c_int32), ("q_stride", ctypes.c_int64), ("lse_stride", ctypes.c_int64),
                ("softmax_scale", ctypes.c_float)]


class mssa_plan_desc(ctypes.Structure):
    _fields_ = [("num_states", ctypes.c_int32), ("scales", ctypes.c_int32 * MSSA_MAX_STATES),
                ("grid_h", ctypes.c_int32), ("grid_w", ctypes.c_int32),
                ("frames_per_state", ctypes.c_int32), ("sink_frames", ctypes.c_int32),
                ("hist_frames", ctypes.c_int32), ("num_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float), ("flags", ctypes.c_int32)]


_I32S = ctypes.c_int32 * MSSA_MAX_STATES
_I64S = ctypes.c_int64 * MSSA_MAX_STATES


class mssa_plan_info(ctypes.Structure):
    _fields_ = [("n_q", ctypes.c_int64), ("n_sink_tok", ctypes.c_int64),
                ("n_hist_tok", ctypes.c_int64), ("workspace_bytes", ctypes.c_int64),
                ("pairs_per_head", ctypes.c_int64), ("flops_alg", ctypes.c_int64),
                ("pool_bytes_alg", ctypes.c_int64), ("n_groups", ctypes.c_int32),
                ("group_scale", _I32S), ("q_begin", _I32S), ("q_end", _I32S),
                ("n_kv", _I64S), ("pooled_k_offset", _I64S), ("pooled_v_offset", _I64S),
                ("pooled_tokens", _I64S)]


def _load():
    # torch ships its own HIP runtime with the same soname as ROCm's
    # (libamdhip64.so.7).  Loading torch first makes libmssa bind to that one
    # runtime; a second runtime in the process would see no device.
    import torch  # noqa: F401

    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2607_20940_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    P, V, I64 = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64
    lib.mssa_plan_create.argtypes = [ctypes.POINTER(mssa_plan_desc), ctypes.POINTER(P)]
    lib.mssa_plan_create_ex.argtypes = [ctypes.POINTER(mssa_plan_desc), ctypes.c_int32, ctypes.POINTER(P)]
    lib.mssa_plan_destroy.argtypes = [P]
    lib.mssa_plan_destroy.restype = None
    lib.mssa_plan_query.argtypes = [P, ctypes.POINTER(mssa_plan_info)]
    lib.mssa_plan_tables.argtypes = [P, ctypes.POINTER(I64), I64, ctypes.POINTER(I64)]
    lib.mssa_pool_kv.argtypes = [P, V, V, V, V, V, I64, V]
    lib.mssa_forward.argtypes = [P, V, V, V, V, V, V, V, V, I64, V, V]
    lib.mssa_hist_append.argtypes = [P, V, V, V, V, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32),
                                     ctypes.POINTER(ctypes.c_int32), V]
    PP = ctypes.POINTER(ctypes.c_void_p)
    lib.mssa_pool_hist_ring.argtypes = [P, V, V, PP, PP, V]
    lib.mssa_forward_ring.argtypes = [P, V, V, V, V, V, PP, PP, V, V, V, I64, V, V]
    lib.mssa_hist_append_ring.argtypes = [P, V, V, V, I64, V, V, PP, PP, ctypes.c_int32,
                                          ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32), V]
    lib.mssa_forward_lse.argtypes = [P, V, V, V, V, V, V, V, V, I64, V, V, V]
    lib.mssa_attention_noalloc.argtypes = [P, V, V, V, V, V, V, V, V, V]
    I32 = ctypes.c_int32
    lib.mssa_pool_kv_head_ring.argtypes = [P, V, V, V, V, PP, PP, V, I64, I32, I32, I32, V]
    lib.mssa_forward_head_ring.argtypes = [P, V, V, V, V, V, PP, PP, V, V, V, I64, V, I32, I32, I32, V]
    lib.mssa_head_ring_roll.argtypes = [P, I32, ctypes.POINTER(I32), ctypes.POINTER(I32)]
    lib.mssa_backward_workspace_size.argtypes = [P, ctypes.POINTER(I64)]
    lib.mssa_backward.argtypes = [P, V, V, V, V, V, V, V, V, V, V, V, I64, V, V, V, V, V, V, V, V]
    TD = ctypes.POINTER(mssa_tier_desc)
    lib.mssa_tier_workspace_size.argtypes = [P, TD, ctypes.POINTER(I64)]
    lib.mssa_patch_embed.argtypes = [P, TD, V, PP, PP, V, I64, V, V]
    lib.mssa_patch_unembed.argtypes = [P, TD, V, PP, PP, V, I64, V, V]
    lib.mssa_qkv_project.argtypes = [I64, ctypes.c_int32, V, V, V, V, V, V, V]
    lib.mssa_qkv_project_scaled.argtypes = [I64, ctypes.c_int32, V, V, V, ctypes.c_float, V, V, V, V]
    ND, PD, AD = (ctypes.POINTER(t) for t in (mssa_norm_desc, mssa_mx_project_desc, mssa_mx_attention_desc))
    lib.mssa_add_rms_norm.argtypes = [ND, V, V, V, V, V, V, V, V]
    lib.mssa_add_rms_norm_workspace_size.argtypes = [ND, ctypes.POINTER(I64)]
    lib.mssa_add_rms_norm_backward.argtypes = [ND, V, V, V, V, V, V, I64, V, V, V]
    lib.mssa_mx_quantize.argtypes = [I64, I32, I32, V, I64, V, V, V]
    lib.mssa_mx_dequantize.argtypes = [I64, I32, I32, V, V, V, I64, V]
    lib.mssa_mx_project.argtypes = [PD, V, V, V, V, V, PP, V]
    lib.mssa_mx_attention_workspace_size.argtypes = [AD, ctypes.POINTER(I64)]
    lib.mssa_mx_attention.argtypes = [AD, V, V, V, V, V, V, V, V, V, I64, V, V, V]
    APD, PPD, PAD = (ctypes.POINTER(t) for t in (mssa_adapter_project_desc, mssa_paged_append_desc,
                                                 mssa_paged_attention_desc))
    lib.mssa_adapter_project_workspace_size.argtypes = [APD, ctypes.POINTER(I64)]
    lib.mssa_adapter_project.argtypes = [APD, V, V, V, V, V, V, V, V, V, I64, PP, V]
    lib.mssa_paged_append.argtypes = [PPD, V, V, V, V, V, V, V, V, V, V, V, V]
    lib.mssa_paged_attention_workspace_size.argtypes = [PAD, ctypes.POINTER(I64)]
    lib.mssa_paged_attention.argtypes = [PAD, V, V, V, V, V, V, V, V, V, I64, V, V, V]
    lib.mssa_status_string.argtypes = [ctypes.c_int]
    lib.mssa_status_string.restype = ctypes.c_char_p
    lib.mssa_last_error.argtypes = []
    lib.mssa_last_error.restype = ctypes.c_char_p
    for name in ("mssa_plan_create", "mssa_plan_create_ex", "mssa_plan_query", "mssa_plan_tables", "mssa_pool_kv",
                 "mssa_forward", "mssa_hist_append", "mssa_pool_hist_ring", "mssa_forward_ring",
                 "mssa_hist_append_ring"):
        getattr(lib, name).restype = ctypes.c_int
    runtimes = _loaded_hip_runtimes()
    if len(runtimes) > 1:
        raise ImportError(f"two HIP runtimes are loaded ({sorted(runtimes)}); libmssa would not see "
                          "the device torch uses")
    return lib


def _loaded_hip_runtimes():
    paths = set()
    try:
        with open("/proc/self/maps") as f:
            for line in f:
                if "libamdhip64" in line:
                    paths.add(os.path.realpath(line.split()[-1]))
    except OSError:
        pass
    return paths


lib = _load()


class MssaError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        name = lib.mssa_status_string(status).decode()
        detail = lib.mssa_last_error().decode()
        super().__init__(f"{where}: {name}: {detail}")


def _check(status, where):
    if status != MSSA_OK:
        raise MssaError(status, where)


def _ptr(x):
    """Device pointer of a tensor (or an int address); None -> NULL."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _nbytes(x):
    if x is None:
        return 0
    return x.numel() * x.element_size()


def _current_stream():
    """hipStream_t of torch's current stream.  torch.cuda.current_stream()
    builds a Stream object (2.9 us, as much as a launch); where this torch
    hands out the handle itself, that is taken (0.3 us)."""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        return torch.cuda.current_stream().cuda_stream
    return raw(torch.cuda.current_device())


def _stream(stream):
    if stream is not None:
        return stream if isinstance(stream, int) else stream.cuda_stream
    return _current_stream()


class Plan:
    """Owning handle of an mssa_plan (released when garbage collected)."""

    def __init__(self, handle, desc):
        self._h = handle
        self.desc = dict(desc)

    @property
    def handle(self):
        return self._h

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        # at interpreter exit the module globals may already be gone
        if h and lib is not None:
            lib.mssa_plan_destroy(h)

    def info(self):
        return mssa_plan_query(self)

    def tables(self):
        return mssa_plan_tables(self)


def make_desc(desc):
    """dict (oracle-style keys, plus optional dtype 'bf16'/'f32') -> struct."""
    d = mssa_plan_desc()
    d.num_states = int(desc["num_states"])
    sc = list(desc["scales"])[:MSSA_MAX_STATES]
    for i, s in enumerate(sc):
        d.scales[i] = int(s)
    d.grid_h, d.grid_w = int(desc["grid_h"]), int(desc["grid_w"])
    d.frames_per_state = int(desc["frames_per_state"])
    d.sink_frames, d.hist_frames = int(desc["sink_frames"]), int(desc["hist_frames"])
    d.num_heads, d.head_dim = int(desc["num_heads"]), int(desc["head_dim"])
    dt = desc.get("dtype", "bf16")
    d.dtype = MSSA_BF16 if dt in ("bf16", MSSA_BF16) else MSSA_F32 if dt in ("f32", MSSA_F32) else int(dt)
    d.softmax_scale = float(desc.get("softmax_scale", 0.0) or 0.0)
    d.flags = int(desc.get("flags", 0) or 0)
    resample = desc.get("resample", "mean")
    if resample not in ("mean", "stride"):
        raise ValueError("resample must be 'mean' or 'stride'")
    if resample == "stride":
        d.flags |= MSSA_PLAN_STRIDED_SUBSAMPLE
    if desc.get("q_prescaled"):
        d.flags |= MSSA_PLAN_Q_PRESCALED
    return d


def mssa_plan_create(desc):
    h = ctypes.c_void_p()
    d = make_desc(desc)
    _check(lib.mssa_plan_create(ctypes.byref(d), ctypes.byref(h)), "mssa_plan_create")
    return Plan(h.value, desc)


def mssa_plan_create_ex(desc, attention_blocks):
    h = ctypes.c_void_p()
    d = make_desc(desc)
    _check(lib.mssa_plan_create_ex(ctypes.byref(d), int(attention_blocks), ctypes.byref(h)), "mssa_plan_create_ex")
    return Plan(h.value, desc)


def mssa_plan_query(plan):
    info = mssa_plan_info()
    _check(lib.mssa_plan_query(plan.handle, ctypes.byref(info)), "mssa_plan_query")
    G = info.n_groups
    return dict(
        n_q=info.n_q, n_sink_tok=info.n_sink_tok, n_hist_tok=info.n_hist_tok,
        workspace_bytes=info.workspace_bytes, pairs_per_head=info.pairs_per_head,
        flops_alg=info.flops_alg, pool_bytes_alg=info.pool_bytes_alg, n_groups=G,
        group_scale=list(info.group_scale[:G]), q_begin=list(info.q_begin[:G]),
        q_end=list(info.q_end[:G]), n_kv=list(info.n_kv[:G]),
        pooled_k_offset=list(info.pooled_k_offset[:G]),
        pooled_v_offset=list(info.pooled_v_offset[:G]),
        pooled_tokens=list(info.pooled_tokens[:G]))


def mssa_plan_tables(plan):
    need = ctypes.c_int64()
    lib.mssa_plan_tables(plan.handle, None, 0, ctypes.byref(need))
    buf = (ctypes.c_int64 * need.value)()
    _check(lib.mssa_plan_tables(plan.handle, buf, need.value, ctypes.byref(need)), "mssa_plan_tables")
    t = np.frombuffer(buf, dtype=np.int64).copy()
    ng, nq, ns = int(t[0]), int(t[1]), int(t[2])
    o = 3
    GRID = t[o: o + 4 * ng].reshape(ng, 4)
    o += 4 * ng
    QGRP = t[o: o + 4 * nq].reshape(nq, 4)
    o += 4 * nq
    SEG = t[o: o + 8 * ns].reshape(ns, 8)
    o += 8 * ns
    return {"GRID": GRID, "QGRP": QGRP, "SEG": SEG, "TOTAL": t[o: o + 2]}


def mssa_pool_kv(plan, k_hist, v_hist, k_win, v_win, workspace, workspace_bytes=None, stream=None):
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    _check(lib.mssa_pool_kv(plan.handle, _ptr(k_hist), _ptr(v_hist), _ptr(k_win), _ptr(v_win),
                            _ptr(workspace), wb, _stream(stream)), "mssa_pool_kv")


def mssa_forward(plan, q_win, k_sink, v_sink, k_hist, v_hist, k_win, v_win, workspace, out,
                 workspace_bytes=None, stream=None):
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    _check(lib.mssa_forward(plan.handle, _ptr(q_win), _ptr(k_sink), _ptr(v_sink), _ptr(k_hist),
                            _ptr(v_hist), _ptr(k_win), _ptr(v_win), _ptr(workspace), wb,
                            _ptr(out), _stream(stream)), "mssa_forward")


def mssa_forward_lse(plan, q_win, k_sink, v_sink, k_hist, v_hist, k_win, v_win, workspace, out, lse,
                     workspace_bytes=None, stream=None):
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    _check(lib.mssa_forward_lse(plan.handle, _ptr(q_win), _ptr(k_sink), _ptr(v_sink), _ptr(k_hist),
                                _ptr(v_hist), _ptr(k_win), _ptr(v_win), _ptr(workspace), wb,
                                _ptr(out), _ptr(lse), _stream(stream)), "mssa_forward_lse")


def mssa_attention_noalloc(plan, q_win, k_sink, v_sink, k_hist, v_hist, k_win, v_win, out, stream=None):
    _check(lib.mssa_attention_noalloc(plan.handle, _ptr(q_win), _ptr(k_sink), _ptr(v_sink), _ptr(k_hist),
                                      _ptr(v_hist), _ptr(k_win), _ptr(v_win), _ptr(out), _stream(stream)),
           "mssa_attention_noalloc")


def mssa_backward_workspace_size(plan):
    n = ctypes.c_int64()
    _check(lib.mssa_backward_workspace_size(plan.handle, ctypes.byref(n)), "mssa_backward_workspace_size")
    return n.value


def mssa_backward(plan, q_win, k_sink, v_sink, k_hist, v_hist, k_win, v_win, out, lse, d_out, workspace,
                  dq_win, dk_sink, dv_sink, dk_hist, dv_hist, dk_win, dv_win, workspace_bytes=None,
                  stream=None):
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    _check(lib.mssa_backward(plan.handle, _ptr(q_win), _ptr(k_sink), _ptr(v_sink), _ptr(k_hist),
                             _ptr(v_hist), _ptr(k_win), _ptr(v_win), _ptr(out), _ptr(lse), _ptr(d_out),
                             _ptr(workspace), wb, _ptr(dq_win), _ptr(dk_sink), _ptr(dv_sink),
                             _ptr(dk_hist), _ptr(dv_hist), _ptr(dk_win), _ptr(dv_win), _stream(stream)),
           "mssa_backward")


def tier_desc(latent_channels, patch, hidden):
    return mssa_tier_desc(int(latent_channels), int(patch), int(hidden))


def mssa_tier_workspace_size(plan, tier):
    n = ctypes.c_int64()
    _check(lib.mssa_tier_workspace_size(plan.handle, ctypes.byref(tier), ctypes.byref(n)),
           "mssa_tier_workspace_size")
    return n.value


def mssa_patch_embed(plan, tier, latent, w_embed, b_embed, workspace, tokens, workspace_bytes=None, stream=None):
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    _check(lib.mssa_patch_embed(plan.handle, ctypes.byref(tier), _ptr(latent), _ptr_array(w_embed),
                                _ptr_array(b_embed), _ptr(workspace), wb, _ptr(tokens), _stream(stream)),
           "mssa_patch_embed")


def mssa_patch_unembed(plan, tier, tokens, w_out, b_out, workspace, latent, workspace_bytes=None, stream=None):
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    _check(lib.mssa_patch_unembed(plan.handle, ctypes.byref(tier), _ptr(tokens), _ptr_array(w_out),
                                  _ptr_array(b_out), _ptr(workspace), wb, _ptr(latent), _stream(stream)),
           "mssa_patch_unembed")


def mssa_qkv_project(n_tokens, hidden, x, w_qkv, b_qkv, q, k, v, stream=None):
    _check(lib.mssa_qkv_project(int(n_tokens), int(hidden), _ptr(x), _ptr(w_qkv), _ptr(b_qkv), _ptr(q), _ptr(k),
                                _ptr(v), _stream(stream)), "mssa_qkv_project")


def mssa_qkv_project_scaled(n_tokens, hidden, x, w_qkv, b_qkv, q_scale, q, k, v, stream=None):
    _check(lib.mssa_qkv_project_scaled(int(n_tokens), int(hidden), _ptr(x), _ptr(w_qkv), _ptr(b_qkv),
                                       float(q_scale), _ptr(q), _ptr(k), _ptr(v), _stream(stream)),
           "mssa_qkv_project_scaled")


_DTYPES = {"bf16": MSSA_BF16, "f32": MSSA_F32, "e4m3": MSSA_E4M3, "mxfp4": MSSA_MXFP4}


def _dtype(name):
    if name in _DTYPES:
        return _DTYPES[name]
    if isinstance(name, int):
        return name
    raise ValueError(f"unknown type {name!r}: one of {sorted(_DTYPES)}")


def norm_desc(rows, cols, dtype="bf16", out=None, eps=1e-6, x_stride=0, residual_stride=0, sum_stride=0):
    """Descriptor of mssa_add_rms_norm and its backward (out: the type of y,
    dtype or "e4m3"; strides in elements between rows, 0 = cols)."""
    return mssa_norm_desc(int(rows), int(cols), _dtype(dtype), _dtype(dtype if out is None else out), float(eps),
                          int(x_stride), int(residual_stride), int(sum_stride))


def mx_project_desc(rows, in_features, out_features, parts=1, x_format="e4m3", out="bf16", part0_scale=1.0):
    return mssa_mx_project_desc(int(rows), int(in_features), int(out_features), int(parts), _dtype(x_format),
                                _dtype(out), float(part0_scale))


def mx_attention_desc(batch, n_q, q_heads, kv_heads, head_dim, cache_tokens, softmax_scale=0.0, lse_stride=0):
    return mssa_mx_attention_desc(int(batch), int(n_q), int(q_heads), int(kv_heads), int(head_dim),
                                  int(cache_tokens), int(lse_stride), float(softmax_scale))


def mx_shapes(rows, cols):
    """Shapes (in bytes) of the codes and scales of `rows` MXFP4 rows of `cols` values."""
    blocks = -(-int(cols) // 32)
    return (int(rows), 16 * blocks), (int(rows), blocks)


def mssa_add_rms_norm(desc, x, residual, weight, sum_out, y, y_scale=None, rstd=None, stream=None):
    _check(lib.mssa_add_rms_norm(ctypes.byref(desc), _ptr(x), _ptr(residual), _ptr(weight), _ptr(sum_out), _ptr(y),
                                 _ptr(y_scale), _ptr(rstd), _stream(stream)), "mssa_add_rms_norm")


def mssa_add_rms_norm_workspace_size(desc):
    n = ctypes.c_int64()
    _check(lib.mssa_add_rms_norm_workspace_size(ctypes.byref(desc), ctypes.byref(n)),
           "mssa_add_rms_norm_workspace_size")
    return n.value


def mssa_add_rms_norm_backward(desc, sum_in, weight, rstd, dy, dsum, workspace, dx, dweight, workspace_bytes=None,
                               stream=None):
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    _check(lib.mssa_add_rms_norm_backward(ctypes.byref(desc), _ptr(sum_in), _ptr(weight), _ptr(rstd), _ptr(dy),
                                          _ptr(dsum), _ptr(workspace), wb, _ptr(dx), _ptr(dweight), _stream(stream)),
           "mssa_add_rms_norm_backward")


def mssa_mx_quantize(rows, cols, dtype, x, codes, scales, x_stride=0, stream=None):
    _check(lib.mssa_mx_quantize(int(rows), int(cols), _dtype(dtype), _ptr(x), int(x_stride), _ptr(codes),
                                _ptr(scales), _stream(stream)), "mssa_mx_quantize")


def mssa_mx_dequantize(rows, cols, dtype, codes, scales, y, y_stride=0, stream=None):
    _check(lib.mssa_mx_dequantize(int(rows), int(cols), _dtype(dtype), _ptr(codes), _ptr(scales), _ptr(y),
                                  int(y_stride), _stream(stream)), "mssa_mx_dequantize")


def mssa_mx_project(desc, x, x_scales, w, w_scales, bias, y, stream=None):
    """y: the desc.parts outputs."""
    if len(y) != desc.parts:
        raise ValueError("one output per part")
    _check(lib.mssa_mx_project(ctypes.byref(desc), _ptr(x), _ptr(x_scales), _ptr(w), _ptr(w_scales), _ptr(bias),
                               _ptr_array(y), _stream(stream)), "mssa_mx_project")


def mssa_mx_attention_workspace_size(desc):
    n = ctypes.c_int64()
    _check(lib.mssa_mx_attention_workspace_size(ctypes.byref(desc), ctypes.byref(n)),
           "mssa_mx_attention_workspace_size")
    return n.value


def mssa_mx_attention(desc, q, k_codes, k_scales, v_codes, v_scales, kv_len, prior_out, prior_lse, workspace, out,
                      lse=None, workspace_bytes=None, stream=None):
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    _check(lib.mssa_mx_attention(ctypes.byref(desc), _ptr(q), _ptr(k_codes), _ptr(k_scales), _ptr(v_codes),
                                 _ptr(v_scales), _ptr(kv_len), _ptr(prior_out), _ptr(prior_lse), _ptr(workspace), wb,
                                 _ptr(out), _ptr(lse), _stream(stream)), "mssa_mx_attention")


def adapter_project_desc(rows, in_features, out_features, segments, adapters, rank, parts=1, part0_scale=1.0,
                         x_stride=0):
    return mssa_adapter_project_desc(int(rows), int(in_features), int(out_features), int(parts), int(segments),
                                     int(adapters), int(rank), float(part0_scale), int(x_stride))


def paged_append_desc(tokens, batch, q_heads, kv_heads, head_dim, page_tokens, pages, table_pages, rotate_dims=None,
                      halves=False, axis_pairs=None, q_stride=0, k_stride=0, v_stride=0):
    """Descriptor of mssa_paged_append (rotate_dims: None turns the whole head;
    axis_pairs: the pairs of each position axis, None: one axis has them all)."""
    turned = int(head_dim if rotate_dims is None else rotate_dims)
    split = [turned // 2] if axis_pairs is None else [int(p) for p in axis_pairs]
    if not 1 <= len(split) <= 3:
        raise ValueError("axis_pairs has one to three entries")
    pairs = (ctypes.c_int32 * 3)(*split, *[0] * (3 - len(split)))
    return mssa_paged_append_desc(int(tokens), int(batch), int(q_heads), int(kv_heads), int(head_dim), int(page_tokens),
                                  int(table_pages), int(pages), turned, int(halves), len(split), pairs, int(q_stride),
                                  int(k_stride), int(v_stride))


def paged_attention_desc(tokens, batch, max_chunk, q_heads, kv_heads, head_dim, page_tokens, pages, table_pages,
                         mask_block=0, softmax_scale=0.0, q_stride=0, lse_stride=0):
    return mssa_paged_attention_desc(int(tokens), int(batch), int(max_chunk), int(q_heads), int(kv_heads), int(head_dim),
                                     int(page_tokens), int(table_pages), int(pages), int(mask_block), int(q_stride),
                                     int(lse_stride), float(softmax_scale))


def mssa_adapter_project_workspace_size(desc):
    n = ctypes.c_int64()
    _check(lib.mssa_adapter_project_workspace_size(ctypes.byref(desc), ctypes.byref(n)),
           "mssa_adapter_project_workspace_size")
    return n.value


def mssa_adapter_project(desc, x, w, bias, segment_begin, adapter, a, b, scale, workspace, y, workspace_bytes=None,
                         stream=None):
    """y: the desc.parts outputs."""
    if len(y) != desc.parts:
        raise ValueError("one output per part")
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    _check(lib.mssa_adapter_project(ctypes.byref(desc), _ptr(x), _ptr(w), _ptr(bias), _ptr(segment_begin), _ptr(adapter),
                                    _ptr(a), _ptr(b), _ptr(scale), _ptr(workspace), wb, _ptr_array(y), _stream(stream)),
           "mssa_adapter_project")


def mssa_paged_append(desc, q, k, v, chunk_begin, kv_len, page_table, positions, freqs, q_out, k_pages, v_pages,
                      stream=None):
    _check(lib.mssa_paged_append(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(chunk_begin), _ptr(kv_len),
                                 _ptr(page_table), _ptr(positions), _ptr(freqs), _ptr(q_out), _ptr(k_pages),
                                 _ptr(v_pages), _stream(stream)), "mssa_paged_append")


def mssa_paged_attention_workspace_size(desc):
    n = ctypes.c_int64()
    _check(lib.mssa_paged_attention_workspace_size(ctypes.byref(desc), ctypes.byref(n)),
           "mssa_paged_attention_workspace_size")
    return n.value


def mssa_paged_attention(desc, q, k_pages, v_pages, chunk_begin, kv_len, page_table, prior_out, prior_lse, workspace, out,
                         lse=None, workspace_bytes=None, stream=None):
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    _check(lib.mssa_paged_attention(ctypes.byref(desc), _ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(chunk_begin),
                                    _ptr(kv_len), _ptr(page_table), _ptr(prior_out), _ptr(prior_lse), _ptr(workspace), wb,
                                    _ptr(out), _ptr(lse), _stream(stream)), "mssa_paged_attention")


class HeadRing:
    """Host-side state of the rings of a MSSA_PLAN_HEAD_IN_RING plan: slots
    (ring_frames), history frames (count) and the first spare slot (spare),
    where window state 1 of the current pass lives."""

    def __init__(self, frames, count=0, spare=None):
        self.frames = int(frames)
        self.count = int(count)
        self.spare = int(count if spare is None else spare)


def mssa_pool_kv_head_ring(plan, k_ring, v_ring, k_win, v_win, k_ring_pooled, v_ring_pooled, workspace, ring,
                           workspace_bytes=None, stream=None):
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    _check(lib.mssa_pool_kv_head_ring(plan.handle, _ptr(k_ring), _ptr(v_ring), _ptr(k_win), _ptr(v_win),
                                      _ptr_array(k_ring_pooled), _ptr_array(v_ring_pooled), _ptr(workspace), wb,
                                      ring.frames, ring.count, ring.spare, _stream(stream)),
           "mssa_pool_kv_head_ring")


def mssa_forward_head_ring(plan, q_win, k_sink, v_sink, k_ring, v_ring, k_ring_pooled, v_ring_pooled, k_win, v_win,
                           workspace, out, ring, workspace_bytes=None, stream=None):
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    _check(lib.mssa_forward_head_ring(plan.handle, _ptr(q_win), _ptr(k_sink), _ptr(v_sink), _ptr(k_ring),
                                      _ptr(v_ring), _ptr_array(k_ring_pooled), _ptr_array(v_ring_pooled),
                                      _ptr(k_win), _ptr(v_win), _ptr(workspace), wb, _ptr(out), ring.frames,
                                      ring.count, ring.spare, _stream(stream)),
           "mssa_forward_head_ring")


def mssa_head_ring_roll(plan, ring):
    count = ctypes.c_int32(ring.count)
    spare = ctypes.c_int32(ring.spare)
    _check(lib.mssa_head_ring_roll(plan.handle, ring.frames, ctypes.byref(count), ctypes.byref(spare)),
           "mssa_head_ring_roll")
    ring.count, ring.spare = count.value, spare.value


class Ring:
    """Host-side head/count of a history ring used with mssa_hist_append."""

    def __init__(self, cap_frames, count=0, head=0):
        self.cap = int(cap_frames)
        self.count = int(count)
        self.head = int(head)


def mssa_hist_append(plan, k_win, v_win, k_ring, v_ring, ring, stream=None):
    head = ctypes.c_int32(ring.head)
    count = ctypes.c_int32(ring.count)
    _check(lib.mssa_hist_append(plan.handle, _ptr(k_win), _ptr(v_win), _ptr(k_ring), _ptr(v_ring),
                                ring.cap, ctypes.byref(head), ctypes.byref(count), _stream(stream)),
           "mssa_hist_append")
    ring.head, ring.count = head.value, count.value


def _ptr_array(xs):
    """Per-group pointer array (None entries -> NULL)."""
    arr = (ctypes.c_void_p * max(1, len(xs)))()
    for i, x in enumerate(xs):
        arr[i] = _ptr(x)
    return arr


def mssa_pool_hist_ring(plan, k_ring, v_ring, k_ring_pooled, v_ring_pooled, stream=None):
    _check(lib.mssa_pool_hist_ring(plan.handle, _ptr(k_ring), _ptr(v_ring), _ptr_array(k_ring_pooled),
                                   _ptr_array(v_ring_pooled), _stream(stream)), "mssa_pool_hist_ring")


def mssa_forward_ring(plan, q_win, k_sink, v_sink, k_hist, v_hist, k_hist_pooled, v_hist_pooled, k_win,
                      v_win, workspace, out, workspace_bytes=None, stream=None):
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    _check(lib.mssa_forward_ring(plan.handle, _ptr(q_win), _ptr(k_sink), _ptr(v_sink), _ptr(k_hist),
                                 _ptr(v_hist), _ptr_array(k_hist_pooled), _ptr_array(v_hist_pooled),
                                 _ptr(k_win), _ptr(v_win), _ptr(workspace), wb, _ptr(out),
                                 _stream(stream)), "mssa_forward_ring")


def mssa_hist_append_ring(plan, k_win, v_win, workspace, k_ring, v_ring, k_ring_pooled, v_ring_pooled, ring,
                          workspace_bytes=None, stream=None):
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    head = ctypes.c_int32(ring.head)
    count = ctypes.c_int32(ring.count)
    _check(lib.mssa_hist_append_ring(plan.handle, _ptr(k_win), _ptr(v_win), _ptr(workspace), wb,
                                     _ptr(k_ring), _ptr(v_ring), _ptr_array(k_ring_pooled),
                                     _ptr_array(v_ring_pooled), ring.cap, ctypes.byref(head),
                                     ctypes.byref(count), _stream(stream)), "mssa_hist_append_ring")
    ring.head, ring.count = head.value, count.value
