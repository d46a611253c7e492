"""Performance cases of the low-bit layer: what one transformer layer does around and inside its attention
when activations go through the products in 8 bits, weights and the K/V history in 4 bits.

A case is a dict of plain values.  Kinds (``kind``):

``norm``    serving: the residual's addition, the root-mean-square norm and its output, in the input's type or in
            8 bits (e4m3) with one scale a row;
``train``   the same norm with its backward: output, gradient of the input, gradient of the gain;
``quant``   values into MXFP4 (32 e2m1 values under one power-of-two scale) and back;
``project`` tokens in 8 or 4 bits times MXFP4 weights, plus bias, split into q, k, v;
``attend``  queries over a K/V cache held in MXFP4, alone or joined with the attention over other keys.

``prepare`` makes inputs from the seed alone, ``run`` is one pass through the public entry points or, where ``own``
is false, the same mathematics in elementary torch operations in 32 bits, ``work`` the bytes and operations a pass
cannot do without, ``exact`` the same outputs in 64 bits.
"""

import math

import torch

own = False

DEVICE = "cuda"
EPS = 1e-6
E4M3_MAX = 448.0
TINY = 2.0 ** -100  # the smallest row maximum that an 8-bit scale is made from
BLOCK = 32  # values under one MXFP4 scale
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4, "e4m3": 1}


def _norm(name, rows, cols, dtype="bf16", out="e4m3", residual=True, pad=0):
    return dict(name=name, kind="norm", rows=rows, cols=cols, dtype=dtype, out=out, residual=residual, pad=pad)


def _train(name, rows, cols, dtype="bf16", pad=0):
    return dict(name=name, kind="train", rows=rows, cols=cols, dtype=dtype, pad=pad)


def _quant(name, rows, cols, dtype="bf16"):
    return dict(name=name, kind="quant", rows=rows, cols=cols, dtype=dtype)


def _project(name, rows, cols, features, x="e4m3", out="bf16", parts=3):
    return dict(name=name, kind="project", rows=rows, cols=cols, features=features, x=x, out=out, parts=parts)


def _attend(name, batch, n_q, heads, kv_heads, head_dim, tokens, prior=False):
    return dict(name=name, kind="attend", batch=batch, n_q=n_q, heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                tokens=tokens, prior=prior)


def listed():
    return [
        # One token of the Wan-1.3B width before its projection: latency is all of it.
        _norm("norm_token", 1, 1536),
        # The tokens of the Wan-1.3B window (12870) between attention and the next projection.
        _norm("norm_window", 12870, 1536),
        # Training at the Wan-14B 720p window (27840 tokens of 5120), forward and backward: the largest norm.
        _train("train_norm_14b", 27840, 5120),
        # Training of a small fp32 model of odd width, rows cut out of a wider tensor.
        _train("train_norm_odd_f32", 1001, 1023, "f32", pad=5),
        # The keys of one emitted state (3 frames x 1560 tokens x 12 heads) on their way into the 4-bit history.
        _quant("quant_frames", 3 * 1560 * 12, 128),
        # The fp32 QKV weights of the Wan-14B layer, laid out once when a model is loaded.
        _quant("quant_weights_14b", 15360, 5120, "f32"),
        # QKV of one token at the Wan-14B width: the weights are read once, the bus bounds it.
        _project("qkv_token_14b", 1, 5120, 15360),
        # QKV of the Wan-1.3B window, 8-bit tokens and 4-bit weights: the ordinary pass.
        _project("qkv_window", 12870, 1536, 4608),
        # QKV of the Wan-14B 720p window with 4-bit tokens: the largest product.
        _project("qkv_14b_mxfp4", 27840, 5120, 15360, x="mxfp4"),
        # Single queries of 16 streams, 40 query heads over 8 key heads, histories up to 21 frames (32760 tokens),
        # one of them still empty.
        _attend("attend_token", 16, 1, 40, 8, 128, 32760),
        # The native-scale queries of a Wan-1.3B pass (9360) over a full 21-frame history, joined with the
        # attention over sink and window: the largest.
        _attend("attend_history", 1, 9360, 12, 12, 128, 32760, prior=True),
        # A small head_dim 64 model on a 17 x 23 grid, three streams of different lengths.
        _attend("attend_ragged_d64", 3, 391, 6, 2, 64, 5 * 391),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "train", "quant", "project", "attend"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("norm", "train"):
        cols = _log_int(rng, 64, 5120)
        if rng.random() < 0.6:
            cols = max(64, cols // 64 * 64)
        rows = _log_int(rng, 1, 27840)
        pad = rng.choice([0, 0, 8, 3])
        if kind == "train":
            return {k: v for k, v in _train("", rows, cols, dtype, pad).items() if k != "name"}
        out = rng.choice(["e4m3", "e4m3", dtype])
        return {k: v for k, v in _norm("", rows, cols, dtype, out, rng.random() < 0.8, pad).items() if k != "name"}
    if kind == "quant":
        cols = rng.choice([64, 128, _log_int(rng, 1, 5120), _log_int(rng, 1, 160) * 32])
        rows = _log_int(rng, 1, min(200000, 15360 * 5120 // cols))
        return {k: v for k, v in _quant("", rows, cols, dtype).items() if k != "name"}
    if kind == "project":
        cols = _log_int(rng, 64, 5120)
        if rng.random() < 0.7:
            cols = max(64, cols // 64 * 64)
        parts = rng.choice([1, 3, 3])
        features = parts * rng.choice([_log_int(rng, 64, 5120), max(64, _log_int(rng, 64, 5120) // 64 * 64)])
        return {k: v for k, v in _project("", _log_int(rng, 1, 27840), cols, features, rng.choice(["e4m3", "mxfp4"]),
                                          rng.choice(["bf16", "bf16", "f32"]), parts).items() if k != "name"}
    head_dim = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 6, 8, 12])
    heads = kv_heads * rng.choice([1, 1, 2, 5])
    batch = rng.choice([1, 1, 2, 3, 8])
    n_q = rng.choice([1, _log_int(rng, 1, 64), _log_int(rng, 64, 9360)])
    most = 9360 * 32760 * 12 // (batch * n_q * heads)
    tokens = _log_int(rng, 1, max(2, min(32760, most)))
    return {k: v for k, v in _attend("", batch, n_q, heads, kv_heads, head_dim, tokens, rng.random() < 0.4).items()
            if k != "name"}


def _padded(cols):
    return -(-cols // BLOCK) * BLOCK


def _lengths(case):
    """Tokens each stream's cache holds: spread from an empty one to a full one; one stream has a full one."""
    b, t = case["batch"], case["tokens"]
    return [t] if b == 1 else [t * i // (b - 1) for i in range(b)]


# --------------------------------------------------------------- formats


def _pow2(e):
    """2^e in float32 from whole numbers e in [-127, 127], bit by bit."""
    return torch.where(e > -127, (e + 127) << 23, torch.full_like(e, 1 << 22)).to(torch.int32).view(torch.float32)


def _blocks(x):
    """[..., cols] -> [..., blocks, 32] in float32, the last block filled with zeros."""
    x = torch.nn.functional.pad(x.float(), (0, _padded(x.shape[-1]) - x.shape[-1]))
    return x.reshape(*x.shape[:-1], -1, BLOCK)


def _mx(x):
    """Codes (0..15, one a value) and scale bytes of x: exponent floor(log2 max) - 2, nearest even, saturating; a
    block that holds an infinity or a NaN has scale 255, which stands for NaN."""
    v = _blocks(x)
    top = v.abs().amax(-1, keepdim=True)
    e = torch.where(top > 0, torch.frexp(top).exponent - 3, torch.full_like(top, -127, dtype=torch.int32)).clamp(-127, 127)
    a = v * ((127 - e) << 23).to(torch.int32).view(torch.float32)
    m = a.abs()
    code = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0))
    code = code + 8 * (a < 0)
    scale = torch.where(torch.isfinite(top), e + 127, torch.full_like(e, 255))
    return code.to(torch.uint8).flatten(-2), scale.squeeze(-1).to(torch.uint8)


def _values(code, scale, table):
    """What codes (one a value) and scale bytes stand for, in float32."""
    s = torch.where(scale == 255, torch.full_like(scale, 0, dtype=torch.float32) / 0, _pow2(scale.int() - 127))
    return (table[code.int()].unflatten(-1, (-1, BLOCK)) * s.unsqueeze(-1)).flatten(-2)


def _pack(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _unpack(packed):
    return torch.stack((packed & 15, packed >> 4), -1).flatten(-2)


def _table(dtype=torch.float32):
    return torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=dtype, device=DEVICE)


def _e4m3(v):
    """Rows in 8 bits: codes and one scale a row."""
    scale = v.abs().amax(-1).clamp_min(TINY) / E4M3_MAX
    return torch.nn.functional.pad((v / scale.unsqueeze(-1)).to(torch.float8_e4m3fn).view(torch.uint8),
                                   (0, _padded(v.shape[-1]) - v.shape[-1])).view(torch.float8_e4m3fn), scale


# --------------------------------------------------------------- inputs


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=g, device=DEVICE) * std

    s = dict(case=dict(case), desc=None, table=_table())
    kind = case["kind"]
    if kind in ("norm", "train"):
        rows, cols, pad, t = case["rows"], case["cols"], case["pad"], TYPES[case["dtype"]]
        # rows of the residual stream differ in size, and a few channels carry most of it
        size = torch.exp(normal(rows, 1, std=0.5)) * torch.exp(normal(1, cols + pad, std=0.7))
        s["x"] = (normal(rows, cols + pad) * size).to(t)[:, :cols]
        s["residual"] = (normal(rows, cols + pad, std=2.0) * size).to(t)[:, :cols]
        s["weight"] = (1 + normal(cols, std=0.2)).to(t)
        if kind == "train":
            s["dy"] = normal(rows, cols).to(t)
            s["dsum"] = normal(rows, cols).to(t)
        elif not case["residual"]:
            s["residual"] = None
        out = case.get("out", case["dtype"])
        s["sum"] = torch.empty(rows, cols, dtype=t, device=DEVICE)
        s["y"] = (torch.empty(rows, _padded(cols), dtype=torch.float8_e4m3fn, device=DEVICE) if out == "e4m3"
                  else torch.empty(rows, cols, dtype=t, device=DEVICE))
        s["y_scale"] = torch.empty(rows, device=DEVICE) if out == "e4m3" else None
        s["rstd"] = torch.empty(rows, device=DEVICE)
        s["dx"] = torch.empty(rows, cols, dtype=t, device=DEVICE)
        s["dweight"] = torch.empty(cols, device=DEVICE)
    elif kind == "quant":
        rows, cols, t = case["rows"], case["cols"], TYPES[case["dtype"]]
        s["x"] = (normal(rows, cols) * torch.exp(normal(rows, 1, std=1.5))).to(t)
        s["codes"] = torch.empty(rows, _padded(cols) // 2, dtype=torch.uint8, device=DEVICE)
        s["scales"] = torch.empty(rows, _padded(cols) // BLOCK, dtype=torch.uint8, device=DEVICE)
        s["y"] = torch.empty_like(s["x"])
    elif kind == "project":
        rows, cols, n, t = case["rows"], case["cols"], case["features"], TYPES[case["out"]]
        x = normal(rows, cols) * torch.exp(normal(1, cols, std=0.5))
        if case["x"] == "e4m3":
            s["x"], s["x_scale"] = _e4m3(x)
        else:
            code, s["x_scale"] = _mx(x)
            s["x"] = _pack(code)
        code, s["w_scale"] = _mx(normal(n, cols, std=cols ** -0.5))
        s["w"] = _pack(code)
        s["bias"] = normal(n, std=0.1).to(t)
        s["y"] = [torch.empty(rows, n // case["parts"], dtype=t, device=DEVICE) for _ in range(case["parts"])]
        s["factor"] = 1.4426950408889634 / math.sqrt(128.0) if case["parts"] == 3 else 1.0
    else:
        b, n_q, h, kvh, d, t = (case[k] for k in ("batch", "n_q", "heads", "kv_heads", "head_dim", "tokens"))
        s["q"] = normal(b, n_q, h, d).to(torch.bfloat16)
        for name in ("k", "v"):
            code, s[name + "_scale"] = _mx(normal(b, t, kvh, d))
            s[name] = _pack(code)
        order = torch.randperm(b, generator=g, device=DEVICE)
        s["kv_len"] = torch.tensor(_lengths(case), dtype=torch.int32, device=DEVICE)[order].contiguous()
        s["prior_out"] = normal(b, n_q, h, d, std=0.1).to(torch.bfloat16) if case["prior"] else None
        s["prior_lse"] = (math.log(t) + 0.5 + normal(b, h, n_q)) if case["prior"] else None
        s["out"] = torch.empty(b, n_q, h, d, dtype=torch.bfloat16, device=DEVICE)
        s["lse"] = torch.empty(b, h, n_q, device=DEVICE)
    s["workspace"] = None
    return s


# --------------------------------------------------------------- own


def _plan(s):
    """The descriptor and workspace that a program keeps for its calls, made by the first of them."""
    from paper_2607_20940_amd import mssa

    c = s["case"]
    kind = c["kind"]
    if kind in ("norm", "train"):
        s["desc"] = mssa.norm_desc(c["rows"], c["cols"], dtype=c["dtype"], out=c.get("out", c["dtype"]), eps=EPS,
                                   x_stride=c["cols"] + c["pad"],
                                   residual_stride=c["cols"] + c["pad"] if s["residual"] is not None else 0)
        size = mssa.mssa_add_rms_norm_workspace_size(s["desc"])
    elif kind == "project":
        s["desc"] = mssa.mx_project_desc(c["rows"], c["cols"], c["features"], parts=c["parts"], x_format=c["x"],
                                         out=c["out"], part0_scale=s["factor"])
        size = 0
    elif kind == "attend":
        s["desc"] = mssa.mx_attention_desc(c["batch"], c["n_q"], c["heads"], c["kv_heads"], c["head_dim"], c["tokens"])
        size = mssa.mssa_mx_attention_workspace_size(s["desc"])
    else:
        s["desc"], size = True, 0
    s["workspace"] = torch.empty(max(256, size), dtype=torch.uint8, device=DEVICE)


def _run_own(s):
    from paper_2607_20940_amd import mssa

    c = s["case"]
    if s["desc"] is None:
        _plan(s)
    if c["kind"] == "norm":
        mssa.mssa_add_rms_norm(s["desc"], s["x"], s["residual"], s["weight"],
                               s["sum"] if s["residual"] is not None else None, s["y"], s["y_scale"], None)
        return [v for v in (s["sum"] if s["residual"] is not None else None, s["y"], s["y_scale"]) if v is not None]
    if c["kind"] == "train":
        mssa.mssa_add_rms_norm(s["desc"], s["x"], s["residual"], s["weight"], s["sum"], s["y"], None, s["rstd"])
        mssa.mssa_add_rms_norm_backward(s["desc"], s["sum"], s["weight"], s["rstd"], s["dy"], s["dsum"],
                                        s["workspace"], s["dx"], s["dweight"])
        return [s["sum"], s["y"], s["dx"], s["dweight"]]
    if c["kind"] == "quant":
        mssa.mssa_mx_quantize(c["rows"], c["cols"], c["dtype"], s["x"], s["codes"], s["scales"])
        mssa.mssa_mx_dequantize(c["rows"], c["cols"], c["dtype"], s["codes"], s["scales"], s["y"])
        return s["y"]
    if c["kind"] == "project":
        mssa.mssa_mx_project(s["desc"], s["x"], s["x_scale"], s["w"], s["w_scale"], s["bias"], s["y"])
        return s["y"]
    mssa.mssa_mx_attention(s["desc"], s["q"], s["k"], s["k_scale"], s["v"], s["v_scale"], s["kv_len"], s["prior_out"],
                           s["prior_lse"], s["workspace"], s["out"], s["lse"])
    return [s["out"], s["lse"]]


# --------------------------------------------------------------- plain


def _norm_plain(s):
    """The sum as the residual stream keeps it, its rows' 1 / rms, and the normalised rows, in 32 bits."""
    x = s["x"].float()
    total = x if s["residual"] is None else (x + s["residual"].float()).to(s["x"].dtype).float()
    rstd = 1 / torch.sqrt((total * total).mean(-1, keepdim=True) + EPS)
    return total, rstd, total * rstd * s["weight"].float()


def _project_plain(s):
    c = s["case"]
    x = s["x"].float() * s["x_scale"].unsqueeze(-1) if c["x"] == "e4m3" else _values(_unpack(s["x"]), s["x_scale"], s["table"])
    y = torch.matmul(x, _values(_unpack(s["w"]), s["w_scale"], s["table"]).t()) + s["bias"].float()
    first, *rest = y.chunk(c["parts"], -1)
    return [v.to(TYPES[c["out"]]) for v in (first * s["factor"], *rest)]


def _attend_plain(s):
    c = s["case"]
    b, n_q, h, kvh, d = (c[k] for k in ("batch", "n_q", "heads", "kv_heads", "head_dim"))
    k = _values(_unpack(s["k"]), s["k_scale"], s["table"]).permute(0, 2, 3, 1).contiguous()
    v = _values(_unpack(s["v"]), s["v_scale"], s["table"]).permute(0, 2, 1, 3).contiguous()
    q = s["q"].float().reshape(b, n_q, kvh, h // kvh, d).permute(0, 2, 3, 1, 4).reshape(b, kvh, -1, d) * d ** -0.5
    score = torch.matmul(q, k)
    gone = torch.arange(c["tokens"], device=DEVICE) >= s["kv_len"].unsqueeze(-1)
    score.masked_fill_(gone[:, None, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    score = score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score, v) / torch.where(total > 0, total, torch.ones_like(total))
    lse = top + total.log()
    out = out.reshape(b, h, n_q, d)
    lse = lse.reshape(b, h, n_q)
    if s["prior_out"] is not None:
        both = torch.logaddexp(lse, s["prior_lse"])
        out = (out * (lse - both).exp().unsqueeze(-1)
               + s["prior_out"].float().permute(0, 2, 1, 3) * (s["prior_lse"] - both).exp().unsqueeze(-1))
        lse = both
    return [out.permute(0, 2, 1, 3).to(torch.bfloat16).contiguous(), lse]


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "project":
        return _project_plain(s)
    if kind == "attend":
        return _attend_plain(s)
    t = s["x"].dtype
    if kind == "quant":
        code, scale = _mx(s["x"])
        return _values(code, scale, s["table"])[:, : s["case"]["cols"]].to(t)
    total, rstd, y = _norm_plain(s)
    if kind == "train":
        g = s["dy"].float() * s["weight"].float()
        inner = (g * total).mean(-1, keepdim=True)
        dx = s["dsum"].float() + rstd * (g - total * (rstd * rstd * inner))
        return [total.to(t), y.to(t), dx.to(t), (s["dy"].float() * total * rstd).sum(0)]
    outs = [total.to(t)] if s["residual"] is not None else []
    return outs + (list(_e4m3(y)) if s["case"]["out"] == "e4m3" else [y.to(t)])


def run(state):
    return _run_own(state) if own else _run_plain(state)


# --------------------------------------------------------------- work


def work(case):
    kind = case["kind"]
    if kind in ("norm", "train"):
        n, b = case["rows"] * case["cols"], SIZE[case["dtype"]]
        if kind == "train":  # forward: x, residual, sum, y; backward: sum, dy, dsum, dx
            return {"bytes": 8.0 * n * b + 4 * case["rows"] * 2 + case["cols"] * (2 * b + 4), "flops": 20.0 * n}
        return {"bytes": float(n * (b * (3 if case["residual"] else 1) + SIZE[case["out"]]) + case["cols"] * b),
                "flops": 8.0 * n}
    if kind == "quant":  # values read, codes and scales written, read again, values written
        n = case["rows"] * _padded(case["cols"])
        return {"bytes": 2.0 * case["rows"] * case["cols"] * SIZE[case["dtype"]] + 2 * n * (0.5 + 1 / BLOCK), "flops": 4.0 * n}
    if kind == "project":
        m, k, n = case["rows"], _padded(case["cols"]), case["features"]
        x = m * k if case["x"] == "e4m3" else m * k * (0.5 + 1 / BLOCK)
        return {"bytes": x + n * k * (0.5 + 1 / BLOCK) + SIZE[case["out"]] * (m * n + n), "flops": 2.0 * m * n * k}
    kv = sum(_lengths(case))
    q = case["batch"] * case["n_q"] * case["heads"]
    return {"bytes": 2.0 * kv * case["kv_heads"] * case["head_dim"] * (0.5 + 1 / BLOCK)
            + q * (case["head_dim"] * (6 if case["prior"] else 4) + (8 if case["prior"] else 4)),
            "flops": 4.0 * case["n_q"] * case["heads"] * case["head_dim"] * kv}


# --------------------------------------------------------------- exact


def _values64(packed, scale):
    """What packed codes and scale bytes stand for, from the format's definition: sign, exponent and one mantissa
    bit of each value, times two to the scale's power."""
    out = []
    for nibble in (packed & 15, packed >> 4):
        expo, mant = ((nibble >> 1) & 3).double(), (nibble & 1).double()
        mag = torch.where(expo == 0, mant / 2, (1 + mant / 2) * torch.exp2(expo - 1))
        out.append(torch.where(nibble >= 8, -mag, mag))
    v = torch.stack(out, -1).flatten(-2).unflatten(-1, (-1, BLOCK))
    s = torch.pow(torch.full((), 2.0, dtype=torch.float64, device=DEVICE), scale.double() - 127)
    return (v * torch.where(scale == 255, torch.full_like(s, math.nan), s).unsqueeze(-1)).flatten(-2)


def _nearest_e2m1(m):
    """The e2m1 magnitude nearest to m >= 0, ties to the one whose last bit is even, 6 at most."""
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0)).double()
    return (torch.round(m / step) * step).clamp_max(6.0)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "quant":
        rows, cols = s["x"].shape
        v = torch.zeros(rows, _padded(cols), dtype=torch.float64, device=DEVICE)
        v[:, :cols] = s["x"].double()
        v = v.view(rows, -1, BLOCK)
        top = v.abs().amax(-1, keepdim=True)
        unit = torch.where(top > 0, torch.exp2(torch.floor(torch.log2(top)) - 2), torch.ones_like(top))
        # log2 rounds: a maximum just under a power of two may have been taken for it
        unit = torch.where(top < 4 * unit, unit / 2, unit)
        unit = torch.where(top >= 8 * unit, unit * 2, unit)
        unit = torch.clamp_min(unit, 2.0 ** -127)
        return (torch.sign(v) * _nearest_e2m1(v.abs() / unit) * unit).view(rows, -1)[:, :cols]
    if kind == "project":
        w = _values64(s["w"], s["w_scale"])
        x = s["x"].double() * s["x_scale"].double()[:, None] if case["x"] == "e4m3" else _values64(s["x"], s["x_scale"])
        n = case["features"] // case["parts"]
        ys = []
        for p in range(case["parts"]):
            y = torch.mm(x, w[p * n:(p + 1) * n].t().contiguous()) + s["bias"][p * n:(p + 1) * n].double()
            ys.append(y * s["factor"] if p == 0 else y)
        return ys
    if kind == "attend":
        b, n_q, h, d = s["q"].shape
        group = h // case["kv_heads"]
        out = torch.zeros(b, n_q, h, d, dtype=torch.float64, device=DEVICE)
        lse = torch.full((b, h, n_q), -math.inf, dtype=torch.float64, device=DEVICE)
        for i, n in enumerate(s["kv_len"].tolist()):
            for j in range(h if n else 0):
                kj = j // group
                k = _values64(s["k"][i, :n, kj].contiguous(), s["k_scale"][i, :n, kj])
                v = _values64(s["v"][i, :n, kj].contiguous(), s["v_scale"][i, :n, kj])
                p = torch.mm(s["q"][i, :, j].double() / math.sqrt(d), k.t().contiguous())
                lse[i, j] = torch.logsumexp(p, -1)
                out[i, :, j] = torch.mm(torch.exp(p - lse[i, j][:, None]), v)
        if case["prior"]:
            a, other = torch.exp(lse), torch.exp(s["prior_lse"].double())
            share = (a / (a + other)).transpose(1, 2).unsqueeze(-1)
            out = share * out + (1 - share) * s["prior_out"].double()
            lse = torch.log(a + other)
        return [out, lse]
    x = s["x"].double()
    total = x if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(s["x"].dtype).double()
    n = case["cols"]
    rms = torch.sqrt(torch.einsum("rc,rc->r", total, total) / n + EPS)[:, None]
    w = s["weight"].double()
    y = total / rms * w
    if kind == "train":
        hat, dy = total / rms, s["dy"].double()
        dx = s["dsum"].double() + (w * dy - hat * ((w * dy * hat).sum(-1, keepdim=True) / n)) / rms
        return [total, y, dx, (dy * hat).sum(0)]
    outs = [total] if s["residual"] is not None else []
    if case["out"] != "e4m3":
        return outs + [y]
    scale = torch.clamp_min(y.abs().max(-1).values, TINY) / E4M3_MAX
    v = y / scale[:, None]
    # three mantissa bits above 2^-6, steps of 2^-9 below
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    code = torch.zeros(case["rows"], _padded(n), dtype=torch.float64, device=DEVICE)
    code[:, :n] = torch.round(v / step) * step
    return outs + [code, scale]
