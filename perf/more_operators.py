"""Performance cases of a layer that serves several streams at once: the shared projection with every stream's
own low-rank adapter, new keys and values rotated and put into a paged cache, and the attention of the new tokens
over that cache.

A case is a dict of plain values.  Kinds (``kind``):

``adapt``   tokens times shared weights plus bias, split into parts, and beside it a low-rank adapter per segment of
            rows (a request's tokens, or a patchification tier's);
``append``  the chunk's queries rotated, its keys rotated and put with the values into the pages of their sequences;
``attend``  a chunk of new tokens a sequence (one or many) over all that the sequence's pages hold.

``prepare`` makes inputs from the seed alone, ``run`` is one pass through the public entry points or, where ``own``
is false, the same mathematics in elementary torch operations in 32 bits (angles in 64), ``work`` the bytes and
operations a pass cannot do without, ``exact`` the same outputs in 64 bits.
"""

import math

import torch

own = False

DEVICE = "cuda"
THETA = 10000.0
LOG2E = 1.4426950408889634
GRID_H, GRID_W = 30, 52  # native tokens of a latent frame


def _adapt(name, rows, cols, features, rank, segments, adapters, parts=3):
    return dict(name=name, kind="adapt", rows=rows, cols=cols, features=features, rank=rank, segments=segments,
                adapters=adapters, parts=parts)


def _append(name, batch, chunk, history, heads, kv_heads, head_dim, page, axes=1, rotate=0, halves=False, pad=0):
    return dict(name=name, kind="append", batch=batch, chunk=chunk, history=history, heads=heads, kv_heads=kv_heads,
                head_dim=head_dim, page=page, axes=axes, rotate=rotate or head_dim, halves=halves, pad=pad)


def _attend(name, batch, chunk, history, heads, kv_heads, head_dim, page, mask=0, prior=False):
    return dict(name=name, kind="attend", batch=batch, chunk=chunk, history=history, heads=heads, kv_heads=kv_heads,
                head_dim=head_dim, page=page, mask=mask, prior=prior)


def listed():
    return [
        # One token of each of 16 requests at the Wan-14B width, eight adapters among them: the weights' bytes count.
        _adapt("adapt_tokens_14b", 16, 5120, 15360, 16, 16, 8),
        # The Wan-1.3B window (12870 tokens): the native tier's adapter and the 2x2 tier's.
        _adapt("adapt_window", 12870, 1536, 4608, 32, 2, 2),
        # The Wan-14B 720p window with three tiers' adapters: the largest product.
        _adapt("adapt_window_14b", 27840, 5120, 15360, 64, 3, 3),
        # Prompts of 13 requests of odd lengths in a small model, an odd rank, one output.
        _adapt("adapt_ragged", 611, 608, 1000, 12, 13, 5, parts=1),
        # One token of each of 16 streams, 40 query heads over 8 key heads: latency is all of it.
        _append("append_token", 16, 1, 32760, 40, 8, 128, 64, halves=True),
        # An emitted state of Wan-1.3B (3 frames x 1560 tokens), positions in frame, row and column, a frame a page.
        _append("append_state", 1, 3 * 1560, 18 * 1560, 12, 12, 128, 1560, axes=3),
        # States of four Wan-14B 720p streams (3 frames x 3600 tokens each): the largest.
        _append("append_states_14b", 4, 3 * 3600, 0, 40, 40, 128, 256, axes=3),
        # Three streams of a small head_dim 64 model, half of each head rotated, rows cut out of a wider tensor.
        _append("append_ragged_d64", 3, 391, 5 * 391, 6, 2, 64, 16, rotate=32, halves=True, pad=8),
        # Single queries of 16 streams, 40 query heads over 8 key heads, histories of 0 to 21 frames.
        _attend("attend_token", 16, 1, 32759, 40, 8, 128, 64),
        # A state's queries over 21 frames of history and itself, joined with the attention over sink and window.
        _attend("attend_state", 1, 3 * 1560, 21 * 1560, 12, 12, 128, 1560, prior=True),
        # Three streams that prefill different numbers of frames, a frame seeing itself and those before: the largest.
        _attend("attend_frames", 3, 6 * 1560, 15 * 1560, 12, 12, 128, 256, mask=1560),
        # A small head_dim 64 model, three streams of different lengths, token by token.
        _attend("attend_ragged_d64", 3, 391, 5 * 391, 6, 2, 64, 16, mask=1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _unnamed(case):
    return {k: v for k, v in case.items() if k != "name"}


def draw(rng):
    kind = rng.choice(["adapt", "append", "attend"])
    if kind == "adapt":
        cols = _log_int(rng, 64, 5120)
        if rng.random() < 0.7:
            cols = max(64, cols // 64 * 64)
        parts = rng.choice([1, 3, 3])
        features = parts * rng.choice([_log_int(rng, 64, 5120), max(64, _log_int(rng, 64, 5120) // 64 * 64)])
        rank = rng.choice([8, 16, 32, 64, _log_int(rng, 1, 64)])
        rows = rng.choice([_log_int(rng, 1, 64), _log_int(rng, 64, 27840)])
        segments = rng.choice([rows if rows <= 64 else 3, min(rows, _log_int(rng, 1, 40))])
        return _unnamed(_adapt("", rows, cols, features, rank, segments, rng.choice([1, 2, 3, 5, 8, 16]), parts))
    head_dim = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 6, 8, 12])
    heads = kv_heads * rng.choice([1, 1, 2, 5])
    batch = rng.choice([1, 1, 2, 3, 8, 16])
    page = rng.choice([16, 64, 256, 1560, _log_int(rng, 1, 2000)])
    if kind == "append":
        chunk = rng.choice([1, _log_int(rng, 1, 64), _log_int(rng, 64, max(65, 43200 // batch))])
        axes = rng.choice([1, 3])
        rotate = head_dim if axes == 3 else rng.choice([head_dim, head_dim // 2])
        return _unnamed(_append("", batch, chunk, _log_int(rng, 1, 32760) - 1, heads, kv_heads, head_dim, page, axes,
                                rotate, rng.random() < 0.5, rng.choice([0, 0, 8, 24])))
    chunk = rng.choice([1, _log_int(rng, 1, 64), _log_int(rng, 64, max(65, min(9360, 9360 * 24 // (batch * heads))))])
    most = 9360 * 32760 * 12 // (batch * chunk * heads) - chunk
    history = _log_int(rng, 1, max(2, min(32760, most))) - 1
    mask = rng.choice([0, 1, 1, _log_int(rng, 2, 1560)])
    return _unnamed(_attend("", batch, chunk, history, heads, kv_heads, head_dim, page, mask, rng.random() < 0.3))


def _spread(case):
    """New tokens of each sequence and tokens that its cache holds with them: chunks from the whole down to half,
    histories from none to the longest."""
    b, n, h = case["batch"], case["chunk"], case["history"]
    chunks = [n - n * i // (2 * b) for i in range(b)]
    before = [h] if b == 1 else [h * i // (b - 1) for i in range(b)]
    return chunks, [c + p for c, p in zip(chunks, before)]


def _segments(case):
    """First row of each segment, and the end: lengths grow evenly, or a row each."""
    r, s = case["rows"], case["segments"]
    return [i if r == s else r * i * (i + 1) // (s * (s + 1)) for i in range(s)] + [r]


# --------------------------------------------------------------- inputs


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=g, device=DEVICE) * std

    def order(n):
        return torch.randperm(n, generator=g, device=DEVICE)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device=DEVICE)

    bf16 = torch.bfloat16
    s = dict(case=dict(case), desc=None, workspace=None)
    if case["kind"] == "adapt":
        rows, cols, n, parts, rank = (case[k] for k in ("rows", "cols", "features", "parts", "rank"))
        s["x"] = (normal(rows, cols) * torch.exp(normal(1, cols, std=0.5))).to(bf16)
        s["w"] = normal(n, cols, std=cols ** -0.5).to(bf16)
        s["bias"] = normal(n, std=0.1).to(bf16)
        s["a"] = normal(case["adapters"], parts, rank, cols, std=cols ** -0.5).to(bf16)
        s["b"] = normal(case["adapters"], n, rank, std=0.3 * rank ** -0.5).to(bf16)
        s["scale"] = 0.5 + torch.rand(case["adapters"], generator=g, device=DEVICE)
        s["begin"] = ints(_segments(case))
        which = [i % case["adapters"] for i in range(case["segments"])]
        if case["segments"] > 3:
            which[-1] = -1  # a request without an adapter
        s["which"] = ints(which)[order(case["segments"])].contiguous()
        s["factor"] = LOG2E / math.sqrt(128.0) if parts == 3 else 1.0
        s["y"] = [torch.empty(rows, n // parts, dtype=bf16, device=DEVICE) for _ in range(parts)]
        return s
    heads, kvh, d, page = (case[k] for k in ("heads", "kv_heads", "head_dim", "page"))
    chunks, lens = _spread(case)
    # the streams arrive in any order
    mix = order(case["batch"])
    new, held = ints(chunks)[mix], ints(lens)[mix]
    tokens = sum(chunks)
    s["begin"] = torch.nn.functional.pad(new.cumsum(0), (1, 0)).int()
    s["kv_len"] = held.contiguous()
    # pages in no order, spare ones among them; the table's entries past a sequence's pages name none
    used = [-(-n // page) for n in lens]
    s["pages"] = sum(used) + 3
    s["table"] = torch.full((case["batch"], max(used)), -1, dtype=torch.int32, device=DEVICE)
    there = torch.arange(max(used), device=DEVICE) < ((held + page - 1) // page)[:, None]
    s["table"][there] = order(s["pages"])[: sum(used)].int()
    pool = (s["pages"], page, kvh, d)
    s["k_pages"], s["v_pages"] = normal(*pool).to(bf16), normal(*pool).to(bf16)
    if case["kind"] == "append":
        pad = case["pad"]
        s["q"] = normal(tokens, heads * d + pad).to(bf16)[:, : heads * d]
        s["k"] = normal(tokens, kvh * d + pad).to(bf16)[:, : kvh * d]
        s["v"] = normal(tokens, kvh * d + pad).to(bf16)[:, : kvh * d]
        pairs = case["rotate"] // 2
        split = [pairs] if case["axes"] == 1 else [pairs - pairs // 3 * 2, pairs // 3, pairs // 3]
        s["split"] = split
        s["freqs"] = torch.cat([THETA ** (-torch.arange(p, device=DEVICE, dtype=torch.float64) / p) for p in split]).float()
        s["positions"] = None
        if case["axes"] == 3:
            at = _cache_index(s, torch.arange(tokens, device=DEVICE))[1]
            s["positions"] = torch.stack((at // (GRID_H * GRID_W), at // GRID_W % GRID_H, at % GRID_W)).int().contiguous()
        s["q_out"] = torch.empty(tokens, heads, d, dtype=bf16, device=DEVICE)
        return s
    s["q"] = normal(tokens, heads, d).to(bf16)
    s["prior_out"] = normal(tokens, heads, d, std=0.1).to(bf16) if case["prior"] else None
    s["prior_lse"] = math.log(max(lens)) + 0.5 + normal(heads, tokens) if case["prior"] else None
    s["out"] = torch.empty(tokens, heads, d, dtype=bf16, device=DEVICE)
    s["lse"] = torch.empty(heads, tokens, device=DEVICE)
    return s


def _cache_index(s, row):
    """The sequence that each row belongs to, and the row's place in its cache."""
    seq = torch.searchsorted(s["begin"][1:].contiguous().long(), row, right=True)
    end = s["begin"][1:].long()[seq]
    return seq, s["kv_len"].long()[seq] - end + row


# --------------------------------------------------------------- own


def _plan(s):
    """The descriptor and workspace that a program keeps for its calls, made by the first of them."""
    from paper_2607_20940_amd import mssa

    c = s["case"]
    if c["kind"] == "adapt":
        s["desc"] = mssa.adapter_project_desc(c["rows"], c["cols"], c["features"], c["segments"], c["adapters"], c["rank"],
                                              parts=c["parts"], part0_scale=s["factor"])
        size = mssa.mssa_adapter_project_workspace_size(s["desc"])
    elif c["kind"] == "append":
        s["desc"] = mssa.paged_append_desc(s["q"].shape[0], c["batch"], c["heads"], c["kv_heads"], c["head_dim"], c["page"],
                                           s["pages"], s["table"].shape[1], rotate_dims=c["rotate"], halves=c["halves"],
                                           axis_pairs=s["split"], q_stride=s["q"].stride(0), k_stride=s["k"].stride(0),
                                           v_stride=s["v"].stride(0))
        size = 0
    else:
        s["desc"] = mssa.paged_attention_desc(s["q"].shape[0], c["batch"], c["chunk"], c["heads"], c["kv_heads"],
                                              c["head_dim"], c["page"], s["pages"], s["table"].shape[1],
                                              mask_block=c["mask"])
        size = mssa.mssa_paged_attention_workspace_size(s["desc"])
    s["workspace"] = torch.empty(max(256, size), dtype=torch.uint8, device=DEVICE)


def _run_own(s):
    from paper_2607_20940_amd import mssa

    if s["desc"] is None:
        _plan(s)
    kind = s["case"]["kind"]
    if kind == "adapt":
        mssa.mssa_adapter_project(s["desc"], s["x"], s["w"], s["bias"], s["begin"], s["which"], s["a"], s["b"], s["scale"],
                                  s["workspace"], s["y"])
        return s["y"]
    if kind == "append":
        mssa.mssa_paged_append(s["desc"], s["q"], s["k"], s["v"], s["begin"], s["kv_len"], s["table"], s["positions"],
                               s["freqs"], s["q_out"], s["k_pages"], s["v_pages"])
        return [s["q_out"], s["k_pages"], s["v_pages"]]
    mssa.mssa_paged_attention(s["desc"], s["q"], s["k_pages"], s["v_pages"], s["begin"], s["kv_len"], s["table"],
                              s["prior_out"], s["prior_lse"], s["workspace"], s["out"], s["lse"])
    return [s["out"], s["lse"]]


# --------------------------------------------------------------- plain


def _adapt_plain(s):
    c = s["case"]
    rows, n, parts, rank, adapters = (c[k] for k in ("rows", "features", "parts", "rank", "adapters"))
    x = s["x"].float()
    y = torch.matmul(x, s["w"].float().t()) + s["bias"].float()
    seg = torch.searchsorted(s["begin"][1:].contiguous(), torch.arange(rows, device=DEVICE, dtype=torch.int32), right=True)
    mine = s["which"][seg]
    # every row against every adapter, all but its own weighed with 0
    share = (mine[:, None] == torch.arange(adapters, device=DEVICE)) * s["scale"]
    u = torch.matmul(x, s["a"].float().flatten(0, 2).t()).view(rows, adapters, parts, rank) * share[:, :, None, None]
    u = u.permute(2, 0, 1, 3).reshape(parts, rows, adapters * rank)
    b = s["b"].float().view(adapters, parts, n // parts, rank).permute(1, 0, 3, 2).reshape(parts, adapters * rank, -1)
    y = y.view(rows, parts, n // parts).transpose(0, 1) + torch.matmul(u, b)
    y[0] *= s["factor"]
    return list(y.to(torch.bfloat16))


def _rotated(x, cos, sin, halves):
    """x [tokens, heads, head_dim] in 32 bits, its first 2 P dims turned as pairs; cos and sin [tokens, P]."""
    p = cos.shape[1]
    turn, rest = x[..., : 2 * p], x[..., 2 * p:]
    cos, sin = cos[:, None], sin[:, None]
    a, b = (turn[..., :p], turn[..., p:]) if halves else (turn[..., 0::2], turn[..., 1::2])
    a, b = a * cos - b * sin, a * sin + b * cos
    turn = torch.cat((a, b), -1) if halves else torch.stack((a, b), -1).flatten(-2)
    return torch.cat((turn, rest), -1)


def _append_plain(s):
    c = s["case"]
    tokens = s["q"].shape[0]
    seq, at = _cache_index(s, torch.arange(tokens, device=DEVICE))
    axis = torch.repeat_interleave(torch.arange(len(s["split"]), device=DEVICE), torch.tensor(s["split"], device=DEVICE))
    place = at[:, None].expand(-1, len(axis)) if s["positions"] is None else s["positions"].t()[:, axis]
    angle = place.double() * s["freqs"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    q = s["q"].float().view(tokens, c["heads"], -1)
    k = s["k"].float().view(tokens, c["kv_heads"], -1)
    s["q_out"].copy_(_rotated(q, cos, sin, c["halves"]))
    page = s["table"][seq, at // c["page"]].long()
    s["k_pages"][page, at % c["page"]] = _rotated(k, cos, sin, c["halves"]).to(torch.bfloat16)
    s["v_pages"][page, at % c["page"]] = s["v"].reshape(tokens, c["kv_heads"], -1)
    return [s["q_out"], s["k_pages"], s["v_pages"]]


def _attend_plain(s):
    c = s["case"]
    b, h, kvh, d, longest = (c[k] for k in ("batch", "heads", "kv_heads", "head_dim", "chunk"))
    tokens = s["q"].shape[0]
    begin, lens = s["begin"].long(), s["kv_len"].long()
    new = begin[1:] - begin[:-1]
    # sequences side by side, as long as the longest of them
    cap = s["table"].shape[1] * c["page"]
    k = s["k_pages"][s["table"].clamp_min(0).long()].view(b, cap, kvh, d).permute(0, 2, 3, 1).float().contiguous()
    v = s["v_pages"][s["table"].clamp_min(0).long()].view(b, cap, kvh, d).permute(0, 2, 1, 3).float().contiguous()
    i = torch.arange(longest, device=DEVICE)
    row = (begin[:-1, None] + i).clamp_max(tokens - 1)
    q = s["q"][row].float() * d ** -0.5  # [b, longest, h, d]
    q = q.view(b, longest, kvh, h // kvh, d).permute(0, 2, 3, 1, 4).reshape(b, kvh, -1, d)
    score = torch.matmul(q, k).view(b, h, longest, cap)
    sees = lens[:, None].expand(b, longest)
    if c["mask"]:
        sees = torch.minimum(sees, (lens - new)[:, None] + (i // c["mask"] + 1) * c["mask"])
    score.masked_fill_((torch.arange(cap, device=DEVICE) >= sees[..., None])[:, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    score = score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score.view(b, kvh, -1, cap), v).view(b, h, longest, d)
    out = out / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + total.log()).squeeze(-1)
    there = i < new[:, None]  # the rows that are tokens, in their order
    out, lse = out.transpose(1, 2)[there], lse.transpose(1, 2)[there].t().contiguous()
    if s["prior_out"] is not None:
        both = torch.logaddexp(lse, s["prior_lse"])
        out = (out * (lse - both).exp().t().unsqueeze(-1)
               + s["prior_out"].float() * (s["prior_lse"] - both).exp().t().unsqueeze(-1))
        lse = both
    return [out.to(torch.bfloat16), lse]


def run(state):
    if own:
        return _run_own(state)
    return {"adapt": _adapt_plain, "append": _append_plain, "attend": _attend_plain}[state["case"]["kind"]](state)


# --------------------------------------------------------------- work


def _pairs(case):
    """Query-key pairs of a head that the mask leaves."""
    total = 0
    for n, held in zip(*_spread(case)):
        before, m = held - n, case["mask"]
        if not m:
            total += n * held
            continue
        whole, rest = divmod(n, m)
        total += n * before + m * m * whole * (whole + 1) // 2 + rest * n
    return total


def work(case):
    if case["kind"] == "adapt":
        m, k, n = case["rows"], case["cols"], case["features"]
        low = case["rank"] * (case["parts"] * k + n)
        with_one = m if case["segments"] <= 3 else m - max(1, m // case["segments"])
        return {"bytes": 2.0 * (m * k + n * k + n + m * n + min(case["adapters"], case["segments"]) * low),
                "flops": 2.0 * m * n * k + 2.0 * with_one * low}
    chunks, lens = _spread(case)
    new, d = sum(chunks), case["head_dim"]
    if case["kind"] == "append":
        return {"bytes": 4.0 * new * d * (case["heads"] + 2 * case["kv_heads"]),
                "flops": 3.0 * new * case["rotate"] * (case["heads"] + case["kv_heads"])}
    rows = new * case["heads"]
    return {"bytes": 4.0 * sum(lens) * case["kv_heads"] * d
            + rows * (d * (6 if case["prior"] else 4) + (8 if case["prior"] else 4)),
            "flops": 4.0 * _pairs(case) * case["heads"] * d}


# --------------------------------------------------------------- exact


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "adapt":
        n, parts, x = case["features"] // case["parts"], case["parts"], s["x"].double()
        begin, which = s["begin"].tolist(), s["which"].tolist()
        ys = []
        for p in range(parts):
            y = torch.mm(x, s["w"][p * n:(p + 1) * n].double().t().contiguous()) + s["bias"][p * n:(p + 1) * n].double()
            for i, j in enumerate(which):
                a, b = begin[i], begin[i + 1]
                if j >= 0 and b > a:
                    low = torch.mm(x[a:b], s["a"][j, p].double().t().contiguous())
                    y[a:b] += s["scale"][j].double() * torch.mm(low, s["b"][j, p * n:(p + 1) * n].double().t().contiguous())
            ys.append(y * s["factor"] if p == 0 else y)
        return ys
    begin, lens, table, page = s["begin"].tolist(), s["kv_len"].tolist(), s["table"].tolist(), case["page"]
    heads, kvh, d = case["heads"], case["kv_heads"], case["head_dim"]
    if case["kind"] == "append":
        k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
        q_out = torch.zeros(begin[-1], heads, d, dtype=torch.float64, device=DEVICE)
        axis = [x for x, p in enumerate(s["split"]) for _ in range(p)]
        half = case["rotate"] // 2
        for b, n in enumerate(lens):
            r = torch.arange(begin[b], begin[b + 1], device=DEVICE)
            at = r - begin[b + 1] + n
            pos = [at if s["positions"] is None else s["positions"][x][r] for x in range(len(s["split"]))]
            # e^(i angle) times the pair as a complex number
            angle = torch.stack([pos[x].double() * s["freqs"][j].double() for j, x in enumerate(axis)], -1)
            turn = torch.polar(torch.ones_like(angle), angle)[:, None]
            for name, m in (("q", heads), ("k", kvh)):
                y = s[name][r].double().view(-1, m, d).clone()
                i = torch.arange(half, device=DEVICE)
                re, im = (i, i + half) if case["halves"] else (2 * i, 2 * i + 1)
                z = torch.complex(y[..., re], y[..., im]) * turn
                y[..., re], y[..., im] = z.real, z.imag
                if name == "q":
                    q_out[r] = y
                else:
                    slot = torch.tensor(table[b], device=DEVICE)[at // page]
                    k_pages[slot, at % page] = y
                    v_pages[slot, at % page] = s["v"][r].double().view(-1, kvh, d)
        return [q_out, k_pages, v_pages]
    out = torch.zeros(begin[-1], heads, d, dtype=torch.float64, device=DEVICE)
    lse = torch.full((heads, begin[-1]), -math.inf, dtype=torch.float64, device=DEVICE)
    for b, n in enumerate(lens):
        first, m = begin[b], begin[b + 1] - begin[b]
        mine = [p for p in table[b] if p >= 0]
        keys, values = (t[mine].view(-1, kvh, d)[:n] for t in (s["k_pages"], s["v_pages"]))
        i = torch.arange(m, device=DEVICE)[:, None]
        end = n - m + (i // case["mask"] + 1) * case["mask"] if case["mask"] else torch.full_like(i, n)
        hidden = torch.arange(n, device=DEVICE) >= end
        for j in range(heads):
            p = torch.mm(s["q"][first:first + m, j].double() / math.sqrt(d), keys[:, j // (heads // kvh)].double().t().contiguous())
            p = p.masked_fill(hidden, -math.inf)
            lse[j, first:first + m] = torch.logsumexp(p, -1)
            p = torch.exp(p - lse[j, first:first + m, None])
            out[first:first + m, j] = torch.mm(p, values[:, j // (heads // kvh)].double())
    if case["prior"]:
        a, other = torch.exp(lse), torch.exp(s["prior_lse"].double())
        share = (a / (a + other)).t().unsqueeze(-1)
        out = share * out + (1 - share) * s["prior_out"].double()
        lse = torch.log(a + other)
    return [out, lse]
