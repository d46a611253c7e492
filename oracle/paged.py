"""Plain definitions of the operators for streams served together, in 64 bits
(numpy): the shared projection with an adapter per segment, the rotation of
queries and keys, storing in pages, attention over pages."""

import numpy as np


def chunks(chunk_begin, batch, tokens):
    """(first, end) of every sequence's rows."""
    if chunk_begin is None:
        return [(b * (tokens // batch), (b + 1) * (tokens // batch)) for b in range(batch)]
    return [(int(chunk_begin[b]), int(chunk_begin[b + 1])) for b in range(batch)]


# ------------------------------------------------------------------ project


def adapter_project(x, w, bias, segment_begin, adapter, a, b, scale, parts, part0_scale):
    """x [M, K], w [N, K], a [J, parts, R, K], b [J, N, R].  Returns the parts and, per output, the sum of magnitudes of
    the shared product and of the adapter's (what rounding errors scale with)."""
    n = w.shape[0] // parts
    ys, mags, lows = [], [], []
    for p in range(parts):
        wp = w[p * n:(p + 1) * n]
        y, mag, low = x @ wp.T, np.abs(x) @ np.abs(wp).T, np.zeros((x.shape[0], n))
        if bias is not None:
            y = y + bias[p * n:(p + 1) * n]
        for s, j in enumerate(adapter):
            r0, r1 = int(segment_begin[s]), int(segment_begin[s + 1])
            if 0 <= j < len(a) and r1 > r0:
                f = 1.0 if scale is None else float(scale[j])
                bp = b[j, p * n:(p + 1) * n]
                y[r0:r1] += f * (x[r0:r1] @ a[j, p].T) @ bp.T
                low[r0:r1] = abs(f) * (np.abs(x[r0:r1]) @ np.abs(a[j, p]).T) @ np.abs(bp).T
        f = part0_scale if p == 0 else 1.0
        ys.append(y * f)
        mags.append(mag * abs(f))
        lows.append(low * abs(f))
    return ys, mags, lows


# ------------------------------------------------------------------- append


def rotate(x, angle, halves):
    """x [tokens, heads, D], angle [tokens, P]: dims 0 .. 2 P - 1 turned as pairs.  Returns the result and |u| + |v| of
    every value's pair."""
    out, mag = x.copy(), np.abs(x)
    p = angle.shape[1]
    i = np.arange(p)
    u, v = (i, i + p) if halves else (2 * i, 2 * i + 1)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    out[..., u], out[..., v] = x[..., u] * c - x[..., v] * s, x[..., u] * s + x[..., v] * c
    mag[..., u] = mag[..., v] = np.abs(x[..., u]) + np.abs(x[..., v])
    return out, mag


def places(chunk_begin, kv_len, page_table, page_tokens, pages, tokens):
    """Per row: its cache index (None in no sequence) and (page, token in it), None where it is stored nowhere."""
    table = np.asarray(page_table)
    index, place = [None] * tokens, [None] * tokens
    for b, (r0, r1) in enumerate(chunks(chunk_begin, table.shape[0], tokens)):
        for r in range(r0, r1):
            c = index[r] = int(kv_len[b]) - (r1 - r)
            if 0 <= c < table.shape[1] * page_tokens and 0 <= table[b, c // page_tokens] < pages:
                place[r] = (int(table[b, c // page_tokens]), c % page_tokens)
    return index, place


# ---------------------------------------------------------------- attention


def attention(q, k_pages, v_pages, chunk_begin, kv_len, page_table, scale, mask_block=0, prior=None):
    """q [tokens, H, D], pages [pages, page_tokens, KH, D], prior (out, lse [H, tokens]).  Returns out, lse and the
    softmax mean of |v| per output; rows of no sequence are NaN."""
    T, H, D = q.shape
    pages, pt, KH, _ = k_pages.shape
    table = np.asarray(page_table)
    out, mag, lse = np.full(q.shape, np.nan), np.full(q.shape, np.nan), np.full((H, T), np.nan)
    for b, (r0, r1) in enumerate(chunks(chunk_begin, table.shape[0], T)):
        n = min(max(int(kv_len[b]), 0), table.shape[1] * pt)
        at = np.arange(n)
        page = table[b, at // pt]
        have = (page >= 0) & (page < pages)
        for r in range(r0, r1):
            i = r - r0
            end = int(kv_len[b]) - (r1 - r0) + (i // mask_block + 1) * mask_block if mask_block else n
            see = at[have & (at < end)]
            for h in range(H):
                o, m, s = np.zeros(D), np.zeros(D), -np.inf
                if len(see):
                    kk = k_pages[table[b, see // pt], see % pt, h // (H // KH)]
                    vv = v_pages[table[b, see // pt], see % pt, h // (H // KH)]
                    x = scale * (kk @ q[r, h])
                    top = x.max()
                    p = np.exp(x - top)
                    o, m, s = p @ vv / p.sum(), p @ np.abs(vv) / p.sum(), top + np.log(p.sum())
                if prior is not None:
                    po, pl = prior[0][r, h], float(prior[1][h, r])
                    joint = np.logaddexp(s, pl)
                    ref = 0.0 if np.isneginf(joint) else joint
                    o = o * np.exp(s - ref) + po * np.exp(pl - ref)
                    m = m * np.exp(s - ref) + np.abs(po) * np.exp(pl - ref)
                    s = joint
                out[r, h], mag[r, h], lse[h, r] = o, m, s
    return out, lse, mag
