"""fp64 oracle of the low-bit layers: the root-mean-square norm with the
residual's addition and its gradients, the MXFP4 and 8-bit row formats, the
product with MXFP4 weights, the attention over an MXFP4 cache.  numpy only;
formats are written out from their definitions (sign, exponent and mantissa
bits), not from tables of the library."""

import numpy as np

BLOCK = 32
E4M3_MAX = 448.0
TINY = 2.0 ** -100


def padded(cols):
    return -(-cols // BLOCK) * BLOCK


# --------------------------------------------------------------------- norm


def norm(s, weight, eps):
    """y and 1/rms of rows s (already the rounded sum x + r)."""
    rstd = 1.0 / np.sqrt((s * s).mean(-1) + eps)
    return s * rstd[:, None] * weight, rstd


def norm_grad(s, weight, eps, dy, dsum=None):
    """dx and dweight of sum(dy * y) + sum(dsum * s)."""
    n = s.shape[1]
    rms = np.sqrt((s * s).mean(-1, keepdims=True) + eps)
    g = dy * weight
    dx = g / rms - s * ((g * s).sum(-1, keepdims=True) / (n * rms ** 3))
    return (dx if dsum is None else dx + dsum), (dy * s / rms).sum(0)


# --------------------------------------------------------------------- e4m3


def e4m3_value(code):
    """Values of e4m3 bytes (OCP: bias 7, no infinities, 0x7f / 0xff NaN)."""
    code = np.asarray(code, dtype=np.int64)
    sign = np.where(code & 0x80, -1.0, 1.0)
    e, m = (code >> 3) & 15, (code & 7).astype(np.float64)
    mag = np.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * 2.0 ** (e - 7.0))
    return sign * np.where((code & 0x7f) == 0x7f, np.nan, mag)


# -------------------------------------------------------------------- MXFP4


def e2m1_value(code):
    code = np.asarray(code, dtype=np.int64)
    e, m = (code >> 1) & 3, (code & 1).astype(np.float64)
    return np.where(code & 8, -1.0, 1.0) * np.where(e == 0, m / 2, (1 + m / 2) * 2.0 ** (e - 1.0))


def mx_scale_byte(x):
    """Scale bytes [rows, blocks] of rows x."""
    rows, cols = x.shape
    v = np.zeros((rows, padded(cols)))
    v[:, :cols] = x
    v = np.abs(v.reshape(rows, -1, BLOCK))
    bad = ~np.isfinite(v).all(-1)
    top = np.where(np.isfinite(v), v, 0).max(-1)
    _, e = np.frexp(top)  # top in [2^(e-1), 2^e)
    byte = np.where(top > 0, np.maximum(e - 1 - 2 + 127, 0), 0)
    return np.where(bad, 255, byte)


def mx_codes(x):
    """(codes [rows, padded cols], scale bytes): nearest value, ties to the
    even code, found by distance to every representable magnitude."""
    rows, cols = x.shape
    byte = mx_scale_byte(x)
    v = np.zeros((rows, padded(cols)))
    v[:, :cols] = x
    v = v.reshape(rows, -1, BLOCK)
    bad = byte == 255
    a = np.where(bad[..., None], 0.0, v) / 2.0 ** (np.where(bad, 127, byte) - 127.0)[..., None]
    mags = e2m1_value(np.arange(8))
    dist = np.abs(np.abs(a)[..., None] - mags)
    # of two equally near ones the even code: odd codes lose ties
    code = np.argmin(dist * 16 + (dist == dist.min(-1, keepdims=True)) * (np.arange(8) % 2) * 1e-9, -1)
    code = np.where((a < 0), code + 8, code)
    return code.reshape(rows, -1), byte


def mx_pack(code):
    return (code[:, 0::2] | (code[:, 1::2] << 4)).astype(np.uint8)


def mx_unpack(packed):
    packed = np.asarray(packed, dtype=np.int64)
    return np.stack((packed & 15, packed >> 4), -1).reshape(packed.shape[0], 2 * packed.shape[1])


def mx_values(packed, byte):
    """Values [rows, padded cols] of packed codes and scale bytes."""
    v = e2m1_value(mx_unpack(packed)).reshape(len(packed), 2 * np.shape(packed)[1] // BLOCK, BLOCK)
    byte = np.asarray(byte, dtype=np.float64)
    scale = np.where(byte == 255, np.nan, 2.0 ** (byte - 127))
    return (v * scale[..., None]).reshape(len(packed), 2 * np.shape(packed)[1])


# ------------------------------------------------------------------ product


def project(x, w, bias, parts, part0_scale):
    y = x @ w.T + (0 if bias is None else bias)
    ys = np.split(y, parts, axis=1)
    ys[0] = ys[0] * part0_scale
    return ys


# ---------------------------------------------------------------- attention


def attention(q, k, v, scale, kv_len, prior=None):
    """q [B, n, H, D]; k, v [B, T, KH, D] values; prior (out, lse).  Returns
    out, lse [B, H, n] and, per output, the softmax mean of |v| (what rounding
    errors scale with)."""
    B, n, H, D = q.shape
    KH = k.shape[2]
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    lse = np.full((B, H, n), -np.inf)
    for b in range(B):
        t = int(kv_len[b])
        for h in range(H):
            kh = h // (H // KH)
            if t:
                s = scale * (q[b, :, h] @ k[b, :t, kh].T)
                top = s.max(-1, keepdims=True)
                p = np.exp(s - top)
                tot = p.sum(-1, keepdims=True)
                out[b, :, h] = p @ v[b, :t, kh] / tot
                mag[b, :, h] = p @ np.abs(v[b, :t, kh]) / tot
                lse[b, h] = (top + np.log(tot))[:, 0]
            if prior is not None:
                po, pl = prior[0][b, :, h], prior[1][b, h]
                joint = np.logaddexp(lse[b, h], pl)
                ref = np.where(np.isneginf(joint), 0, joint)  # no keys on either side: both shares are 0
                w, wp = np.exp(lse[b, h] - ref)[:, None], np.exp(pl - ref)[:, None]
                out[b, :, h] = out[b, :, h] * w + po * wp
                mag[b, :, h] = mag[b, :, h] * w + np.abs(po) * wp
                lse[b, h] = joint
    return out, lse, mag
