"""fp64 oracle of the operators around the expert layer: block norms, balance
loss, 4-bit values and their products, written from the definitions."""
from __future__ import annotations

import numpy as np


# ---------------------------------------------------------------- block norms
def combine(Y, slot_row, slot_weights):
    """(sum, sum of magnitudes) over a token's slots; rows out of range add nothing."""
    T, k = slot_row.shape
    y = np.zeros((T, Y.shape[1]))
    mag = np.zeros_like(y)
    for t in range(T):
        for j in range(k):
            r = slot_row[t, j]
            if 0 <= r < Y.shape[0]:
                y[t] += slot_weights[t, j] * Y[r]
                mag[t] += np.abs(slot_weights[t, j] * Y[r])
    return y, mag


def block_norm(h, y, w_pre=None, w_post=None, scale=None, gate=None, residual_scale=1.0, eps=1e-6, y_mag=None):
    """(h_out, x, magnitude of the terms of h_out, scale of x's error): fp64."""
    if y is None:
        out, mag = h, np.abs(h)
    else:
        f = np.ones_like(h)
        if w_post is not None:
            f = f / np.sqrt(np.mean(y * y, 1, keepdims=True) + eps) * w_post
        if gate is not None:
            f = f * gate[:, None]
        if scale is not None:
            f = f * scale
        out = residual_scale * h + f * y
        mag = np.abs(residual_scale * h) + np.abs(f) * (np.abs(y) if y_mag is None else y_mag)
    if w_pre is None:
        return out, None, mag, None
    r = 1 / np.sqrt(np.mean(out * out, 1, keepdims=True) + eps)
    return out, out * r * w_pre, mag, (mag + np.abs(out)) * r * np.abs(w_pre)


def block_norm_grads(h_out, y, dx, dh_out, w_pre=None, w_post=None, scale=None, gate=None, residual_scale=1.0, eps=1e-6):
    """{name: (gradient, sum of magnitudes of its terms)} in fp64."""
    D = np.zeros_like(h_out) if dh_out is None else dh_out.copy()
    A = np.abs(D)
    out = {}
    if w_pre is not None:
        r = 1 / np.sqrt(np.mean(h_out * h_out, 1, keepdims=True) + eps)
        m, dm = h_out * r, dx * w_pre
        D = D + r * (dm - m * np.mean(dm * m, 1, keepdims=True))
        A = A + r * (np.abs(dm) + np.abs(m) * np.mean(np.abs(dm * m), 1, keepdims=True))
        out["dw_pre"] = ((dx * m).sum(0), np.abs(dx * m).sum(0))
    if y is None:
        out["dh"] = (D, A)
        return out
    out["dh"] = (residual_scale * D, abs(residual_scale) * A)
    g = 1.0 if gate is None else gate[:, None]
    s = 1.0 if scale is None else scale
    w = 1.0 if w_post is None else w_post
    ry = 1.0 if w_post is None else 1 / np.sqrt(np.mean(y * y, 1, keepdims=True) + eps)
    n = y * ry
    if gate is not None:
        out["dgate"] = ((D * s * w * n).sum(1), (A * np.abs(s * w * n)).sum(1))
    if scale is not None:
        out["dscale"] = ((D * g * w * n).sum(0), (A * np.abs(g * w * n)).sum(0))
    dn = D * g * s * w
    An = A * np.abs(g * s * w)
    if w_post is not None:
        out["dw_post"] = ((D * g * s * n).sum(0), (A * np.abs(g * s * n)).sum(0))
        dn, An = (ry * (dn - n * np.mean(dn * n, 1, keepdims=True)),
                  ry * (An + np.abs(n) * np.mean(An * np.abs(n), 1, keepdims=True)))
    out["dy"] = (dn, An)
    return out


# ---------------------------------------------------------------- balance loss
def softmax(z):
    """Rows of only -inf become rows of zeros."""
    top = z.max(1, keepdims=True)
    e = np.exp(z - np.where(np.isneginf(top), 0.0, top))
    s = e.sum(1, keepdims=True)
    return np.divide(e, s, out=np.zeros_like(e), where=s != 0)


def balance(logits, ids, mask=None, coef=1.0, dloss=1.0):
    """loss, counts, prob, n, dlogits, magnitude of dlogits' terms."""
    T, E = logits.shape
    k = ids.shape[1]
    keep = np.ones(T, bool) if mask is None else mask.astype(bool)
    n = int(keep.sum())
    counts = np.zeros(E, np.int64)
    for e in ids[keep].ravel():
        if 0 <= e < E:
            counts[e] += 1
    d = np.zeros((T, E))
    if n == 0:
        return 0.0, counts, np.zeros(E), 0, d, d
    p = softmax(logits[keep].astype(np.float64))
    prob = p.sum(0) / n
    f = counts / (k * n)
    w = dloss * coef * E / n
    dot = (p * f).sum(1, keepdims=True)
    d[keep] = w * p * (f - dot)
    mag = np.zeros((T, E))
    mag[keep] = abs(w) * p * (f + dot)
    return coef * E * float((f * prob).sum()), counts, prob, n, d, mag


# ---------------------------------------------------------------- 4-bit values
GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
LUT = np.concatenate([GRID, -GRID])


def padded(K):
    return -(-K // 128) * 128


def quantize(x):
    """fp64 [rows][K] -> (codes, scales, distance of each value to the nearest
    place where its code changes, in units of the block's scale)."""
    rows, K = x.shape
    b = np.zeros((rows, padded(K)))
    b[:, :K] = x
    b = b.reshape(rows, -1, 32)
    top = np.abs(b).max(2)
    bad = ~np.isfinite(top)
    _, e = np.frexp(np.where(bad | (top == 0), 1.0, top))
    s = np.where(top == 0, 0, np.clip(e - 3 + 127, 0, 254))
    q = np.where(bad[:, :, None], 0.0, b) / np.exp2(s - 127.0)[:, :, None]
    a = np.minimum(np.abs(q), 6.0)
    d = np.abs(a[..., None] - GRID)
    near = d.min(-1, keepdims=True)
    # of two values equally near, the one with the even code
    code = np.argmax((d == near) & ((np.arange(8) % 2 == 0) | ((d == near).sum(-1, keepdims=True) == 1)), -1)
    mids = (GRID[1:] + GRID[:-1]) / 2
    slack = np.abs(np.abs(q)[..., None] - mids).min(-1)
    code = np.where(np.signbit(q), code + 8, code)
    code = np.where(bad[:, :, None], 0, code)
    s = np.where(bad, 255, s)
    code = code.reshape(rows, -1)
    return (code[:, 0::2] | (code[:, 1::2] << 4)).astype(np.uint8), s.astype(np.uint8), slack.reshape(rows, -1)[:, :K]


def dequantize(codes, scales, K):
    c = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (-1,))
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (LUT[c] * np.repeat(s, 32, -1))[..., :K]


def silu_mul(x):
    K = x.shape[1] // 2
    g, u = x[:, :K], x[:, K:]
    return g / (1 + np.exp(-g)) * u


def gemm(a, b, M, offsets=None, row_map=None):
    """a [rows][K], b [G][N][K] fp64 -> [M][N]; rows of no group are NaN."""
    out = np.full((M, b.shape[1]), np.nan)
    rm = np.arange(M) if row_map is None else row_map
    A = np.zeros((M, a.shape[1]))
    ok = (rm >= 0) & (rm < a.shape[0])
    A[ok] = a[rm[ok]]
    off = [0, M] if offsets is None else [int(v) for v in offsets]
    for g in range(b.shape[0]):
        if off[g + 1] > off[g]:
            out[off[g]:off[g + 1]] = A[off[g]:off[g + 1]] @ b[g].T
    return out
