"""CPU oracle of the step in front of the attention call: norms of Q and K per head, their rotation by the token's (frame,
height, width) position, and the gradients of both.  float64 NumPy, written from the formulas; test infrastructure only.

Rows are the last axis: x [..., N, d], tokens in default order, image tokens (F * Hg * Wg of them) first."""
from __future__ import annotations

import numpy as np


def rope_table(extents, dims, pos, inv_freq):
    """float32 [entries, 2]: cosine and sine of coordinate times frequency, axis by axis, coordinate by coordinate."""
    out, p0, i0 = [], 0, 0
    for extent, dim in zip(extents, dims):
        for i in range(extent):
            for p in range(dim // 2):
                angle = np.float64(pos[i0 + i]) * np.float64(inv_freq[p0 + p])
                out.append((np.float32(np.cos(angle)), np.float32(np.sin(angle))))
        i0 += extent
        p0 += dim // 2
    return np.array(out, np.float32).reshape(-1, 2)


def token_angles(grid, T_text, d, dims, table):
    """(cosine, sine) [N, d / 2] of every token: what the table holds for its coordinates; (1, 0) where nothing turns."""
    F, Hg, Wg = grid
    n = F * Hg * Wg + T_text
    cos, sin = np.ones((n, d // 2)), np.zeros((n, d // 2))
    t = 0
    for f in range(F):
        for h in range(Hg):
            for w in range(Wg):
                p, base = 0, 0
                for coord, extent, dim in zip((f, h, w), (F, Hg, Wg), dims):
                    part = table[base + coord * (dim // 2): base + (coord + 1) * (dim // 2)]
                    cos[t, p: p + dim // 2], sin[t, p: p + dim // 2] = part[:, 0], part[:, 1]
                    p += dim // 2
                    base += extent * (dim // 2)
                t += 1
    return cos, sin


def pair_channels(d, halves):
    """The two channel numbers of every pair: int [d / 2] each."""
    p = np.arange(d // 2)
    return (p, p + d // 2) if halves else (2 * p, 2 * p + 1)


def turn(x, cos, sin, halves, inverse=False):
    a, b = pair_channels(x.shape[-1], halves)
    s = -sin if inverse else sin
    y = np.array(x, np.float64)
    still = (cos == 1) & (sin == 0)  # what does not turn stays as it is, whatever its partner holds
    with np.errstate(invalid="ignore"):
        y[..., a] = np.where(still, x[..., a], x[..., a] * cos - x[..., b] * s)
        y[..., b] = np.where(still, x[..., b], x[..., a] * s + x[..., b] * cos)
    return y


def normed(x, kind, eps):
    """(x - m) r and r of every row; kind "rms" or "layer"."""
    x = np.asarray(x, np.float64)
    if kind == "layer":
        x = x - x.mean(-1, keepdims=True)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return x * r, r


def per_token(shared, text, n_img, n):
    """Weights (or biases) [d] of every token [N, d]; text tokens take `text` where it is given."""
    return np.concatenate([np.tile(shared, (n_img, 1)), np.tile(shared if text is None else text, (n - n_img, 1))]).astype(np.float64)


def norm_rope(x, kind, eps, w, b, cos, sin, halves):
    """w, b: [N, d] (per_token)."""
    u = np.asarray(x, np.float64) if kind == "none" else normed(x, kind, eps)[0] * w + b
    return turn(u, cos, sin, halves)


def norm_rope_backward(x, dy, kind, eps, w, cos, sin, halves):
    """dx, and per row the terms g h and g whose sums over rows are the gradients of weights and biases."""
    g = turn(np.asarray(dy, np.float64), cos, sin, halves, inverse=True)
    if kind == "none":
        return g, None, None
    h, r = normed(x, kind, eps)
    v = g * w
    dx = v - h * (v * h).mean(-1, keepdims=True)
    if kind == "layer":
        dx = dx - v.mean(-1, keepdims=True)
    return r * dx, g * h, g
