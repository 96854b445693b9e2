"""Plain float64 forms, on the CPU, of the calls in which frames see each other, and the bounds that their results are held to.

Bounds, beside those of layer_oracle.  u = 2^-24, h half a step of the operands' type relative to the value (2^-8 bfloat16, 2^-11
float16).
Norm and rotation: a sum of D squares, a division, a root and three products are within (D + 8) u; sines and cosines (series and
the angle's rounding to 32 bits) within 2^-22 of 1; a rotated value is a sum of two products.
Scores: D products of 16-bit values, exact in float32, summed: e_S = (D + 2) u scale sum |q k|.  A probability relative to the row's
reference is off by e_S, by the reference's own (the same sums), by the product with log2 e (2 u |S - m|, at most 2 u (|S| + |m|))
and by the exponential (2^-21 of it): relative e_P = 2 max_s e_S + 4 u max |S| + 2^-21, and half a step h when it is rounded; below
2^-14 float16 is subnormal, which leaves 2^-25 relative to the row's largest term at least.  A sum of n terms adds n u of their magnitudes,
and rows that are joined from parts are scaled by two more factors of this kind.
Gradients, y and L being inputs: P = exp(S - L) as above; dP and delta are sums of D products; dS = P (dP - delta) is off by
(e_P + h) |dS| + P (e_dP + e_delta), where P >= 2^-126 (the exponential and the matrix cores know no smaller numbers), and its sums over frames (and the heads of a group) by n u more."""
import numpy as np
import torch

from layer_oracle import U32, f64, rounding

HALF = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


def frames_there(B, T, lengths):
    n = np.full(B, T) if lengths is None else np.clip(np.asarray(lengths), 0, T)
    return n, np.arange(T)[None] < n[:, None]


def split(x, D):
    """[B, T, columns] to [B, T, heads, D]"""
    return x.reshape(*x.shape[:-1], -1, D)


def rotate(n, positions, frequencies, sign=1.0):
    """n [B, T, heads, D], positions [B, T]: pairs (i, i + R / 2) by the angle position * frequency (both exact in float64)"""
    h = len(frequencies)
    a = sign * np.asarray(positions, np.longdouble)[:, :, None, None] * np.asarray(frequencies, np.longdouble)
    c, s = np.cos(a).astype(np.float64), np.sin(a).astype(np.float64)
    x, y = n[..., :h], n[..., h:2 * h]
    return np.concatenate([x * c - y * s, y * c + x * s, n[..., 2 * h:]], -1)


def head_norm(x, D, gain, positions, frequencies, there, eps=1e-5):
    """(y, bound before the last rounding), [B, T, heads, D]"""
    x = np.where(there[:, :, None, None], split(x, D), 0.0)
    n = x if gain is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain
    h = len(frequencies)
    y = rotate(n, positions, frequencies)
    m = np.abs(n).copy()
    m[..., :h] = m[..., h:2 * h] = np.abs(n[..., :h]) + np.abs(n[..., h:2 * h])
    return y, m * ((0 if gain is None else (D + 8) * U32) + 2.0 ** -22 + 4 * U32)


def head_norm_grad(dy, x, D, gain, positions, frequencies, there, eps=1e-5):
    """(dx, its bound, dgain, its bound)"""
    w = there[:, :, None, None]
    x, dy = np.where(w, split(x, D), 0.0), np.where(w, split(dy, D), 0.0)
    h = len(frequencies)
    dn = rotate(dy, positions, frequencies, -1.0)
    m = np.abs(dy).copy()
    m[..., :h] = m[..., h:2 * h] = np.abs(dy[..., :h]) + np.abs(dy[..., h:2 * h])
    e = m * (2.0 ** -22 + 4 * U32)                                  # of dn
    if gain is None:
        return dn, e, None, None
    inv = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    u, eu = dn * gain, (e + np.abs(dn) * 2 * U32) * np.abs(gain)
    dot = (u * x).mean(-1, keepdims=True)
    edot = (eu * np.abs(x)).mean(-1, keepdims=True) + (D + 4) * U32 * np.abs(u * x).mean(-1, keepdims=True)
    dx = inv * (u - x * inv ** 2 * dot)
    edx = inv * (eu + np.abs(x) * inv ** 2 * (edot + (3 * D + 30) * U32 * np.abs(dot)) + (D + 12) * U32 * (np.abs(u) + np.abs(x) * inv ** 2 * np.abs(dot)))
    terms = dn * x * inv
    dg = terms.sum((0, 1, 2))
    edg = (e * np.abs(x) * inv).sum((0, 1, 2)) + (terms.shape[0] * terms.shape[1] * terms.shape[2] + D + 16) * U32 * np.abs(terms).sum((0, 1, 2))
    return dx, edx, dg, edg


def seen(at, total, n, left, right, sinks):
    """[len(at), n] whether a frame at position at[i] sees frame s < n, of which `total` exist"""
    s, p = np.arange(n)[None], np.asarray(at)[:, None]
    m = s < total
    if right is not None:
        m = m & (s <= p + right)
    if left is not None:
        m = m & ((s >= p - left) | (s < sinks))
    return m


def _probabilities(q, k, m, scale, kind):
    """(S, P, row logarithms, relative bound of P without its rounding) of [T, D], [n, D] and what is seen"""
    S = scale * (q @ k.T)
    eS = (q.shape[1] + 2) * U32 * scale * (np.abs(q) @ np.abs(k).T)
    S = np.where(m, S, -np.inf)
    top = S.max(-1, keepdims=True)
    e = np.exp(S - top)
    L = (top + np.log(e.sum(-1, keepdims=True)))[:, 0]
    big = np.where(m, np.abs(S), 0).max(-1, keepdims=True)
    eP = 2 * np.where(m, eS, 0).max(-1, keepdims=True) + 4 * U32 * big + 2.0 ** -21
    return S, e / e.sum(-1, keepdims=True), L, eP


def attention(q, k, v, m, scale, kind):
    """(y, bound before the last rounding, L, its bound) of one head's q [T, D], k, v [n, D] and m [T, n] what is seen"""
    S, P, L, eP = _probabilities(q, k, m, scale, kind)
    v = np.where(m.any(0)[:, None], v, 0.0)
    y, mag = P @ v, P @ np.abs(v)
    n = m.sum(-1, keepdims=True)
    e = mag * (2 * eP + HALF[kind] + (2 * n + 16) * U32 + 3 * 2.0 ** -21)
    if kind == "f16":
        e = e + 2.0 ** -25 * (m @ np.abs(v))
    return y, e, L, eP[:, 0] + (n[:, 0] + 8) * U32 + 4 * U32 * (np.abs(L) + 1) + 2.0 ** -21


def attention_grad(dy, q, k, v, y, L, m, scale, kind):
    """((dq, bound), (dk, bound), (dv, bound)) of one head, y and L given"""
    S, _, _, eP = _probabilities(q, k, m, scale, kind)
    D = q.shape[1]
    P = np.where(m, np.exp(np.where(m, S, 0) - L[:, None]), 0.0)
    eP = eP + 2 * U32 * np.abs(L)[:, None]
    dP, mdP = dy @ v.T, np.abs(dy) @ np.abs(v).T
    delta, mdelta = (dy * y).sum(-1, keepdims=True), (np.abs(dy) * np.abs(y)).sum(-1, keepdims=True)
    dS = P * (dP - delta)
    edS = np.abs(dS) * (eP + HALF[kind] + 4 * U32) + P * (D + 4) * U32 * (mdP + mdelta)
    eW = P * (eP + HALF[kind])
    if kind == "f16":
        edS, eW = edS + 2.0 ** -25 * m, eW + 2.0 ** -25 * m
    # (a probability, or a product's operand, below 2^-126 comes out as zero)
    edS, eW = edS + 2.0 ** -126 * m * (1 + mdP + mdelta), eW + 2.0 ** -126 * m
    n, t = m.shape[1], m.shape[0]
    return ((scale * dS @ k, scale * (edS @ np.abs(k) + (n + 4) * U32 * np.abs(dS) @ np.abs(k))),
            (scale * dS.T @ q, scale * (edS.T @ np.abs(q) + (t + 4) * U32 * np.abs(dS).T @ np.abs(q))),
            (P.T @ dy, eW.T @ np.abs(dy) + (t + 4) * U32 * P.T @ np.abs(dy)))


def whole_attention(q, k, v, D, lengths, left, right, sinks, scale, kind):
    """y, bound, L, bound of [B, T, columns] in float64; frames that do not exist: zeros"""
    B, T = q.shape[:2]
    n, there = frames_there(B, T, lengths)
    q, k, v = split(q, D), split(k, D), split(v, D)
    H, G = q.shape[2], k.shape[2]
    y, e, L, eL = np.zeros(q.shape), np.zeros(q.shape), np.zeros((B, T, H)), np.zeros((B, T, H))
    for b in range(B):
        m = seen(np.arange(n[b]), n[b], n[b], left, right, sinks)
        for h in range(H if n[b] else 0):
            g, w = h // (H // G), slice(0, n[b])
            y[b, w, h], e[b, w, h], L[b, w, h], eL[b, w, h] = attention(q[b, w, h], k[b, w, g], v[b, w, g], m, scale, kind)
    return y.reshape(B, T, -1), e.reshape(B, T, -1), L, eL


def whole_attention_grad(dy, q, k, v, y, L, D, lengths, left, right, sinks, scale, kind):
    """[(gradient, bound before the last rounding)] of q, k and v"""
    B, T = q.shape[:2]
    n, _ = frames_there(B, T, lengths)
    dy, q, k, v, y = (split(x, D) for x in (dy, q, k, v, y))
    H, G = q.shape[2], k.shape[2]
    out = [[np.zeros(x.shape), np.zeros(x.shape)] for x in (q, k, v)]
    for b in range(B):
        m, w = seen(np.arange(n[b]), n[b], n[b], left, right, sinks), slice(0, n[b])
        for h in range(H if n[b] else 0):
            g = h // (H // G)
            one = attention_grad(dy[b, w, h], q[b, w, h], k[b, w, g], v[b, w, g], y[b, w, h], L[b, w, h], m, scale, kind)
            for (x, e), (got, bound), at in zip(out, one, (h, g, g)):
                x[b, w, at] += got
                e[b, w, at] += bound + H // G * U32 * np.abs(got)
    return [(x.reshape(B, T, -1), e.reshape(B, T, -1)) for x, e in out]


def cached_frames(pages, table, n):
    """[n, kv_heads, D] of one item's frames from pages [pages, kv_heads, page, D]"""
    P = pages.shape[2]
    return np.stack([pages[table[s // P], :, s % P] for s in range(n)]) if n else np.zeros((0, pages.shape[1], pages.shape[3]))


def whole_cached(q, pages_k, pages_v, table, used, lengths, left, right, sinks, scale, kind):
    """y, bound of new frames [B, T, columns]"""
    D = pages_k.shape[3]
    B, T = q.shape[:2]
    n, _ = frames_there(B, T, lengths)
    q = split(q, D)
    H, G = q.shape[2], pages_k.shape[1]
    y, e = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(B):
        total = used[b] + n[b]
        if n[b] == 0:
            continue
        k, v = (cached_frames(p, table[b], total) for p in (pages_k, pages_v))
        m = seen(used[b] + np.arange(n[b]), total, total, left, right, sinks)
        for h in range(H):
            g, w = h // (H // G), slice(0, n[b])
            y[b, w, h], e[b, w, h], _, _ = attention(q[b, w, h], k[:, g], v[:, g], m, scale, kind)
    return y.reshape(B, T, -1), e.reshape(B, T, -1)


def rounded(e, want, kind):
    """A bound with the result's last rounding, of a value that is itself off by e."""
    return e * (1 + HALF[kind]) + rounding(want, kind)
