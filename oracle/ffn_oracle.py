"""The operators of a layer's feed-forward half, from their definitions, in 64 bits (numpy; test infrastructure).

Shares no code with the HIP path: rows and experts are plain loops, weights are made from the caller's codes.
"""
import numpy as np


def residual_norm(residual, y, weight=None, post_weight=None, post_norm=False, gate=None, offset=0.0, eps=1e-6, residual_scale=1.0,
                  block_scale=1.0):
    """float64 rows (or None) -> (x, r', the magnitude of the two terms of r', and that of x's)."""
    def normed(t, w):
        f = 1.0 / np.sqrt((t ** 2).mean(-1, keepdims=True) + eps)
        return f if w is None else f * (w + offset)

    b = np.zeros_like(residual) if y is None else y
    if post_norm:
        b = b * normed(b, post_weight)
    if gate is not None:
        b = b * gate
    old = np.zeros_like(b) if residual is None else residual
    r = residual_scale * old + block_scale * b
    mag = np.abs(residual_scale * old) + np.abs(block_scale * b)
    f = normed(r, weight)
    return r * f, r, mag, mag * np.abs(f)


def route(x, W, top_k, score="softmax", renormalise=True, scale=1.0, choice_bias=None, n_groups=1, top_groups=1, group_top=1):
    """-> (ids, weights, logits, by how much each row's choices are apart: the smallest gap that decided anything)."""
    M, E = x.shape[0], W.shape[0]
    size = E // n_groups
    ids, weights, gaps = np.zeros((M, top_k), int), np.zeros((M, top_k)), np.full(M, np.inf)
    logits = x @ W.T
    for m in range(M):
        l = logits[m]
        p = np.exp(l - l.max()) if score == "softmax" else 1.0 / (1.0 + np.exp(-l))
        if score == "softmax":
            p = p / p.sum()
        c = p if choice_bias is None else p + choice_bias
        best = [sum(sorted(c[g * size:(g + 1) * size])[::-1][:group_top]) for g in range(n_groups)]
        order = sorted(range(n_groups), key=lambda g: (-best[g], g))
        if top_groups < n_groups:
            gaps[m] = best[order[top_groups - 1]] - best[order[top_groups]]
        free = [e for g in sorted(order[:top_groups]) for e in range(g * size, (g + 1) * size)]
        free.sort(key=lambda e: (-c[e], e))
        for i in range(min(top_k, len(free) - 1)):
            gaps[m] = min(gaps[m], c[free[i]] - c[free[i + 1]])
        ids[m] = free[:top_k]
        w = p[ids[m]]
        weights[m] = scale * (w / w.sum() if renormalise else w)
    return ids, weights, logits, gaps


def dequantise(codes, scales, G, zero):
    """codes [K, N], scales [K/G, N] float64 -> weights."""
    return (codes.astype(np.float64) - zero) * np.repeat(scales, G, 0)


def experts(x, ids, weights, w1, w2, base=None):
    """w1(e) [hidden, 2 inter] (gate and up by 16 columns), w2(e) [inter, hidden]: functions of an expert -> (Y, a bound on what
    the roundings and sums inside may add up to: the magnitude of the terms, that of h's error with them)."""
    M, k = ids.shape
    y = np.zeros(x.shape) if base is None else base.copy()
    mag, h_err = np.abs(y), np.zeros(x.shape)
    for e in sorted(set(ids.ravel().tolist())):
        w = w1(e)
        if w is None:                                         # no such expert
            continue
        z = (x @ w).reshape(M, -1, 2, 16)
        zm = (np.abs(x) @ np.abs(w)).reshape(M, -1, 2, 16)
        g, u = z[:, :, 0], z[:, :, 1]
        sig = 1.0 / (1.0 + np.exp(-g))
        h = (g * sig * u).reshape(M, -1)
        # |d silu| <= 1.1 |dg|: what an error of one unit of the sums' magnitude does to h
        hm = (1.1 * zm[:, :, 0] * np.abs(u) + np.abs(g * sig) * zm[:, :, 1]).reshape(M, -1)
        down = w2(e)
        for j in range(k):
            rows = ids[:, j] == e
            f = weights[rows, j:j + 1]
            y[rows] += f * (h[rows] @ down)
            mag[rows] += np.abs(f) * (np.abs(h[rows]) @ np.abs(down))
            h_err[rows] += np.abs(f) * (hm[rows] @ np.abs(down))
    return y, mag, h_err
