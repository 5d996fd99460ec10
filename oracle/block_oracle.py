"""The operators between the projections, from their definitions, in 64 bits (numpy; test infrastructure).

Shares no code with the HIP path: frequencies are floating numbers here, adapters, pages and masks plain loops.
"""
import math

import numpy as np


def lora(X, A, B, adapter, base, rank=None, scale=None, part_of_column=None, act=0):
    """X [M,K], A [n, P*R, K], B [n, N, R], base [M,N] or None, all float64; returns (Y, magnitude of the terms)."""
    M, N, R = X.shape[0], B.shape[1], B.shape[2]
    part = np.zeros(N, int) if part_of_column is None else np.asarray(part_of_column)
    z = np.zeros((M, N)) if base is None else base.astype(np.float64).copy()
    mag = np.abs(z)
    for m in range(M):
        a = int(adapter[m])
        if not 0 <= a < A.shape[0]:
            continue
        r = R if rank is None else min(max(int(rank[a]), 0), R)
        s = 1.0 if scale is None else float(scale[a])
        for p in np.unique(part):
            rows = slice(p * R, p * R + r)
            cols = part == p
            z[m, cols] += s * (B[a][cols][:, :r] @ (A[a, rows] @ X[m]))
            mag[m, cols] += abs(s) * (np.abs(B[a][cols][:, :r]) @ (np.abs(A[a, rows]) @ np.abs(X[m])))
    if act == 0:
        return z, mag
    sig = lambda t: 1.0 / (1.0 + np.exp(-t))  # noqa: E731
    if act == 1:
        return z * sig(z), 1.1 * mag
    zz, mm = z.reshape(M, N // 32, 2, 16), mag.reshape(M, N // 32, 2, 16)
    g, u = zz[:, :, 0], zz[:, :, 1]
    return (g * sig(g) * u).reshape(M, -1), (1.1 * mm[:, :, 0] * np.abs(u) + (np.abs(g) + mm[:, :, 0]) * mm[:, :, 1]).reshape(M, -1)


def rope_frequencies(rotary_dim, base, scaling=None):
    """Radians per position of every pair."""
    i = np.arange(rotary_dim // 2)
    if scaling and scaling[0] == "ntk":
        base = base * scaling[1] ** (rotary_dim / (rotary_dim - 2.0))
    theta = base ** (-2.0 * i / rotary_dim)
    if scaling and scaling[0] == "linear":
        theta = theta / scaling[1]
    if scaling and scaling[0] == "bands":
        _, factor, original, low, high = scaling
        for p in i:
            u = original * theta[p] / (2 * math.pi)
            w = 0.0 if u <= low else 1.0 if u >= high else (u - low) / (high - low)
            theta[p] = w * theta[p] + (1 - w) * theta[p] / factor
    return theta


def norm_rope(t, weight, eps, theta, interleaved, mscale, positions):
    """t [M, heads, D] float64 -> (the same normed and rotated, a bound on the numbers that are added in each)."""
    t = t.astype(np.float64).copy()
    if weight is not None:
        t = t / np.sqrt((t ** 2).mean(-1, keepdims=True) + eps) * weight
    rd = 0 if theta is None else 2 * len(theta)
    out, mag = t.copy(), np.abs(t)
    for p in range(rd // 2):
        x, y = (2 * p, 2 * p + 1) if interleaved else (p, p + rd // 2)
        for m in range(t.shape[0]):
            ang = math.fmod(float(positions[m]) * theta[p], 2 * math.pi)
            c, s = math.cos(ang) * mscale, math.sin(ang) * mscale
            out[m, :, x] = t[m, :, x] * c - t[m, :, y] * s
            out[m, :, y] = t[m, :, y] * c + t[m, :, x] * s
            mag[m, :, x] = mag[m, :, y] = (np.abs(t[m, :, x]) + np.abs(t[m, :, y])) * abs(mscale)
    return out, mag


def attention(q, k, v, n_drafted, mask, scale):
    """One request: q [T, Hq, D], k and v [L, Hkv, D] float64, mask [T, words] uint64 or None; absent keys are NaN in k.

    Returns (out, lse, sum of p |v|, largest sum of |q||k| * scale)."""
    T, hq, D = q.shape
    L, hkv, _ = k.shape
    out, lse, mag = np.zeros((T, hq, D)), np.full((T, hq), -np.inf), np.zeros((T, hq, D))
    big = 0.0
    for i in range(T):
        seen = []
        for c in range(L):
            j = c - (L - n_drafted)
            if np.isnan(k[c, 0, 0]):
                continue
            if j < 0 or (mask is None and j <= i) or \
                    (mask is not None and j < 64 * mask.shape[1] and int(mask[i, j // 64]) >> (j % 64) & 1):
                seen.append(c)
        if not seen:
            continue
        for h in range(hq):
            kk, vv = k[seen, h * hkv // hq], v[seen, h * hkv // hq]
            s = scale * (kk @ q[i, h])
            big = max(big, float(np.max(np.abs(scale) * (np.abs(kk) @ np.abs(q[i, h])))))
            top = s.max()
            p = np.exp(s - top)
            lse[i, h] = top + math.log(p.sum())
            p /= p.sum()
            out[i, h], mag[i, h] = p @ vv, p @ np.abs(vv)
    return out, lse, mag, big
