"""Cross attention in 64 bits, and how far a result of the library may be from it: bounds from the roundings that its kernels make, none measured."""
from __future__ import annotations

import numpy as np

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}     # half a step, relative to the value
U = 2.0 ** -24


def visible(B, M, kv_len, mask):
    v = np.ones((B, M), dtype=bool)
    if kv_len is not None:
        v &= np.arange(M) < np.clip(np.asarray(kv_len), 0, M)[:, None]
    if mask is not None:
        v &= np.asarray(mask) != 0
    return v


def _weight_step(dtype, few):
    """What is lost of a weight (P, dS) on its way into a product: bfloat16's half step; where few rows add up, that of a second number that holds the first's remainder."""
    return 0.0 if dtype != "bf16" else HALF[dtype] ** 2 if few else HALF[dtype]


def _scores(q, k, scale):
    """Scores and a bound of their error: d products and their sums in 32 bits, then the scale and the exponent's multiply-add."""
    s = q @ k.T * scale
    off = (q.shape[1] + 4) * U * scale * (np.abs(q) @ np.abs(k).T) + 4 * U * np.abs(s)
    return s, off


def forward(Q, K, V, vis, scale, dtype):
    """O, lse, and bounds of both. Weights are rounded for the second product."""
    B, Hq, N, d = Q.shape
    M = K.shape[2]
    O, lse = np.zeros((B, Hq, N, d)), np.full((B, Hq, N), -np.inf)
    bO, bl = np.zeros_like(O), np.zeros((B, Hq, N))
    w = _weight_step(dtype, False)
    for b in range(B):
        j = np.nonzero(vis[b])[0]
        if len(j) == 0:
            continue
        for h in range(Hq):
            hk = h * K.shape[1] // Hq
            k, v = K[b, hk, j], V[b, hk, j]
            s, off = _scores(Q[b, h], k, scale)
            top = s.max(1, keepdims=True)
            e = np.exp(s - top)
            l = e.sum(1, keepdims=True)
            p = e / l
            O[b, h], lse[b, h] = p @ v, (top + np.log(l))[:, 0]
            delta = off.max(1, keepdims=True) + 8 * U * (1 + np.abs(s).max(1, keepdims=True))
            size = p @ np.abs(v)
            bO[b, h] = size * (w + 2 * delta + (M + 8) * U) + HALF[dtype] * np.abs(O[b, h])
            bl[b, h] = delta[:, 0] + (M + 8) * U + 4 * U * np.abs(lse[b, h])
    return O, lse, 1.01 * bO + 1e-30, 1.01 * bl


def backward(Q, K, V, O, lse, dO, vis, scale, dtype):
    """dQ, dK, dV from the outputs and statistics that the call is given, and their bounds. P and dS are rounded where a product consumes them."""
    B, Hq, N, d = Q.shape
    Hkv, M = K.shape[1], K.shape[2]
    rows, half = Hq // Hkv * N, HALF[dtype]
    wq, wk = _weight_step(dtype, rows <= 64), _weight_step(dtype, rows <= 32)
    dQ, dK, dV = np.zeros(Q.shape), np.zeros(K.shape), np.zeros(K.shape)
    bQ, bK, bV = np.zeros(Q.shape), np.zeros(K.shape), np.zeros(K.shape)
    terms = N * (Hq // Hkv) + 40
    for b in range(B):
        j = np.nonzero(vis[b])[0]
        if len(j) == 0:
            continue
        for h in range(Hq):
            hk = h * Hkv // Hq
            q, k, v, g, l = Q[b, h], K[b, hk, j], V[b, hk, j], dO[b, h], lse[b, h][:, None]
            s, off = _scores(q, k, scale)
            seen = np.isfinite(l)
            p = np.where(seen, np.exp(s - np.where(seen, l, 0.0)), 0.0)
            eps = off + 8 * U * (1 + np.abs(s) + np.abs(np.where(seen, l, 0.0)))
            dp, D = g @ v.T, (g * O[b, h]).sum(1, keepdims=True)
            edp = (d + 4) * U * (np.abs(g) @ np.abs(v).T + (np.abs(g) * np.abs(O[b, h])).sum(1, keepdims=True))
            ds = p * (dp - D)
            eds = p * (np.abs(dp - D) * (2 * eps + 4 * U) + edp * (1 + 2 * eps))
            edsq, edsk = (eds + w * np.abs(ds) * (1 + 2 * eps) for w in (wq, wk))
            dQ[b, h] = ds @ k * scale
            bQ[b, h] = scale * ((edsq + (M + 8) * U * np.abs(ds)) @ np.abs(k)) + half * np.abs(dQ[b, h])
            dK[b, hk, j] += ds.T @ q * scale
            bK[b, hk, j] += scale * ((edsk + terms * U * np.abs(ds)).T @ np.abs(q))
            dV[b, hk, j] += p.T @ g
            bV[b, hk, j] += (p * (wk + 2 * eps + terms * U)).T @ np.abs(g)
    bK += half * np.abs(dK)
    bV += half * np.abs(dV)
    return (dQ, dK, dV), tuple(1.01 * x + 1e-30 for x in (bQ, bK, bV))
