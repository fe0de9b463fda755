"""The operators around the attention in fp64 numpy -- TEST INFRASTRUCTURE, NOT PRODUCT CODE.

Written from the formulas, row by row and key by key; inputs are upcast to fp64 exactly.  Layouts as in the C ABI: token-major
[B,N,heads,d] on the projection's side, head-major [B,heads,N,d] on the attention's.
"""
from __future__ import annotations

import numpy as np


def _pairs(d: int, rot: int, paired: bool):
    """(i, j) index arrays of the rotated pairs; pair m turns by freq[m]."""
    m = np.arange(rot // 2)
    return (2 * m, 2 * m + 1) if paired else (m, m + rot // 2)


def rotate(x, pos, freq, paired: bool, back: bool = False):
    """Rows x [..., d] at positions pos [...] turned pair by pair."""
    x = np.array(x, dtype=np.float64)
    if freq is None:
        return x
    freq = np.asarray(freq, dtype=np.float64)
    i, j = _pairs(x.shape[-1], 2 * len(freq), paired)
    a = np.asarray(pos, dtype=np.float64)[..., None] * freq
    c, s = np.cos(a), np.sin(a) * (-1 if back else 1)
    xi, xj = x[..., i].copy(), x[..., j].copy()
    x[..., i] = xi * c - xj * s
    x[..., j] = xi * s + xj * c
    return x


def _rms(x, eps: float):
    return 1.0 / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)


def norm_rope_rows(x, weight, eps, norm: bool, pos, freq, paired: bool):
    """y of rows x [..., heads, d] at positions pos [...]."""
    x = np.asarray(x, dtype=np.float64)
    if norm:
        x = x * _rms(x, eps) * (1.0 if weight is None else np.asarray(weight, dtype=np.float64))
    return rotate(x, np.broadcast_to(np.asarray(pos)[..., None], x.shape[:-1]), freq, paired)


def norm_rope_rows_backward(x, weight, eps, norm: bool, pos, freq, paired: bool, dy):
    """(dx, dweight) of norm_rope_rows; dweight None without the norm."""
    x, dy = np.asarray(x, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    g = rotate(dy, np.broadcast_to(np.asarray(pos)[..., None], x.shape[:-1]), freq, paired, back=True)
    if not norm:
        return g, None
    r = _rms(x, eps)
    u = x * r
    dweight = (g * u).reshape(-1, x.shape[-1]).sum(0)
    gw = g * (1.0 if weight is None else np.asarray(weight, dtype=np.float64))
    return r * (gw - u * np.mean(gw * u, axis=-1, keepdims=True)), dweight


def append_paged(q, k, v, wq, wk, eps, norm, freq, paired, alpha, start, cached, table, Q, Kp, Vp, cp):
    """The state after the call: (Q, Kp, Vp, cp) as fp64 copies.  q, alpha may be None (Q, cp come back as they were given)."""
    Q, Kp, Vp, cp = (None if x is None else np.array(x, dtype=np.float64) for x in (Q, Kp, Vp, cp))
    pages, page = Kp.shape[0], Kp.shape[2]
    M = table.shape[1]

    def page_of(b, p):
        if p < 0 or p >= M * page:
            return -1
        at = int(table[b, p // page])
        return at if 0 <= at < pages else -1

    for b in range(len(cached)):
        before = int(cached[b])
        prev = page_of(b, before - 1)
        total = cp[prev, :, (before - 1) % page].copy() if alpha is not None and prev >= 0 else 0.0
        for n in range(int(start[b]), int(start[b + 1])):
            p = before + n - int(start[b])
            if q is not None:
                Q[n] = norm_rope_rows(q[n], wq, eps, norm, p, freq, paired)
            at = page_of(b, p)
            if alpha is not None:
                total = total + np.asarray(alpha[n], dtype=np.float64)
            if at < 0:
                continue
            Kp[at, :, p % page] = norm_rope_rows(k[n], wk, eps, norm, p, freq, paired)
            Vp[at, :, p % page] = v[n]
            if alpha is not None:
                cp[at, :, p % page] = total
    return Q, Kp, Vp, cp


def decode_paged(q, Kp, Vp, cp, table, pos, w: int, scale: float, detail: bool = False):
    """o [B,H,d], L [B,H]; with `detail` also sum_i p_i |v_i| [B,H,d], the largest scale * sum |q||k| and the largest |S| over the keys [B,H] and
    the number of keys [B]."""
    B, H, d = q.shape
    pages, Hkv, page, _ = Kp.shape
    T = table.shape[1] * page
    o, L = np.zeros((B, H, d)), np.full((B, H), -np.inf)
    absv, dots, top, count = np.zeros((B, H, d)), np.zeros((B, H)), np.zeros((B, H)), np.zeros(B, dtype=int)
    for b in range(B):
        p = min(int(pos[b]), T - 1)
        if p < 0 or not 0 <= int(table[b, p // page]) < pages:
            continue
        i = np.arange(max(0, p - w + 1), p + 1)
        at = table[b, i // page].astype(np.int64)
        there = (at >= 0) & (at < pages)
        i, at = i[there], at[there]
        count[b] = len(i)
        for h in range(H):
            kh = h // (H // Hkv)
            K, V = (x[at, kh, i % page].astype(np.float64) for x in (Kp, Vp))
            c = cp[at, h, i % page].astype(np.float64)
            qh = np.asarray(q[b, h], dtype=np.float64)
            with np.errstate(invalid="ignore", over="ignore"):
                S = scale * (K @ qh) + (c - float(cp[int(table[b, p // page]), h, p % page]))
            m = S.max()
            if m == -np.inf:  # every score masked: no softmax; an empty row
                continue
            e = np.exp(S - m)
            L[b, h] = m + np.log(e.sum())
            P = e / e.sum()
            o[b, h] = P @ V
            absv[b, h] = P @ np.abs(V)
            fin = S > -1e30
            dots[b, h] = (scale * (np.abs(K) @ np.abs(qh)))[fin].max()
            top[b, h] = np.abs(S[fin]).max()
    return (o, L, absv, dots, top, count) if detail else (o, L)
