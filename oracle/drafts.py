"""TEST INFRASTRUCTURE: a drafted step written out from its definitions (numpy, 64 bits, plain loops): rotary positions, attention of a tree of drafted tokens over
what the 4-bit cache holds, verification of drafts.  Shares no code with the GPU path."""
from __future__ import annotations

import math

import numpy as np

from oracle import kv4
from oracle.attention import bf16_to_f64

PLAIN, LINEAR, BANDS, RAMP = range(4)


def frequencies(rot, base=10000.0, scaling=PLAIN, factor=1.0, context=0.0, low=0.0, high=0.0):
    """(radians a position of every pair, magnitude)."""
    out, magnitude = [], 1.0
    a = b = 0.0
    if scaling == RAMP:
        def place(turns):
            return rot * math.log(context / (2 * math.pi * turns)) / (2 * math.log(base))
        a, b = max(0, math.floor(place(high))), min(rot - 1, math.ceil(place(low)))
        magnitude = 0.1 * math.log(factor) + 1
    for i in range(rot // 2):
        f = base ** (-2 * i / rot)
        if scaling == LINEAR:
            f = f / factor
        elif scaling == BANDS:
            t = context * f / (2 * math.pi)
            f = f / factor if t <= low else f if t >= high else f / factor + (f - f / factor) * (t - low) / (high - low)
        elif scaling == RAMP:
            share = 0.0 if i <= a else 1.0 if i >= b else (i - a) / (b - a)
            f = f / factor * share + f * (1 - share)
        out.append(f)
    return np.array(out), magnitude


def rotate(x, pos, freq, magnitude=1.0, pairs=False):
    """x [n][H][D] float64 turned to pos [n]; pairs (2 i, 2 i + 1) or (i, i + rot / 2)."""
    y = np.array(x, dtype=np.float64)
    half = len(freq)
    for t in range(len(pos)):
        for i, f in enumerate(freq):
            a, b = (2 * i, 2 * i + 1) if pairs else (i, i + half)
            c, s = magnitude * math.cos(float(pos[t]) * f), magnitude * math.sin(float(pos[t]) * f)
            y[t, :, a], y[t, :, b] = x[t, :, a] * c - x[t, :, b] * s, x[t, :, b] * c + x[t, :, a] * s
    return y


def ancestors(parent, n):
    """[n][n] truth values: token i sees itself and what its chain of parents names."""
    sees = np.zeros((n, n), dtype=bool)
    for i in range(n):
        p = i - 1 if parent is None else int(parent[i])
        if 0 <= p < i:
            sees[i] = sees[p]
        sees[i, i] = True
    return sees


def tree(Q, K, V, cache, off, parent, G, row=None, scale=None):
    """Q [tokens][H_q][D], K and V [tokens][H_kv][D] bf16 bits; cache(r, h) -> (keys, values) float64 [n][D] of table row r.  (outputs, sum p |v|, the largest sum over d of
    |q| |k| of a row) in float64; tokens outside `off` are NaN."""
    Qf, Kf, Vf = bf16_to_f64(Q), bf16_to_f64(K), bf16_to_f64(V)
    n, H_q, D = Qf.shape
    scale = 1 / math.sqrt(D) if scale is None else scale
    out, mass, reach = (np.full(Qf.shape, np.nan) for _ in range(3))
    for s in range(len(off) - 1):
        a, b = int(off[s]), int(off[s + 1])
        sees = ancestors(None if parent is None else parent[a:b], b - a)
        for h in range(H_q // G):
            k0, v0 = cache(s if row is None else int(row[s]), h)
            for i in range(b - a):
                at = a + np.flatnonzero(sees[i])
                k, v = np.concatenate([k0, Kf[at, h]]), np.concatenate([v0, Vf[at, h]])
                for hq in range(h * G, (h + 1) * G):
                    q = Qf[a + i, hq]
                    with np.errstate(invalid="ignore", over="ignore"):
                        x = (k @ q) * scale
                        p = np.exp(x - x.max())
                        p /= p.sum()
                        out[a + i, hq], mass[a + i, hq] = p @ v, p @ np.abs(v)
                        reach[a + i, hq] = (np.abs(k) @ np.abs(q)).max() * scale
    return out, mass, reach


def verify(P, Q, token, parent, off, u, u_next, distinct=False, vocab=None, most=64):
    """(accepted [n], next [requests], new_off, rows): P, Q [tokens][vocab] float64 (Q None: drafts that were not drawn)."""
    n = len(token)
    accepted, nxt = np.zeros(n, dtype=np.int32), np.full(len(off) - 1, -1, dtype=np.int32)
    vocab = P.shape[1]
    for s in range(len(off) - 1):
        a, b = int(off[s]), int(off[s + 1])
        if a == b:
            continue
        m = min(b - a, most)
        hand, accepted[a] = 0, 1
        r, tried, left = P[a].copy(), [], 1.0                   # left: of q's sum, without the tokens tried
        for i in range(1, m):
            p = i - 1 if parent is None else int(parent[a + i])
            x = int(token[a + i])
            if p != hand or not 0 <= p < i or not 0 <= x < vocab or left == 0:      # (nothing of q is left: no draft of it)
                continue
            if Q is None:
                q = np.zeros(vocab)
                q[x] = 1.0
            else:
                q = Q[a + hand].copy()
                if distinct:
                    q[tried] = 0.0
                    q = q / left
            if float(u[a + i]) * q[x] < r[x]:
                hand, accepted[a + i] = i, 1
                r, tried, left = P[a + i].copy(), [], 1.0
                continue
            if Q is None:
                rest = r.copy()
                rest[x] = 0.0
            else:
                rest = np.maximum(r - q, 0.0)
            total = rest.sum()
            if total > 0:
                r = rest / total
            if distinct and x not in tried:
                tried.append(x)
                if Q is not None:                               # from the entries that are left, never as 1 - those tried: they are rounded, and may be nearly all there is
                    rest = Q[a + hand].copy()
                    rest[tried] = 0.0
                    left = rest.sum() / (rest.sum() + Q[a + hand, tried].sum()) if rest.sum() > 0 else 0.0
        up = np.cumsum(r)
        if up[-1] > 0:
            nxt[s] = int(np.flatnonzero((up > float(u_next[s]) * up[-1]) & (r > 0))[0])
    new = np.concatenate([[0], np.cumsum(accepted)]).astype(np.int32)
    rows = np.full(n, -1, dtype=np.int32)
    where = np.flatnonzero(accepted)
    rows[:len(where)] = where
    return accepted, nxt, new[np.asarray(off)], rows


def cache_of(pages, D, page_of, length):
    """cache(r, h) for tree(): what ag_kv4_load gives of the row's tokens, those on pages outside the pool left out."""
    K, V = kv4.load(pages, D, np.arange(pages.shape[0] * kv4.PAGE))

    def cache(r, h):
        if r < 0 or r >= len(length):
            return np.zeros((0, D)), np.zeros((0, D))
        n = min(max(int(length[r]), 0), page_of.shape[1] * kv4.PAGE)
        p = np.repeat(page_of[r].astype(np.int64), kv4.PAGE)[:n]
        slots = (p * kv4.PAGE + np.arange(n) % kv4.PAGE)[(p >= 0) & (p < pages.shape[0])]
        return K[slots, h], V[slots, h]
    return cache
