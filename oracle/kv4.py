"""TEST INFRASTRUCTURE: the paged 4-bit key/value cache written out from its definition (numpy, 64 bits, plain loops).

Quantisation of a group of 32 elements x: lo = min, hi = max, s = bf16((hi - lo) / 15) with the subtraction and the division rounded to
32 bits, code = rint((x - lo) / s) clamped to 0..15 (0 when s = 0); an element stands for s * code + lo.  A group with a value that is
not finite (or whose hi - lo is not) stands for NaN.

Layout of a KV head's block of 80 D bytes: see byte_of below.  Tables: page_of [rows][max_pages] (-1 = none), length [rows],
refs [pages]; the functions change them in place, request after request.
"""
from __future__ import annotations

import math

import numpy as np

from oracle.attention import bf16_to_f64

PAGE = 64


def f32_to_bf16_value(v):
    """Nearest bf16 (ties to even) of a float32, as a float32."""
    u = np.asarray(v, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return (((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32)


def bf16_bits(v):
    return (np.asarray(v, dtype=np.float32).view(np.uint32) >> 16).astype(np.uint16)


def quantise(bits):
    """bits [..., D] bf16 patterns -> codes [..., D] (0..15), scale and base [..., D / 32] float32 (bf16 values)."""
    x = bf16_to_f64(bits).astype(np.float32)
    g = x.reshape(*x.shape[:-1], -1, 32)
    codes = np.zeros(g.shape, dtype=np.int64)
    scale = np.zeros(g.shape[:-1], dtype=np.float32)
    base = np.zeros(g.shape[:-1], dtype=np.float32)
    with np.errstate(over="ignore", invalid="ignore"):
        for at in np.ndindex(*g.shape[:-1]):
            v = g[at]
            lo, hi = v.min(), v.max()
            s = f32_to_bf16_value(np.float32(np.float32(hi - lo) / np.float32(15))) if np.isfinite(v).all() and np.isfinite(hi - lo) else np.float32(np.nan)
            scale[at], base[at] = s, lo if np.isfinite(s) else np.nan
            if np.isfinite(s) and s > 0:
                codes[at] = np.clip(np.rint((v - lo) / s), 0, 15).astype(np.int64)
    return codes.reshape(x.shape), scale, base


def values(codes, scale, base):
    """What codes stand for, in float64."""
    return codes.astype(np.float64) * np.repeat(scale.astype(np.float64), 32, -1) + np.repeat(base.astype(np.float64), 32, -1)


def byte_of(D, which, token, d):
    """(byte inside the head's block, high nibble?) of element d of token `token`'s key (which = 0) or value (1) row."""
    run, h = token // 16, token % 16 // 8
    at = which * 32 * D + run * 8 * D + h * 4 * D
    if which == 0:
        g, q, t, i = token % 8, d // 32, d % 32 // 8, d % 8
        return at + (4 * g + t) * (D // 8) + 4 * q + i // 2, i % 2
    t, e = token % 8 // 2, token % 2
    i, j, g = d // 16, d % 16 // 8, d % 8
    return at + (4 * g + t) * (D // 8) + e * (D // 16) + j * (D // 32) + i // 2, i % 2


def scale_byte(D, which, token, group):
    return 64 * D + which * 8 * D + (token * (D // 32) + group) * 4


def store(pages, D, K, V, slot):
    """pages [n][H_kv][80 D] uint8, K and V [tokens][H_kv][D] bf16 bits."""
    for which, rows in enumerate((K, V)):
        codes, scale, base = quantise(rows)
        for i, s in enumerate(slot):
            if s < 0 or s >= pages.shape[0] * PAGE:
                continue
            for h in range(rows.shape[1]):
                block = pages[s // PAGE, h]
                for d in range(D):
                    byte, high = byte_of(D, which, s % PAGE, d)
                    block[byte] = (block[byte] & (0x0F if high else 0xF0)) | (int(codes[i, h, d]) << (4 * high))
                for g in range(D // 32):
                    at = scale_byte(D, which, s % PAGE, g)
                    pair = np.array([scale[i, h, g], base[i, h, g]], dtype=np.float32)
                    block[at:at + 4] = (np.array([0x7FC0, 0x7FC0], dtype=np.uint16) if np.isnan(pair).any() else bf16_bits(pair)).view(np.uint8)


def load(pages, D, slots):
    """float64 (K, V), each [tokens][H_kv][D]."""
    out = []
    d = np.arange(D)
    for which in (0, 1):
        rows = np.zeros((len(slots), pages.shape[1], D))
        for i, s in enumerate(slots):
            r = s % PAGE
            byte = np.array([byte_of(D, which, r, x)[0] for x in d])
            high = np.array([byte_of(D, which, r, x)[1] for x in d])
            for h in range(pages.shape[1]):
                block = pages[s // PAGE, h]
                codes = (block[byte] >> (4 * high)) & 15
                at = scale_byte(D, which, r, 0)
                sb = bf16_to_f64(block[at:at + D // 8].copy().view(np.uint16)).reshape(-1, 2)
                rows[i, h] = codes * np.repeat(sb[:, 0], 32) + np.repeat(sb[:, 1], 32)
        out.append(rows)
    return out


# ---- tables ------------------------------------------------------------------------------------------------
def _pages(n):
    return -(-n // PAGE)


def _grant(refs, wants):
    """Pages for a list of wants: free pages ascending, request by request, all or nothing; refused requests keep their place.  Who wants none gets none,
    whether there are any or not."""
    free = [p for p in range(len(refs)) if refs[p] <= 0]
    at, out = 0, []
    for w in wants:
        out.append(free[at:at + w] if w == 0 or at + w <= len(free) else None)
        at += w
    for pages in out:
        for p in pages or []:
            refs[p] = 1
    return out


def extend(page_of, length, refs, row, new_off, n_tokens):
    rows, max_pages = page_of.shape
    fine, wants = [], []
    for i, r in enumerate(row):
        fresh = new_off[i + 1] - new_off[i]
        f = 0 <= r < rows and fresh >= 0 and r not in list(row[:i])
        f = f and length[r] + fresh <= max_pages * PAGE
        fine.append(f)
        wants.append(_pages(length[r] + fresh) - _pages(length[r]) if f else 0)
    got = _grant(refs, wants)
    slot, ok = np.full(n_tokens, -1, dtype=np.int32), np.zeros(len(row), dtype=np.int32)
    for i, r in enumerate(row):
        if not fine[i] or got[i] is None:
            continue
        ok[i] = 1
        first = _pages(length[r])
        page_of[r, first:first + wants[i]] = got[i]
        for j in range(new_off[i], new_off[i + 1]):
            pos = length[r] + j - new_off[i]
            if j < n_tokens:
                slot[j] = page_of[r, pos // PAGE] * PAGE + pos % PAGE
        length[r] += new_off[i + 1] - new_off[i]
    return slot, ok


def fork(pages, page_of, length, refs, src, dst):
    rows = page_of.shape[0]
    len0, table0 = length.copy(), page_of.copy()
    fine = [0 <= d < rows and 0 <= s < rows and d != s and len0[d] == 0 and d not in list(dst[:i]) for i, (s, d) in enumerate(zip(src, dst))]
    got = _grant(refs, [1 if f and len0[s] % PAGE else 0 for f, s in zip(fine, src)])
    ok = np.zeros(len(src), dtype=np.int32)
    for i, (s, d) in enumerate(zip(src, dst)):
        if not fine[i] or got[i] is None:
            continue
        ok[i] = 1
        full = len0[s] // PAGE
        page_of[d, :full] = table0[s, :full]
        for p in table0[s, :full]:
            refs[p] += 1
        if len0[s] % PAGE:
            page_of[d, full] = got[i][0]
            pages[got[i][0]] = pages[table0[s, full]]
        length[d] = len0[s]
    return ok


def free(page_of, length, refs, row):
    for r in row:
        if 0 <= r < page_of.shape[0]:
            for p in page_of[r]:
                if p >= 0:
                    refs[p] -= 1
            page_of[r], length[r] = -1, 0


def compact(pages, page_of, refs):
    used = [p for p in range(len(refs)) if refs[p] > 0]
    n = len(used)
    holes = [p for p in range(n) if refs[p] <= 0]
    movers = [p for p in used if p >= n]
    moved = np.full(len(refs), -1, dtype=np.int32)
    for p in used:
        moved[p] = p
    for a, b in zip(movers, holes):
        moved[a] = b
        pages[b] = pages[a]
        refs[b], refs[a] = refs[a], 0
    for at in np.ndindex(*page_of.shape):
        if page_of[at] >= 0:
            page_of[at] = moved[page_of[at]]
    return moved


def decode(Q, pages, D, page_of, length, row=None):
    """Single-token attention over the cache: Q [B][H_q][D] bf16 bits, request b = table row row[b] (default b).  float64."""
    Qf = bf16_to_f64(Q)
    B, H_q, _ = Qf.shape
    H_kv = pages.shape[1]
    out = np.zeros(Qf.shape)
    for b in range(B):
        r = b if row is None else int(row[b])
        if r < 0 or r >= len(length):
            continue
        n = min(max(int(length[r]), 0), page_of.shape[1] * PAGE)
        slots = [int(page_of[r, j // PAGE]) * PAGE + j % PAGE for j in range(n) if 0 <= page_of[r, j // PAGE] < pages.shape[0]]
        if not slots:
            continue
        K, V = load(pages, D, slots)
        for hq in range(H_q):
            h = hq // (H_q // H_kv)
            s = K[:, h] @ Qf[b, hq] / math.sqrt(D)
            p = np.exp(s - s.max())
            out[b, hq] = p @ V[:, h] / p.sum()
    return out
