"""TEST INFRASTRUCTURE: fp64 oracle of grouped-query attention decode (one query token per request).

The paper schedules attention kernels (MHA / GQA / MLA, prefill and decode) the same way as its GEMMs
(Section 7.1.2; workload appendix: decode processes S_q = 1 query token per request against a KV sequence of
S_k tokens, H_kv = 8 KV heads for GQA, head dimension D = 128, KV working set 4 B S_k H_kv D bytes).  What such a
kernel computes has a plain definition, written out here:

    for request b, query head hq (its KV head is h = hq // (H_q / H_kv)):
        s_j = (q . k_j) / sqrt(D)            for the first len_b keys of (b, h)
        p_j = exp(s_j - max_j s_j) / sum_j exp(s_j - max_j s_j)
        o   = sum_j p_j v_j

Inputs are bf16 bit patterns (numpy uint16); everything is computed in float64.
"""
from __future__ import annotations

import math

import numpy as np


def bf16_to_f64(bits) -> np.ndarray:
    b = np.ascontiguousarray(bits, dtype=np.uint16)
    return (b.astype(np.uint32) << np.uint32(16)).view(np.float32).astype(np.float64)


def gqa_decode(Q, K, V, kv_len=None) -> np.ndarray:
    """Q [B, Hq, D], K and V [B, Hkv, L, D] as bf16 bits; kv_len [B] (default: L for every request).
    Returns O [B, Hq, D] in float64.  A request with kv_len 0 gives zeros."""
    Q, K, V = bf16_to_f64(Q), bf16_to_f64(K), bf16_to_f64(V)
    B, Hq, D = Q.shape
    _, Hkv, L, _ = K.shape
    assert K.shape == V.shape == (B, Hkv, L, D) and Hq % Hkv == 0
    group = Hq // Hkv
    lens = np.full(B, L, dtype=np.int64) if kv_len is None else np.asarray(kv_len, dtype=np.int64)
    O = np.zeros((B, Hq, D), dtype=np.float64)
    scale = 1.0 / math.sqrt(D)
    for b in range(B):
        n = int(lens[b])
        if n == 0:
            continue
        for hq in range(Hq):
            h = hq // group
            s = (K[b, h, :n] @ Q[b, hq]) * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            O[b, hq] = p @ V[b, h, :n]
    return O


def gqa_decode_loops(Q, K, V, kv_len=None) -> np.ndarray:
    """The same definition with nothing but scalar Python arithmetic (tiny cases only)."""
    Q, K, V = bf16_to_f64(Q), bf16_to_f64(K), bf16_to_f64(V)
    B, Hq, D = Q.shape
    _, Hkv, L, _ = K.shape
    group = Hq // Hkv
    O = np.zeros((B, Hq, D), dtype=np.float64)
    for b in range(B):
        n = L if kv_len is None else int(kv_len[b])
        for hq in range(Hq):
            h = hq // group
            s = []
            for j in range(n):
                acc = 0.0
                for t in range(D):
                    acc += float(Q[b, hq, t]) * float(K[b, h, j, t])
                s.append(acc / math.sqrt(D))
            if not s:
                continue
            m = max(s)
            e = [math.exp(x - m) for x in s]
            z = sum(e)
            for t in range(D):
                O[b, hq, t] = sum(e[j] * float(V[b, h, j, t]) for j in range(n)) / z
    return O


def prompt(Q, K, V, q_off, kv_off=None, causal=True, scale=None):
    """Attention over packed sequences.  Q [Tq, Hq, D], K and V [Tk, Hkv, D] as bf16 bits; sequence i owns tokens
    q_off[i] .. q_off[i + 1] - 1 and keys kv_off[i] .. kv_off[i + 1] - 1 (default: the same).  Causal: query i of n sees keys 0 .. m - n + i
    of m.  Returns (O, mass) in float64, mass = sum_j p_j |v_j|; a row that sees no key, or belongs to no sequence, gives zeros."""
    Q, K, V = bf16_to_f64(Q), bf16_to_f64(K), bf16_to_f64(V)
    kv_off = q_off if kv_off is None else kv_off
    group = Q.shape[1] // K.shape[1]
    scale = 1.0 / math.sqrt(Q.shape[2]) if scale is None else scale
    O, mass = np.zeros(Q.shape), np.zeros(Q.shape)
    for a, b, c, d in zip(q_off[:-1], q_off[1:], kv_off[:-1], kv_off[1:]):
        n, m = b - a, d - c
        if n <= 0 or m <= 0:
            continue
        sees = np.arange(m)[None] <= (m - n + np.arange(n))[:, None] if causal else np.ones((n, m), dtype=bool)
        some = sees.any(axis=1)
        for hq in range(Q.shape[1]):
            h = hq // group
            s = np.where(sees, (Q[a:b, hq] @ K[c:d, h].T) * scale, -np.inf)[some]
            p = np.exp(s - s.max(axis=1, keepdims=True))
            p /= p.sum(axis=1, keepdims=True)
            O[a:b, hq][some] = p @ V[c:d, h]
            mass[a:b, hq][some] = p @ np.abs(V[c:d, h])
    return O, mass
