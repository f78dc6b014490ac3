"""Pins of the prompt attention's oracle, and the refusals of the entry point that need no device."""
import ctypes as C
import math

import numpy as np

from oracle import attention as oa
from paper_2609_24270_b200 import binding as ag
from paper_2609_24270_b200 import inputs


def rows(n, h, d, seed):
    return inputs.uniform_bf16(n * h, d, seed).reshape(n, h, d)


def test_against_scalar_loops():
    Q, K, V = rows(7, 4, 8, 1), rows(9, 2, 8, 2), rows(9, 2, 8, 3)
    q_off, kv_off = [0, 3, 3, 7], [0, 5, 6, 9]
    Qf, Kf, Vf = (oa.bf16_to_f64(x) for x in (Q, K, V))
    for causal in (True, False):
        got, _ = oa.prompt(Q, K, V, q_off, kv_off, causal)
        for i in range(3):
            n, m = q_off[i + 1] - q_off[i], kv_off[i + 1] - kv_off[i]
            for t in range(n):
                for hq in range(4):
                    keys = [j for j in range(m) if not causal or j <= m - n + t]
                    s = [sum(Qf[q_off[i] + t, hq, e] * Kf[kv_off[i] + j, hq // 2, e] for e in range(8)) / math.sqrt(8) for j in keys]
                    w = [math.exp(v) for v in s]
                    for e in range(8):
                        want = sum(a * Vf[kv_off[i] + j, hq // 2, e] for a, j in zip(w, keys)) / sum(w) if keys else 0.0
                        assert abs(got[q_off[i] + t, hq, e] - want) <= 1e-12


def test_last_token_is_a_decode_step_and_rows_may_see_nothing():
    K, V, Q = rows(20, 2, 16, 4), rows(20, 2, 16, 5), rows(20, 4, 16, 6)
    O, _ = oa.prompt(Q, K, V, [0, 20])
    step = oa.gqa_decode(Q[19:], K.transpose(1, 0, 2)[None], V.transpose(1, 0, 2)[None])
    assert np.abs(O[19] - step[0]).max() <= 1e-12
    assert np.abs(O[0, 3] - oa.bf16_to_f64(V)[0, 1]).max() <= 1e-12     # the first token sees itself
    O, _ = oa.prompt(Q[:5], K[:2], V[:2], [0, 5], [0, 2])               # five queries, two keys: three rows see none
    assert not O[:3].any() and np.abs(O[3, 0] - oa.bf16_to_f64(V)[0, 0]).max() <= 1e-12
    O, mass = oa.prompt(Q[:4], K[:3], V[:3], [1, 3], [0, 3], causal=False)
    assert not O[[0, 3]].any() and O[1].any() and (mass >= np.abs(O) - 1e-15).all()


def test_refusals():
    L, P = ag.lib(), 1 << 20
    good = dict(Q=P, K=P, V=P, O=P, q_stride=1024, k_stride=256, v_stride=256, o_stride=1024, H_q=8, H_kv=2, D=128, n_seq=1, q_off=P, kv_off=None,
                q_tokens=10, kv_tokens=10, causal=1, scale=0.0)
    call = lambda **k: L.attention_prompt_persistent(C.byref(ag.PromptAttention(**{**good, **k})), P, None)  # noqa: E731  (the plan is not looked at before these)
    for bad in (dict(Q=None), dict(K=None), dict(V=None), dict(O=None), dict(q_off=None), dict(Q=P + 8), dict(K=P + 2), dict(V=P + 8), dict(O=P + 8), dict(q_off=P + 2),
                dict(kv_off=P + 1), dict(D=96), dict(H_q=7), dict(H_q=0), dict(H_kv=0), dict(H_q=130), dict(n_seq=-1), dict(q_tokens=-1), dict(kv_tokens=-1),
                dict(q_tokens=1 << 31), dict(q_stride=1016), dict(q_stride=1028), dict(k_stride=128), dict(v_stride=260), dict(o_stride=512), dict(q_stride=1 << 40),
                dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert call(**bad) == ag.AG_ERR_ARG, bad
    assert L.attention_prompt_persistent(None, P, None) == ag.AG_ERR_ARG
    assert L.attention_prompt_persistent(C.byref(ag.PromptAttention(**good)), None, None) == ag.AG_ERR_ARG
    assert call(n_seq=0) == ag.AG_OK and call(q_tokens=0) == ag.AG_OK


def test_struct_matches_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "asymgemm.h"', 'int main(void) {', '  printf("%zu\\n", sizeof(ag_prompt_attention));']
    lines += [f'  printf("%zu\\n", offsetof(ag_prompt_attention, {f[0]}));' for f in ag.PromptAttention._fields_]
    src = tmp_path / "abi.c"
    src.write_text("\n".join(lines + ['  return 0;', '}']))
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "abi")])
    seen = [int(v) for v in subprocess.check_output([str(tmp_path / "abi")], text=True).split()]
    assert seen == [C.sizeof(ag.PromptAttention)] + [getattr(ag.PromptAttention, f[0]).offset for f in ag.PromptAttention._fields_]
