"""CPU: what the functions of a drafted step refuse, and their structures as a C compiler sees them."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2609_24270_b200 import binding as ag

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20          # an address that nothing reads: every call below is refused before it would


def test_structs_match_the_header(tmp_path):
    structs = {"ag_rotary": (ag.Rotary, "freq rot layout magnitude"), "ag_rotary_scaling": (ag.RotaryScaling, "rot scaling base factor context low high"),
               "ag_rotary_rows": (ag.RotaryRows, "Q K V Q_out K_out q_stride k_stride v_stride q_out_stride k_out_stride H_q H_kv D n_tokens pos from n_rows"),
               "ag_tree_attention": (ag.TreeAttention, "Q K V O q_stride k_stride v_stride o_stride H_q n_seq row off parent n_tokens max_tokens scale"),
               "ag_draft_verification": (ag.DraftVerification, "P Q p_stride q_stride type vocab distinct n_seq n_tokens off parent token u u_next accepted next new_off from")}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "asymgemm.h"', "int main(void) {"]
    for name, (_, fields) in structs.items():
        lines.append(f'  printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'  printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f in fields.split()]
    src, exe = tmp_path / "abi.c", tmp_path / "abi"
    src.write_text("\n".join(lines + ["  return 0;", "}"]))
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    seen = dict(ln.split() for ln in subprocess.check_output([str(exe)], text=True).splitlines())
    for name, (py, fields) in structs.items():
        assert int(seen[name]) == C.sizeof(py), name
        for f in fields.split():
            assert int(seen[f"{name}.{f}"]) == getattr(py, "from_" if f == "from" else f).offset, (name, f)


def refused(call, good, bad):
    for change in bad:
        assert call(**{**good, **change}) == ag.AG_ERR_ARG, change


def test_rotary_refusals():
    def call(null=(), freq=A, rot=128, layout=0, magnitude=1.0, **kw):
        r = ag.Rotary(freq, rot, layout, magnitude)
        f = dict(Q=A, K=A + 4096, V=None, Q_out=A + 8192, K_out=A + 12288, q_stride=512, k_stride=256, v_stride=0, q_out_stride=512, k_out_stride=256, H_q=4, H_kv=2, D=128,
                 n_tokens=3, pos=A, from_=None, n_rows=0)
        f.update(kw)
        x = ag.RotaryRows(**f)
        return ag.lib().ag_rotary_apply(None if "r" in null else C.byref(r), None if "x" in null else C.byref(x), None)

    refused(call, {}, [dict(null="r"), dict(null="x"), dict(freq=None), dict(freq=A + 4), dict(rot=0), dict(rot=8), dict(rot=24), dict(rot=144), dict(rot=-16), dict(layout=2),
                       dict(magnitude=float("nan")), dict(magnitude=float("inf")), dict(n_tokens=-1), dict(n_tokens=1 << 31), dict(D=96), dict(D=0), dict(Q=A + 8), dict(K=A + 2),
                       dict(Q=None), dict(Q_out=None), dict(K_out=None), dict(Q=None, K=None, Q_out=None, K_out=None), dict(q_stride=504), dict(q_stride=516), dict(k_stride=248),
                       dict(q_out_stride=504), dict(k_out_stride=0), dict(H_q=0), dict(H_q=4097), dict(H_kv=0), dict(pos=None), dict(pos=A + 2), dict(from_=A + 1),
                       dict(from_=A, n_rows=-1), dict(Q_out=A, from_=A, n_rows=3), dict(Q_out=A, q_out_stride=520), dict(K_out=A + 4096, k_out_stride=264), dict(K_out=A + 8192),
                       dict(K_out=A), dict(Q_out=A + 4096)])
    assert call(n_tokens=0) == ag.AG_OK


def test_append_refusals():
    def call(null=(), pages=A, n_pages=4, D=128, slot=A, rot=64, r=True, **kw):
        pool = ag.KV4Pool(pages, n_pages, 2, D)
        f = dict(Q=None, K=A + 4096, V=A + 8192, Q_out=None, K_out=None, q_stride=0, k_stride=256, v_stride=256, q_out_stride=0, k_out_stride=0, H_q=0, H_kv=0, D=0, n_tokens=3,
                 pos=A, from_=None, n_rows=0)
        f.update(kw)
        x, ro = ag.RotaryRows(**f), ag.Rotary(A, rot, 0, 1.0)
        return ag.lib().ag_kv4_append_rotary(None if "pool" in null else C.byref(pool), C.byref(ro) if r else None, None if "x" in null else C.byref(x), slot, None)

    refused(call, {}, [dict(null="pool"), dict(null="x"), dict(pages=None), dict(pages=A + 8), dict(n_pages=0), dict(D=96), dict(D=64, rot=128), dict(slot=None), dict(slot=A + 2),
                       dict(K=None), dict(V=None), dict(V=A + 8), dict(v_stride=128), dict(k_stride=260), dict(pos=None), dict(Q=A, H_q=2, q_stride=256),
                       dict(Q=A, Q_out=A + 16, H_q=0, q_stride=256, q_out_stride=256), dict(K_out=A + 4096, k_out_stride=512), dict(K_out=A + 8192, k_out_stride=256),
                       dict(K_out=A + 4096, k_out_stride=256, from_=A, n_rows=3)])
    assert call(n_tokens=0) == ag.AG_OK


def test_tree_refusals():
    size = ag.attention_tree_kv4_workspace(2, 16, 8, 2, 128, 5)
    assert size > 0

    def call(null=(), H_kv=2, D=128, n_rows=4, max_pages=5, ws=A, ws_bytes=size, **kw):
        pool, table = ag.KV4Pool(A, 4, H_kv, D), ag.KV4Table(A, A, A, n_rows, max_pages)
        f = dict(Q=A, K=A, V=A, O=2 * A, q_stride=1024, k_stride=256, v_stride=256, o_stride=1024, H_q=8, n_seq=2, row=None, off=A, parent=None, n_tokens=20, max_tokens=16, scale=0.0)
        f.update(kw)
        x = ag.TreeAttention(**f)
        return ag.lib().attention_tree_kv4(None if "a" in null else C.byref(x), None if "pool" in null else C.byref(pool), None if "table" in null else C.byref(table), ws, ws_bytes, None)

    refused(call, {}, [dict(null="a"), dict(null="pool"), dict(null="table"), dict(Q=None), dict(K=None), dict(V=None), dict(O=None), dict(off=None), dict(Q=A + 8), dict(O=A + 2),
                       dict(off=A + 2), dict(parent=A + 1), dict(row=A + 3), dict(q_stride=1016), dict(q_stride=1028), dict(k_stride=128), dict(v_stride=252), dict(o_stride=8), dict(H_q=0),
                       dict(H_q=7), dict(H_q=130), dict(n_seq=-1), dict(n_seq=5), dict(n_tokens=-1), dict(n_tokens=1 << 30), dict(max_tokens=0), dict(max_tokens=65),
                       dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(ws=None), dict(ws=A + 8), dict(ws_bytes=size - 1), dict(D=96), dict(max_pages=0)])
    assert call(n_seq=0) == ag.AG_OK and call(n_tokens=0) == ag.AG_OK
    for bad in ((0, 1, 1, 1, 64, 1), (1, 0, 1, 1, 64, 1), (1, 65, 1, 1, 64, 1), (1, 1, 3, 2, 64, 1), (1, 1, 65, 1, 64, 1), (1, 1, 1, 1, 96, 1), (1, 1, 1, 1, 64, 0), (1, 1, 1, 1025, 64, 1)):
        assert ag.attention_tree_kv4_workspace(*bad) == 0, bad
    assert max(ag.attention_tree_kv4_workspace(1000, 64, 64 * h, h, 128, 1 << 20) for h in (1, 8, 64)) <= 40_000_000


def test_verify_refusals():
    def call(null=False, **kw):
        f = dict(P=A, Q=A, p_stride=1000, q_stride=1000, type=ag.AG_F32, vocab=1000, distinct=0, n_seq=2, n_tokens=8, off=A, parent=None, token=A, u=A, u_next=A, accepted=A, next=A,
                 new_off=A, from_=A)
        f.update(kw)
        x = ag.DraftVerification(**f)
        return ag.lib().ag_verify_drafts(None if null else C.byref(x), None)

    refused(call, {}, [dict(null=True), dict(P=None), dict(P=A + 2), dict(Q=A + 1), dict(P=A + 1, type=ag.AG_BF16), dict(type=2), dict(vocab=0), dict(vocab=(1 << 24) + 1),
                       dict(p_stride=999), dict(q_stride=999), dict(n_seq=-1), dict(n_tokens=-1), dict(n_tokens=1 << 30), dict(off=None), dict(token=None), dict(u=None), dict(u_next=None),
                       dict(accepted=None), dict(next=None), dict(new_off=None), dict(from_=None), dict(off=A + 1), dict(token=A + 2), dict(u=A + 3), dict(parent=A + 2)])
    assert call(n_seq=0) == ag.AG_OK


def test_a_device_is_asked_for_only_after_the_arguments():
    """Sound arguments get as far as the device: without one the answer is not AG_ERR_ARG."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("would run")
    r = ag.Rotary(A, 64, 0, 1.0)
    x = ag.RotaryRows(A, None, None, 2 * A, None, 512, 0, 0, 512, 0, 4, 0, 128, 3, A, None, 0)
    assert ag.lib().ag_rotary_apply(C.byref(r), C.byref(x), None) not in (ag.AG_OK, ag.AG_ERR_ARG)


def test_packed_rows_are_the_structure():
    v = [11 << 40, 12, 13, 14, 15, -21, 22, 23, 24, 25 << 33, 31, 32, 33, 34 << 32, 41 << 50, 42, 43]
    assert ag._pack_rotary_rows(*v) == bytes(ag.RotaryRows(*v))


def test_verification_of_no_tokens_is_not_refused():
    """Requests without a token among them all: arrays of no entries have no address."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("would run")
    f = dict(P=None, Q=None, p_stride=1000, q_stride=1000, type=ag.AG_F32, vocab=1000, distinct=0, n_seq=2, n_tokens=0, off=A, parent=None, token=None, u=None, u_next=A, accepted=None,
             next=A, new_off=A, from_=None)
    call = lambda **kw: ag.lib().ag_verify_drafts(C.byref(ag.DraftVerification(**{**f, **kw})), None)  # noqa: E731
    assert call() not in (ag.AG_OK, ag.AG_ERR_ARG) and call(from_=A) != ag.AG_ERR_ARG and call(new_off=None) != ag.AG_ERR_ARG
    assert call(from_=A, new_off=None) == ag.AG_ERR_ARG and call(next=None) == ag.AG_ERR_ARG


def test_the_largest_workspace_is_what_the_header_says():
    sizes = [ag.attention_tree_kv4_workspace(s, t, g * h, h, D, 1 << 20) for s in (1, 1000, 1 << 20) for t in (1, 4, 5, 63, 64) for g in (1, 4, 51, 52, 64) for h in (1, 8, 1024) for D in (64, 128)]
    assert 39_000_000 < max(sizes) <= 39_500_000
