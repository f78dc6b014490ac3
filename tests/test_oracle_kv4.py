"""Pins of the 4-bit cache's oracle, and the refusals of the library's entry points that need no device."""
import ctypes as C

import numpy as np
import pytest

from oracle import kv4
from oracle.attention import bf16_to_f64
from paper_2609_24270_b200 import binding as ag
from paper_2609_24270_b200 import inputs


@pytest.mark.parametrize("D", [64, 128])
def test_every_element_has_its_own_nibble(D):
    for which in (0, 1):
        seen = {kv4.byte_of(D, which, t, d) for t in range(64) for d in range(D)}
        assert len(seen) == 64 * D and {b for b, _ in seen} == set(range(which * 32 * D, (which + 1) * 32 * D))
    at = {kv4.scale_byte(D, w, t, g) for w in (0, 1) for t in range(64) for g in range(D // 32)}
    assert at == set(range(64 * D, 80 * D, 4))
    # worked by hand at D = 128: token 17 = run 1, h 0, g 1; element 41 of K = group 1, t 1, i 1
    if D == 128:
        assert kv4.byte_of(128, 0, 17, 41) == (1024 + (4 + 1) * 16 + 4, 1)
        # token 27 = run 1, h 1, t 1, e 1; element 41 of V = i 2, j 1, g 1
        assert kv4.byte_of(128, 1, 27, 41) == (4096 + 1024 + 512 + (4 + 1) * 16 + 8 + 4 + 1, 0)


def test_quantisation_by_hand():
    x = np.zeros(32, dtype=np.float32)
    x[:16] = np.arange(16)                       # lo 0, hi 15: scale 1, codes are the numbers
    codes, s, b = kv4.quantise(kv4.bf16_bits(x))
    assert s[0] == 1 and b[0] == 0 and (codes[:16] == np.arange(16)).all() and not codes[16:].any()
    x = np.full(32, -2.5, dtype=np.float32)      # one value only: scale 0, the base says it all
    codes, s, b = kv4.quantise(kv4.bf16_bits(x))
    assert s[0] == 0 and b[0] == -2.5 and not codes.any()
    x = np.linspace(-3, 4.5, 32).astype(np.float32)
    x[5] = np.inf
    codes, s, b = kv4.quantise(kv4.bf16_bits(x))
    assert np.isnan(s[0]) and np.isnan(b[0]) and not codes.any()


@pytest.mark.parametrize("D", [64, 128])
def test_store_and_load_are_inverse_up_to_half_a_step(D):
    K = inputs.uniform_bf16(7 * 2, D, 3).reshape(7, 2, D)
    V = inputs.uniform_bf16(7 * 2, D, 4).reshape(7, 2, D)
    pages = np.zeros((3, 2, 80 * D), dtype=np.uint8)
    slot = [5, 64, 130, 63, 191, 0, 77]
    kv4.store(pages, D, K, V, slot)
    for rows, back in zip((K, V), kv4.load(pages, D, slot)):
        x = bf16_to_f64(rows)
        _, s, _ = kv4.quantise(rows)
        # half a step, and what the scale's rounding (2^-9 of it, times 15 codes) leaves out at the top of the range
        assert (np.abs(back - x) <= np.repeat(s, 32, -1).astype(np.float64) * (0.5 + 15 * 2.0 ** -9) * (1 + 1e-6)).all()


def test_tables_keep_their_counts():
    rng = np.random.default_rng(0)
    page_of, length, refs = np.full((6, 8), -1, np.int32), np.zeros(6, np.int32), np.zeros(20, np.int32)
    pages = rng.integers(0, 256, (20, 1, 80 * 64)).astype(np.uint8)
    for step in range(60):
        kind = step % 4
        before = {r: [pages[p].tobytes() for p in page_of[r] if p >= 0] for r in range(6)}
        if kind == 0:
            kv4.extend(page_of, length, refs, rng.permutation(6)[:2], np.array([0, 70, 75]), 75)
        elif kind == 1:
            kv4.fork(pages, page_of, length, refs, rng.integers(0, 6, 2), rng.integers(0, 6, 2))
        elif kind == 2:
            kv4.free(page_of, length, refs, rng.integers(0, 6, 1))
        else:
            kv4.compact(pages, page_of, refs)
            assert before == {r: [pages[p].tobytes() for p in page_of[r] if p >= 0] for r in range(6)}
            assert not (refs[(refs > 0).sum():] > 0).any()
        held = page_of[page_of >= 0]
        assert (np.bincount(held, minlength=20) == refs).all()
        assert all((page_of[r] >= 0).sum() == -(-length[r] // 64) for r in range(6))


def pool_and_table(**kw):
    pool = dict(pages=1 << 20, n_pages=10, H_kv=2, D=128)
    table = dict(page_of=1 << 20, len=1 << 20, refs=1 << 20, n_rows=4, max_pages=8)
    for k, v in kw.items():
        (pool if k in pool else table)[k] = v
    return ag.KV4Pool(*pool.values()), ag.KV4Table(*table.values())


def test_refusals_of_the_cache_functions():
    """Addresses are made up: every call has to be refused before anything touches them (there may be no device at all)."""
    L = ag.lib()
    P = 1 << 20
    pool, table = pool_and_table()
    bad_pools = [pool_and_table(**k)[0] for k in (dict(pages=None), dict(pages=P + 8), dict(n_pages=0), dict(n_pages=1 << 25), dict(H_kv=0), dict(H_kv=1025), dict(D=96))]
    bad_tables = [pool_and_table(**k)[1] for k in (dict(page_of=None), dict(len=None), dict(refs=None), dict(n_rows=0), dict(max_pages=0), dict(refs=P + 2))]
    r = C.byref
    for p in bad_pools + [None]:
        p = r(p) if p is not None else None
        assert L.ag_kv4_store(p, P, P, 1, 256, 256, P, None) == ag.AG_ERR_ARG
        assert L.ag_kv4_load(p, P, 1, P, P, 256, 256, None) == ag.AG_ERR_ARG
        assert L.ag_kv4_extend(p, r(table), P, P, 1, P, 1, P, None) == ag.AG_ERR_ARG
        assert L.ag_kv4_fork(p, r(table), P, P, 1, P, None) == ag.AG_ERR_ARG
        assert L.ag_kv4_free(p, r(table), P, 1, None) == ag.AG_ERR_ARG
        assert L.ag_kv4_compact(p, r(table), P, None) == ag.AG_ERR_ARG
        assert L.ag_kv4_copy(p, P, P, 1, None) == ag.AG_ERR_ARG
    for t in bad_tables + [None]:
        t = r(t) if t is not None else None
        assert L.ag_kv4_extend(r(pool), t, P, P, 1, P, 1, P, None) == ag.AG_ERR_ARG
        assert L.ag_kv4_fork(r(pool), t, P, P, 1, P, None) == ag.AG_ERR_ARG
        assert L.ag_kv4_free(r(pool), t, P, 1, None) == ag.AG_ERR_ARG
        assert L.ag_kv4_compact(r(pool), t, P, None) == ag.AG_ERR_ARG
    for args in [(None, P, 1, 256, 256, P), (P, None, 1, 256, 256, P), (P, P, 1, 256, 256, None), (P + 2, P, 1, 256, 256, P), (P, P + 8, 1, 256, 256, P),
                 (P, P, -1, 256, 256, P), (P, P, 1, 248, 256, P), (P, P, 1, 256, 128, P), (P, P, 1, 260, 256, P), (P, P, 1 << 31, 256, 256, P),
                 (P, P, 1, 256, 256, P + 1)]:
        assert L.ag_kv4_store(r(pool), *args, None) == ag.AG_ERR_ARG, args
        k, v, n, ks, vs, s = args
        assert L.ag_kv4_load(r(pool), s, n, k, v, ks, vs, None) == ag.AG_ERR_ARG, args
    assert L.ag_kv4_extend(r(pool), r(table), P, P, ag.AG_KV4_MAX_ROWS + 1, P, 1, P, None) == ag.AG_ERR_ARG
    assert L.ag_kv4_extend(r(pool), r(table), P, P, -1, P, 1, P, None) == ag.AG_ERR_ARG
    assert L.ag_kv4_extend(r(pool), r(table), P, P, 1, None, 1, P, None) == ag.AG_ERR_ARG
    assert L.ag_kv4_extend(r(pool), r(table), P, P, 1, P, 1, None, None) == ag.AG_ERR_ARG
    assert L.ag_kv4_fork(r(pool), r(table), P, P, ag.AG_KV4_MAX_ROWS + 1, P, None) == ag.AG_ERR_ARG
    assert L.ag_kv4_fork(r(pool), r(table), P, None, 1, P, None) == ag.AG_ERR_ARG
    assert L.ag_kv4_free(r(pool), r(table), None, 1, None) == ag.AG_ERR_ARG
    assert L.ag_kv4_compact(r(pool), r(table), None, None) == ag.AG_ERR_ARG
    for odd in range(4):
        a = [P + 2 if i == odd else P for i in range(4)]
        assert L.ag_kv4_extend(r(pool), r(table), a[0], a[1], 1, a[2], 1, a[3], None) == ag.AG_ERR_ARG
        if odd < 3:
            assert L.ag_kv4_fork(r(pool), r(table), a[0], a[1], 1, a[2], None) == ag.AG_ERR_ARG
        if odd < 1:
            assert L.ag_kv4_free(r(pool), r(table), a[0], 1, None) == ag.AG_ERR_ARG
            assert L.ag_kv4_compact(r(pool), r(table), a[0], None) == ag.AG_ERR_ARG
    for args in [(P, None, 1), (P + 2, P, 1), (None, P + 1, 1), (P, P, -1), (P, P, 11)]:
        assert L.ag_kv4_copy(r(pool), *args, None) == ag.AG_ERR_ARG, args
    assert L.ag_kv4_copy(r(pool), None, P, 0, None) == ag.AG_OK
    # nothing to do is not an error
    assert L.ag_kv4_store(r(pool), P, P, 0, 256, 256, P, None) == ag.AG_OK
    assert L.ag_kv4_free(r(pool), r(table), P, 0, None) == ag.AG_OK
    assert ag.kv4_page_bytes(8, 128) == 8 * 80 * 128 and ag.kv4_page_bytes(8, 96) == 0 and ag.kv4_page_bytes(0, 64) == 0


def test_cache_structs_match_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    py = {"ag_kv4_pool": ag.KV4Pool, "ag_kv4_table": ag.KV4Table}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "asymgemm.h"', 'int main(void) {']
    for name, cls in py.items():
        lines.append(f'  printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'  printf("{name}.{f[0]} %zu\\n", offsetof({name}, {f[0]}));' for f in cls._fields_]
    src = tmp_path / "abi.c"
    src.write_text("\n".join(lines + ['  return 0;', '}']))
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "abi")])
    seen = dict(line.split() for line in subprocess.check_output([str(tmp_path / "abi")], text=True).splitlines())
    for name, cls in py.items():
        assert int(seen[name]) == C.sizeof(cls)
        for f in cls._fields_:
            assert int(seen[f"{name}.{f[0]}"]) == getattr(cls, f[0]).offset


def test_refusals_of_the_decode_attention():
    L = ag.lib()
    P = 1 << 20
    pool, table = pool_and_table()
    r = C.byref
    good = dict(Q=P, pool=r(pool), table=r(table), row=None, O=P, B=2, H_q=8, ws=P, wsb=1 << 30, stream=None)
    for change in (dict(Q=None), dict(O=None), dict(Q=P + 8), dict(O=P + 4), dict(B=-1), dict(B=5), dict(H_q=7), dict(H_q=1), dict(H_q=0), dict(row=P + 2),
                   dict(pool=None), dict(table=None), dict(H_q=2 * 1025)):
        assert L.attention_decode_kv4(*{**good, **change}.values()) == ag.AG_ERR_ARG, change
    need = ag.attention_decode_kv4_workspace(2, 8, 2, 128, 8)
    assert need > 0
    for change in (dict(ws=None), dict(wsb=need - 1), dict(ws=P + 8)):
        assert L.attention_decode_kv4(*{**good, **change}.values()) == ag.AG_ERR_ARG, change
    assert L.attention_decode_kv4(*{**good, "B": 0}.values()) == ag.AG_OK
    long_table = pool_and_table(max_pages=(1 << 25) - 1)[1]                # a run of pages is counted in 31 bits
    for change in (dict(table=r(long_table), B=1 << 15, row=P), dict(table=r(long_table), B=1 << 30, row=P)):
        assert L.attention_decode_kv4(*{**good, **change}.values()) == ag.AG_ERR_ARG, change
    # parts of 8 heads, two a warp and two a block, 2 * 148 blocks at most; shapes that are refused have size 0
    assert ag.attention_decode_kv4_workspace(1000, 32, 8, 128, 1000) == 18 * 2 * 148 * 8 * (128 * 4 + 8) + 2 * 148 * 8
    assert ag.attention_decode_kv4_workspace(2, 7, 2, 128, 1000) == 0 and ag.attention_decode_kv4_workspace(2, 8, 2, 96, 1000) == 0
