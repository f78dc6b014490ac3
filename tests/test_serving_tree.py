"""Attention of drafted tokens over the 4-bit cache against the 64-bit oracle.

Tolerance: o = sum p v / sum p.  A probability is off by 2 e relative for scores that are off by e, and by 2^-11 (its rounding); e <= (2^-11 sum |q| |k| + 2^-19 sum |q| top) scale, top the largest
|base| + 15 s (or drafted element) of a tile; the maximum over the keys is taken.  Sum p and the sum of p v are both off by as much, so an output is by twice that times sum p |v| / sum p.  A
value is off by 2^-11 of itself and 2^-17 of the largest.  Together (2^-11 * 4 + 4 e) mass + 2^-17 largest, and 2^-8 of the output for its own rounding.  Sums in 32 bits add 2^-20 of the mass."""
import gc

import numpy as np
import pytest
import torch

from oracle import drafts, kv4
from oracle.attention import bf16_to_f64
from paper_2609_24270_b200 import binding as ag
from tests.test_serving_kv4 import dev
from tests.test_serving_kv4_decode import make, sensible_pages

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def give_memory_back():
    """Tests that look at addresses or at free memory find torch's allocator without blocks of these."""
    yield
    gc.collect()
    torch.cuda.empty_cache()


def rows(n, H, D, seed, stretch=1.0):
    return kv4.bf16_bits(kv4.f32_to_bf16_value(stretch * np.random.default_rng(seed).standard_normal((n, H, D)).astype(np.float32)))


def parents(counts, seed=0, chain=False):
    rng = np.random.default_rng(seed)
    return np.array([-1 if i == 0 else i - 1 if chain else int(rng.integers(0, i)) for n in counts for i in range(n)], np.int32)


def run(Q, K, V, c, off, parent, H_q, most, row=None, stream=0, scale=0.0, strides=None, O=None, n_tokens=None, twice=True):
    n, _, D = Q.shape
    S = len(off) - 1
    size = ag.attention_tree_kv4_workspace(S, most, H_q, c.pages.shape[1], D, c.page_of.shape[1])
    ws = torch.full((max(size, 16),), 255, dtype=torch.uint8, device="cuda")          # NaN where nothing is written
    dQ, dK, dV = (x if isinstance(x, torch.Tensor) else dev(x) for x in (Q, K, V))
    d_off, d_row, d_par = dev(np.asarray(off, np.int32)), None if row is None else dev(np.asarray(row, np.int32)), None if parent is None else dev(parent)
    O = torch.full((n, H_q, D), float("nan"), dtype=torch.bfloat16, device="cuda") if O is None else O
    torch.cuda.synchronize()
    for _ in range(2 if twice else 1):
        ag.attention_tree_kv4(dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), O.data_ptr(), c.pool, c.table, None if row is None else d_row.data_ptr(), d_off.data_ptr(),
                              None if parent is None else d_par.data_ptr(), S, n if n_tokens is None else n_tokens, most, H_q, ws.data_ptr(), size, scale=scale, stream=stream,
                              **(strides or {}))
    torch.cuda.synchronize()
    assert int(ws[:4].view(torch.int32)[0]) == ag.AG_OK
    return O.float().cpu().numpy().astype(np.float64)


def check(got, Q, K, V, c, off, parent, G, row=None, scale=None):
    cache = drafts.cache_of(c.pages, c.D, c.page_of, c.len)
    want, mass, reach = drafts.tree(Q, K, V, cache, off, parent, G, row, scale)
    here = slice(int(off[0]), int(off[-1]))
    want, mass, reach, got = want[here], mass[here], reach[here], got[here]
    sc = 1 / np.sqrt(c.D) if scale is None else scale
    top = 0.0
    for x in (K, V):
        f = np.abs(bf16_to_f64(x))
        top = max(top, f[np.isfinite(f)].max(initial=0.0))
    pair = bf16_to_f64(np.ascontiguousarray(c.pages[:, :, 64 * c.D:]).view(np.uint16)).reshape(-1, 2)
    with np.errstate(invalid="ignore"):
        edge = np.abs(pair[:, 1]) + 15 * np.abs(pair[:, 0])
    top = max(top, edge[np.isfinite(edge)].max(initial=0.0))
    e = 2.0 ** -11 * reach + 2.0 ** -19 * np.abs(bf16_to_f64(Q))[here].sum(-1, keepdims=True) * top * sc
    bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -9 + 4 * e + 2.0 ** -20) * mass + 2.0 ** -17 * top + 1e-30
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= bound).all(), float((np.abs(got - want) / bound).max())
    return want


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 3, 4, 8, 16, 64])
def test_heads_tokens_and_ragged_lengths(D, G):
    """Every count of rows that changes the layout of a tile (32, 64, 128, 256 and beside them), every kind of last page."""
    lens, counts = [1, 0, 63, 64, 65, 127, 128, 129, 300, 700], [1, 7, 8, 9, 16, 17, 1, 2, 31, 4]
    if G in (4, 8):
        counts[3], counts[5] = 64, 33
    c = make(lens, 2, D, seed=G)
    n = sum(counts)
    off, par = np.concatenate([[0], np.cumsum(counts)]), parents(counts, G)
    for peak, seed in ((1.0, 1), (5.0, 2)):
        Q, K, V = rows(n, 2 * G, D, seed, peak), rows(n, 2, D, 10 + seed, 1.2), rows(n, 2, D, 20 + seed)
        check(run(Q, K, V, c, off, par, 2 * G, 64), Q, K, V, c, off, par, G)


@pytest.mark.parametrize("D,lens,counts,G", [(128, [5000, 1, 2049], [8, 64, 20], 4), (64, [9000], [33], 8), (128, [20000], [64], 16), (128, [3000, 3000], [1, 5], 7), (64, [12345], [1], 1)])
def test_long_rows_are_split_and_joined(D, lens, counts, G):
    c = make(lens, 1, D, seed=7, max_pages=340)
    n, off, par = sum(counts), np.concatenate([[0], np.cumsum(counts)]), parents(counts, 3)
    Q, K, V = rows(n, G, D, 4, 2.0), rows(n, 1, D, 5), rows(n, 1, D, 6)
    got = run(Q, K, V, c, off, par, G, 64)
    check(got, Q, K, V, c, off, par, G)
    assert (got == run(Q, K, V, c, off, par, G, 64)).all()               # bit for bit


def test_one_token_is_the_decode_step():
    """Against attention_decode_kv4 on a cache that holds the token as well: within the two roundings, the token's own of the store among them - none here, a value that four bits hold."""
    lens, D, G = [77, 200, 64], 128, 4
    c = make(lens, 2, D, seed=3)
    Q = rows(3, 8, D, 1)
    K = V = np.zeros((3, 2, D), np.uint16)                                # zeros in the cache: scale 0, base 0
    got = run(Q, K, V, c, [0, 1, 2, 3], None, 8, 1)
    check(got, Q, K, V, c, [0, 1, 2, 3], None, G)
    grown = make([x + 1 for x in lens], 2, D, seed=3)
    grown.pages[:] = 0
    for r, x in enumerate(lens):
        for j in range(x + 1):
            if j < x:
                a, b = c.page_of[r, j // 64], grown.page_of[r, j // 64]
                for h in range(2):
                    for which in (0, 1):
                        for g in range(D // 32):
                            at = kv4.scale_byte(D, which, j % 64, g)
                            grown.pages[b, h, at:at + 4] = c.pages[a, h, at:at + 4]
                        for d in range(D):
                            byte, high = kv4.byte_of(D, which, j % 64, d)
                            grown.pages[b, h, byte] |= (c.pages[a, h, byte] >> (4 * high) & 15) << (4 * high)
    grown.push()
    from tests.test_serving_kv4_decode import reference
    want, mass = reference(Q, grown)
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -5 * mass).all()


def test_a_chain_is_the_default_and_odd_parents_are_none():
    c = make([100, 0], 1, 64, seed=9)
    Q, K, V = rows(12, 2, 64, 1), rows(12, 1, 64, 2), rows(12, 1, 64, 3)
    off = [0, 7, 12]
    one = run(Q, K, V, c, off, None, 2, 8)
    check(one, Q, K, V, c, off, None, 2)
    assert (one == run(Q, K, V, c, off, parents([7, 5], chain=True), 2, 8)).all()
    odd = np.array([-1, 5, 2, -7, 3, 1 << 30, 0, 0, 1, 1, -2 ** 31, 2], np.int32)       # itself, behind itself, far away
    check(run(Q, K, V, c, off, odd, 2, 8), Q, K, V, c, off, odd, 2)


def test_rows_by_number_pages_outside_and_strides():
    """Requests that share a row, rows outside the table, pages outside the pool, parts of one fused projection, another scale."""
    c = make([300, 130, 64], 2, 128, max_pages=9, seed=11)
    c.page_of[0, 2], c.page_of[1, 0], c.page_of[0, 1] = -1, 10 ** 6, c.page_of[0, 0]
    c.len[2] = 10 ** 6                                                    # clamped to the table's width; no pages there
    c.push()
    row, counts = [0, 2, -1, 0, 3, 1], [3, 9, 4, 1, 2, 5]
    n, off, par = sum(counts), np.concatenate([[0], np.cumsum(counts)]), parents(counts, 5)
    Q, K, V = rows(n, 6, 128, 1), rows(n, 2, 128, 2), rows(n, 2, 128, 3)
    qkv = torch.cat([dev(x).view(torch.bfloat16) for x in (Q, K, V)] + [torch.full((n, 1, 128), float("nan"), dtype=torch.bfloat16, device="cuda")], 1)
    w = qkv.stride(0)
    O = torch.full((n, 7, 128), -3.0, dtype=torch.bfloat16, device="cuda")
    size = ag.attention_tree_kv4_workspace(6, 9, 6, 2, 128, 9)
    ws, d = torch.empty(size, dtype=torch.uint8, device="cuda"), [dev(np.asarray(x, np.int32)) for x in (row, off, par)]
    ag.attention_tree_kv4(qkv.data_ptr(), qkv[:, 6:].data_ptr(), qkv[:, 8:].data_ptr(), O.data_ptr(), c.pool, c.table, d[0].data_ptr(), d[1].data_ptr(), d[2].data_ptr(), 6, n, 9, 6,
                          ws.data_ptr(), size, q_stride=w, k_stride=w, v_stride=w, o_stride=O.stride(0), scale=0.2)
    torch.cuda.synchronize()
    check(O[:, :6].float().cpu().numpy().astype(np.float64), Q, K, V, c, off, par, 3, row, 0.2)
    assert (O[:, 6] == -3.0).all()


def test_tokens_of_nobody_and_beyond_the_most():
    c = make([90, 10, 40], 1, 64, seed=13)
    Q, K, V = rows(20, 2, 64, 1), rows(20, 1, 64, 2), rows(20, 1, 64, 3)
    O = torch.full((20, 2, 64), -3.0, dtype=torch.bfloat16, device="cuda")
    got = run(Q, K, V, c, [2, 9, 9, 300], None, 2, 5, O=O, n_tokens=18)   # the last request has more tokens than there are: clamped
    assert (got[:2] == -3).all() and (got[18:] == -3).all() and not got[7:9].any() and not got[14:18].any()
    for a, b, r in ((2, 7, 0), (9, 14, 2)):
        check(got, Q, K, V, c, [a, b], None, 2, [r])


def test_what_is_not_seen_has_no_influence():
    """NaN and infinities in drafted keys and values: those that do not see them are as without them, those that do are not finite where the formula is not.  Codes and pairs of NaN
    behind a row's last token as well."""
    for D, counts in ((128, [9, 5]), (64, [40, 3])):
        c = make([100, 200], 2, D, seed=17)
        for r, x in enumerate((100, 200)):
            last = c.page_of[r, x // 64]
            for tok in range(x % 64, 64):
                for which in (0, 1):
                    at = kv4.scale_byte(D, which, tok, 0)
                    c.pages[last, :, at:at + D // 8] = 0xFF
        c.push()
        n, off = sum(counts), np.concatenate([[0], np.cumsum(counts)])
        par = parents(counts, 19)
        sees = [drafts.ancestors(par[a:b], b - a) for a, b in zip(off[:-1], off[1:])]
        Q, K, V = rows(n, 8, D, 1), rows(n, 2, D, 2), rows(n, 2, D, 3)
        plain = run(Q, K, V, c, off, par, 8, 64)
        check(plain, Q, K, V, c, off, par, 4)
        K2, V2 = K.copy(), V.copy()
        V2[2, 0, 5], V2[4, 0, 5], V2[4, 0, 9], V2[6, 0, 5], V2[off[1] + 1, 1, 3] = 0x7FC0, 0x7F80, 0xFF80, 0xFF80, 0x7F80
        got = run(Q, K, V2, c, off, par, 8, 64)
        with np.errstate(invalid="ignore"):
            want, _, _ = drafts.tree(Q, K, V2, drafts.cache_of(c.pages, D, c.page_of, c.len), off, par, 4)
        assert (np.isnan(got) == np.isnan(want)).all() and (np.isposinf(got) == np.isposinf(want)).all() and (np.isneginf(got) == np.isneginf(want)).all()
        fine = np.isfinite(want)
        assert (got[fine] == plain[fine]).all() and not fine.all()
        K2[3, 1, 7] = 0x7F80
        got = run(Q, K2, V, c, off, par, 8, 64)
        for i in range(counts[0]):
            if sees[0][i, 3]:
                assert not np.isfinite(got[i, 4:]).any() or np.isnan(got[i, 4:]).any()
            else:
                assert (got[i, 4:] == plain[i, 4:]).all()
        assert (got[:, :4] == plain[:, :4]).all() and (got[off[1]:] == plain[off[1]:]).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("count", [5, 12, 25, 50])
@pytest.mark.parametrize("lens", [[1500], [60] * 90])
def test_values_that_are_not_finite_in_every_layout_of_rows(D, count, lens):
    """Rows four times, twice and once in a tile and in both tiles, of units that several blocks share and of whole ones: outputs of tokens that see a value which is not finite are
    not finite where the formula's are not, every other output has the same bits as without it."""
    c = make(lens, 2, D, seed=61)
    counts = [count] * len(lens)
    n, off, par = sum(counts), np.concatenate([[0], np.cumsum(counts)]), parents(counts, 8)
    Q, K, V = rows(n, 8, D, 1), rows(n, 2, D, 2), rows(n, 2, D, 3)
    plain = run(Q, K, V, c, off, par, 8, 64)
    check(plain, Q, K, V, c, off, par, 4)
    V2 = V.copy()
    for first in off[:-1:3]:
        V2[first + 2, 0, 1], V2[first + 3, 0, D - 1], V2[first + 4, 1, 20], V2[first + 2, 1, 20] = 0x7F80, 0xFF80, 0x7F80, 0xFF80
    got = run(Q, K, V2, c, off, par, 8, 64)
    with np.errstate(invalid="ignore"):
        want, _, _ = drafts.tree(Q, K, V2, drafts.cache_of(c.pages, D, c.page_of, c.len), off, par, 4)
    assert (np.isnan(got) == np.isnan(want)).all() and (np.isposinf(got) == np.isposinf(want)).all() and (np.isneginf(got) == np.isneginf(want)).all()
    fine = np.isfinite(want)
    assert (got[fine] == plain[fine]).all() and not fine.all()


@pytest.mark.parametrize("D,counts,lens", [(64, [9, 30], [100, 0]), (128, [20, 4], [900, 70]), (128, [60], [300]), (64, [12] * 60, [50] * 60)])
def test_drafts_far_larger_than_the_others(D, counts, lens):
    """Keys and values up to the type's lowest value in single drafts (padding, say): tokens that do not see them are as the formula has them, and those that see such a value as well."""
    c = make([max(x, 1) for x in lens], 2, D, seed=67)
    n, off = sum(counts), np.concatenate([[0], np.cumsum(counts)])
    par = parents(counts, 9)
    sees = [drafts.ancestors(par[a:b], b - a) for a, b in zip(off[:-1], off[1:])]
    Q, K, V = rows(n, 8, D, 1), rows(n, 2, D, 2), rows(n, 2, D, 3)
    plain = run(Q, K, V, c, off, par, 8, 64)
    check(plain, Q, K, V, c, off, par, 4)
    for scale, which in ((2.0 ** 7, "V"), (2.0 ** 40, "V"), (2.0 ** 127, "V"), (2.0 ** 20, "K"), (2.0 ** 127, "K"), (2.0 ** 127, "KV")):
        K2, V2, touched = K.copy(), V.copy(), np.zeros(n, bool)
        for s, (a, b) in enumerate(zip(off[:-1], off[1:])):
            for t in (2, int(b - a) - 1):
                for x in which:
                    X = K2 if x == "K" else V2
                    X[a + t] = 0xFF7F if scale == 2.0 ** 127 else kv4.bf16_bits(kv4.f32_to_bf16_value((bf16_to_f64(X[a + t]) * scale).astype(np.float32)))
                touched[a:b] |= [bool(sees[s][i, t]) for i in range(b - a)]
        got = run(Q, K2, V2, c, off, par, 8, 64)
        with np.errstate(over="ignore", invalid="ignore"):
            want, mass, reach = drafts.tree(Q, K2, V2, drafts.cache_of(c.pages, D, c.page_of, c.len), off, par, 4)
        # values below 12 (the cache's largest base + 15 scales beside them), or up to 2^6 times a first token's that are in the products; larger ones by probabilities in 32 bits
        e = 2.0 ** -11 * reach + 2.0 ** -19 * np.abs(bf16_to_f64(Q)).sum(-1, keepdims=True) * 12 / np.sqrt(D)
        bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -9 + 4 * e + 2.0 ** -20) * mass + 2.0 ** -17 * 2.0 ** 6 * 12 + 1e-30
        assert (np.abs(got - want) <= bound)[~touched].all() and touched.any() and not touched.all()
        if which == "V":
            fine = touched & (np.abs(want).max((1, 2)) < 3e38)
            assert (np.abs(got - want) <= bound)[fine].all(), float((np.abs(got - want) / bound)[fine].max())


def test_groups_of_nan_in_the_cache():
    c = make([70, 70], 1, 64, seed=23)
    at = kv4.scale_byte(64, 1, 3, 1)
    c.pages[c.page_of[0, 0], 0, at:at + 4] = np.array([0x7FC0, 0x7FC0], np.uint16).view(np.uint8)
    c.push()
    Q, K, V = rows(6, 2, 64, 1), rows(6, 1, 64, 2), rows(6, 1, 64, 3)
    got = run(Q, K, V, c, [0, 3, 6], None, 2, 3)
    assert np.isnan(got[:3, :, 32:]).all() and np.isfinite(got[:3, :, :32]).all()
    check(got, Q, K, V, c, [3, 6], None, 2, [1])


@pytest.mark.parametrize("e", [-100, -30, -8, 0, 12, 60, 100])
def test_sizes_of_values_from_tiny_to_huge(e):
    """Scales, bases and drafted values times 2^e: outputs follow, relative to what they are."""
    c = make([150, 1000], 1, 128, seed=29)
    sb = c.pages[:, :, 72 * 128:].copy().view(np.uint16)
    c.pages[:, :, 72 * 128:] = kv4.bf16_bits(kv4.f32_to_bf16_value((bf16_to_f64(sb) * 2.0 ** e).astype(np.float32))).view(np.uint8)
    c.push()
    Q, K = rows(12, 4, 128, 1), rows(12, 1, 128, 2)
    V = kv4.bf16_bits(kv4.f32_to_bf16_value((bf16_to_f64(rows(12, 1, 128, 3)) * 2.0 ** e).astype(np.float32)))
    got = run(Q, K, V, c, [0, 5, 12], parents([5, 7], 2), 4, 8)
    want, mass, reach = drafts.tree(Q, K, V, drafts.cache_of(c.pages, 128, c.page_of, c.len), [0, 5, 12], parents([5, 7], 2), 4)
    top = 2.0 ** e * 12
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -9 + 2.0 ** -8 * reach) * mass + 2.0 ** -16 * top).all()


@pytest.mark.parametrize("eq,ek", [(40, -40), (-60, 50), (100, -100), (0, -20), (-100, 100), (15, -12)])
def test_sizes_of_queries_and_keys(eq, ek):
    """Queries times 2^eq against keys times 2^ek, cached and drafted: the scores are of ordinary size."""
    c = make([150, 700], 1, 64, seed=31)
    scale = lambda bits, k: kv4.bf16_bits(kv4.f32_to_bf16_value((bf16_to_f64(bits) * 2.0 ** k).astype(np.float32)))  # noqa: E731
    sb = c.pages[:, :, 64 * 64:72 * 64].copy().view(np.uint16)
    c.pages[:, :, 64 * 64:72 * 64] = scale(sb, ek).view(np.uint8)
    c.push()
    off, par = [0, 5, 12], parents([5, 7], 4)
    Q, K, V = scale(rows(12, 4, 64, 1), eq), scale(rows(12, 1, 64, 2), ek), rows(12, 1, 64, 3)
    got = run(Q, K, V, c, off, par, 4, 8, scale=2.0 ** (-eq - ek) / 8)
    check(got, Q, K, V, c, off, par, 4, scale=2.0 ** (-eq - ek) / 8)


def test_a_query_of_one_dominant_element_and_rows_of_zeros():
    c = make([300], 1, 128, seed=37)
    Q, K, V = rows(6, 2, 128, 1), rows(6, 1, 128, 2), rows(6, 1, 128, 3)
    Q[:, 0, 17], Q[2], K[3] = kv4.bf16_bits(np.float32(1000)), 0, 0
    check(run(Q, K, V, c, [0, 6], None, 2, 6), Q, K, V, c, [0, 6], None, 2)


def test_scores_that_grow_from_tile_to_tile():
    """The reference of the exponentials moves again and again, and values grow by binades: outputs are carried along."""
    c = make([1500], 1, 128, seed=41)
    sb = bf16_to_f64(c.pages[:, :, 64 * 128:].copy().view(np.uint16)).reshape(c.pages.shape[0], 1, 2, -1)
    for k, p in enumerate(c.page_of[0]):
        if p >= 0:
            sb[p, :, 0] *= 1 + 0.4 * k
            sb[p, :, 1] *= 2.0 ** (k // 2)
    c.pages[:, :, 64 * 128:] = kv4.bf16_bits(kv4.f32_to_bf16_value(sb.reshape(c.pages.shape[0], 1, -1).astype(np.float32))).view(np.uint8)
    c.push()
    Q, K, V = rows(9, 4, 128, 1, 1.0), rows(9, 1, 128, 2), rows(9, 1, 128, 3)
    check(run(Q, K, V, c, [0, 9], parents([9], 3), 4, 9), Q, K, V, c, [0, 9], parents([9], 3), 4)


def test_many_requests():
    """700 requests of a few tokens: more than there are threads to add them up; more KV heads than blocks."""
    rng = np.random.default_rng(43)
    lens, counts = [int(x) for x in rng.integers(0, 90, 700)], [int(x) for x in rng.integers(0, 4, 700)]
    c = make(lens, 1, 64, seed=43)
    n, off, par = sum(counts), np.concatenate([[0], np.cumsum(counts)]), parents(counts, 6)
    Q, K, V = rows(n, 2, 64, 1), rows(n, 1, 64, 2), rows(n, 1, 64, 3)
    check(run(Q, K, V, c, off, par, 2, 3), Q, K, V, c, off, par, 2)
    c = make([130], 200, 64, seed=44)
    Q, K, V = rows(5, 200, 64, 1), rows(5, 200, 64, 2), rows(5, 200, 64, 3)
    check(run(Q, K, V, c, [0, 5], None, 200, 5), Q, K, V, c, [0, 5], None, 1)


def test_streams_and_graphs():
    """Two calls at once; a captured call reads lengths, tables, trees and tokens when it runs."""
    c = make([500, 900, 30], 2, 128, max_pages=20, seed=47)
    counts = [5, 8, 20]
    n, off, par = sum(counts), np.concatenate([[0], np.cumsum(counts)]).astype(np.int32), parents(counts, 8)
    Q, K, V = rows(n, 8, 128, 1), rows(n, 2, 128, 2), rows(n, 2, 128, 3)
    want = run(Q, K, V, c, off, par, 8, 20)
    size = ag.attention_tree_kv4_workspace(3, 20, 8, 2, 128, 20)
    d = [dev(x) for x in (Q, K, V, off, par)]
    outs, ws, streams = [torch.empty(n, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in range(3)], [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(3)], \
        [torch.cuda.Stream(), torch.cuda.Stream()]

    def call(i, stream):
        ag.attention_tree_kv4(d[0].data_ptr(), d[1].data_ptr(), d[2].data_ptr(), outs[i].data_ptr(), c.pool, c.table, None, d[3].data_ptr(), d[4].data_ptr(), 3, n, 20, 8,
                              ws[i].data_ptr(), size, stream=stream)
    torch.cuda.synchronize()
    for _ in range(6):
        for i in range(2):
            call(i, streams[i].cuda_stream)
    torch.cuda.synchronize()
    for i in range(2):
        assert (outs[i].float().cpu().numpy() == want).all()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=streams[0]):
        call(2, torch.cuda.current_stream().cuda_stream)
    c.len[:] = [100, 1280, 0]
    c.page_of[1, 15:20] = c.page_of[0, :5]
    c.push()
    par = parents(counts, 9)
    d[4].copy_(torch.from_numpy(par))
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    check(outs[2].float().cpu().numpy().astype(np.float64), Q, K, V, c, off, par, 4)


def test_pages_beyond_two_to_the_32_bytes():
    D, H_kv, n_pages = 128, 8, 60000                                       # 4.9 GB
    pages = torch.zeros(n_pages, H_kv, 80 * D, dtype=torch.uint8, device="cuda")
    few = make([200], H_kv, D, seed=53)
    far = [n_pages - 1, n_pages - 3, 52430, n_pages - 2]
    for k in range(4):
        pages[far[k]] = torch.from_numpy(few.pages[few.page_of[0, k]]).cuda()
    page_of, length, refs = dev(np.array([far], np.int32)), dev(np.array([200], np.int32)), torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    Q, K, V = rows(4, 16, D, 1), rows(4, H_kv, D, 2), rows(4, H_kv, D, 3)
    want = run(Q, K, V, few, [0, 4], None, 16, 4)
    few.pool, few.table = ag.KV4Pool(pages.data_ptr(), n_pages, H_kv, D), ag.KV4Table(page_of.data_ptr(), length.data_ptr(), refs.data_ptr(), 1, 4)
    assert (run(Q, K, V, few, [0, 4], None, 16, 4) == want).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows_of", [8, 40, 64, 100, 128, 200])
@pytest.mark.parametrize("jump", [19.75, 23.5, 30.0, 37.5])
@pytest.mark.parametrize("at,below", [(104, 96), (40, 32)])
def test_a_reference_that_moves_inside_a_tile(D, rows_of, jump, at, below):
    """Scores that grow by 2^10.9 after a tile of zeros and then by `jump` further on in the same tile: what has been made of the earlier keys keeps its weight.  Keys, queries and scores are exact
    here (bf16 bases, one element of q that is not 0), log2 e times scale is off by 2^-23 and 2^x by 2^-22: a probability is off by 2^-11 + 2^-15 of itself and 2^-29 of the largest, a value by 2^-17 of
    the largest."""
    c = make([384], 1, D, seed=71)
    score, value = np.zeros(384), np.zeros(384)
    light = 2.0 ** (10.875 - jump)
    for tile in (128, 256):
        score[tile:tile + 128], score[tile:tile + below], score[tile + at] = -40.0, 10.875, jump
        value[tile:tile + below], value[tile + at] = 1.0, -bf16_to_f64(kv4.bf16_bits(kv4.f32_to_bf16_value(np.array([below * light], np.float32))))[0]
    c.pages[:] = 0
    for t in range(384):
        for which, x in enumerate((score, value)):
            for g in range(D // 32):
                b = kv4.scale_byte(D, which, t % 64, g)
                c.pages[c.page_of[0, t // 64], 0, b + 2:b + 4] = kv4.bf16_bits(kv4.f32_to_bf16_value(x[t:t + 1].astype(np.float32))).view(np.uint8)
    c.push()
    G = 8 if rows_of % 8 == 0 else 4
    count, S, scale = rows_of // G, 160, float(np.float32(np.log(2.0)))
    Q, zero = np.zeros((S * count, G, D), np.uint16), np.zeros((S * count, 1, D), np.uint16)
    Q[..., 0] = kv4.bf16_bits(np.float32(1.0))
    got = run(Q, zero, zero, c, count * np.arange(S + 1), np.full(S * count, -1, np.int32), G, 64, row=[0] * S, scale=scale)
    want, mass, _ = drafts.tree(Q[:1], zero[:1], zero[:1], drafts.cache_of(c.pages, D, c.page_of, c.len), [0, 1], None, G, None, scale)
    bound = 2.0 ** -8 * np.abs(want[0]) + (2.0 ** -11 + 2.0 ** -15) * mass[0] + 2.0 ** -17 + 384 * 2.0 ** -29
    assert (np.abs(got - want[0]) <= bound).all(), float((np.abs(got - want[0]) / bound).max())


def scaled(bits, k):
    """bf16 bits times 2^k; k None: the type's lowest value."""
    if k is None:
        return np.full_like(bits, 0xFF7F)
    return kv4.bf16_bits(kv4.f32_to_bf16_value((bf16_to_f64(bits) * 2.0 ** k).astype(np.float32)))


_held = {}


def cache_once(c, *key):
    """drafts.cache_of of a cache that `key` determines, read once."""
    if key not in _held:
        _held[key] = kv4.load(c.pages, c.D, np.arange(c.pages.shape[0] * kv4.PAGE))
    K, V = _held[key]

    def cache(r, h):
        at = (c.page_of[r].astype(np.int64)[:, None] * kv4.PAGE + np.arange(kv4.PAGE)).reshape(-1)[:c.len[r]]
        return K[at, h], V[at, h]
    return cache


def check_beside_large_drafts(got, Q, K, V, c, cache, off, par, untouched, seen):
    """Rows that see nothing large (`untouched`) and rows that see large values (`seen`) against the formula.  Cached elements are below 12 here, those of ordinary drafts as well; values up to 2^6
    times as large may be in the products, larger ones are added with probabilities in 32 bits."""
    with np.errstate(over="ignore", invalid="ignore"):
        want, mass, reach = drafts.tree(Q, K, V, cache, off, par, Q.shape[1] // K.shape[1])
    e = 2.0 ** -11 * reach + 2.0 ** -19 * np.abs(bf16_to_f64(Q)).sum(-1, keepdims=True) * 12 / np.sqrt(c.D)
    bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -9 + 4 * e + 2.0 ** -20) * mass + 2.0 ** -17 * 2.0 ** 6 * 12 + 1e-30
    assert untouched.any()
    for rows_ in (untouched, seen & (np.abs(want).max((1, 2)) < 3e38)):
        assert (np.abs(got - want) <= bound)[rows_].all(), float((np.abs(got - want) / bound)[rows_].max())


LARGE = [(64, [9, 30], [100, 0]), (128, [20, 4], [900, 70]), (128, [60], [300]), (64, [12] * 20, [50] * 20), (128, [5], [900]), (128, [6, 3], [0, 0])]


@pytest.mark.parametrize("D,counts,lens", LARGE)
@pytest.mark.parametrize("which", ["K", "V", "KV"])
@pytest.mark.parametrize("k", [7, 40, 100, None])
def test_large_drafts_behind_a_first_token_of_zeros(D, counts, lens, which, k):
    """The first token's key or value is 0, or what is finite of it: drafts that a row does not see have no influence all the same."""
    c = make(lens, 2, D, seed=73)
    n, off = sum(counts), np.concatenate([[0], np.cumsum(counts)])
    par = parents(counts, 10)
    for a, b in zip(off[:-1], off[1:]):
        par[b - 1] = 0                                                    # a branch of its own: the others do not see it
    Q, K, V = rows(n, 8, D, 1), rows(n, 2, D, 2), rows(n, 2, D, 3)
    for x in which:
        X = K if x == "K" else V
        for a, b in zip(off[:-1], off[1:]):
            X[a] = 0
            X[b - 1] = scaled(X[b - 1], k)
    last = np.zeros(n, bool)
    last[off[1:] - 1] = True
    check_beside_large_drafts(run(Q, K, V, c, off, par, 8, 64), Q, K, V, c, cache_once(c, D, *lens, 73), off, par, ~last, last & (which == "V"))


@pytest.mark.parametrize("D,counts,lens", LARGE)
@pytest.mark.parametrize("which", ["K", "V", "KV"])
@pytest.mark.parametrize("k", [20, 100, None])
@pytest.mark.parametrize("place", ["first", "second"])
def test_large_drafts_in_a_forest(D, counts, lens, which, k, place):
    """Two trees in a request's drafts (a parent outside is none): the one is as if the other were of ordinary size."""
    c = make(lens, 2, D, seed=79)
    n, off = sum(counts), np.concatenate([[0], np.cumsum(counts)])
    par, large = parents(counts, 11), np.zeros(n, bool)
    for a, b in zip(off[:-1], off[1:]):
        h = a + (b - a) // 2
        par[h] = -1 if h > a else par[h]
        par[h + 1:b] = np.maximum(par[h + 1:b], h - a)
        par[a + 1:h] = np.minimum(par[a + 1:h], h - a - 1)
        large[a:h] = place == "first"
        large[h:b] = place == "second"
    Q, K, V = rows(n, 8, D, 1), rows(n, 2, D, 2), rows(n, 2, D, 3)
    for x in which:
        X = K if x == "K" else V
        X[large] = scaled(X[large], k)
    check_beside_large_drafts(run(Q, K, V, c, off, par, 8, 64), Q, K, V, c, cache_once(c, D, *lens, 79), off, par, ~large, large & (which == "V"))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", [[200], [0], [900]])
def test_large_drafts_beside_padding(D, lens):
    """Padding of zeros, a root each, behind a tree: its rows are averages of the cache, whatever the tree's values are, and the tree's rows are the formula's."""
    c = make(lens, 2, D, seed=83)
    off, par = [0, 40], parents([40], 12)
    par[12:] = -1
    Q, K, V = rows(40, 8, D, 1), rows(40, 2, D, 2), rows(40, 2, D, 3)
    K[12:], V[12:] = 0, 0
    tree = np.arange(40) < 12
    check(run(Q, K, V, c, off, par, 8, 64), Q, K, V, c, off, par, 4)
    for k in (4, 9, 60, None):
        V2 = V.copy()
        V2[:12] = scaled(V[:12], k)
        got = run(Q, K, V2, c, off, par, 8, 64)
        check_beside_large_drafts(got, Q, K, V2, c, cache_once(c, D, *lens, 83), off, par, ~tree, tree if k == 60 else tree & False)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("count", [5, 12, 25, 50])
@pytest.mark.parametrize("lens", [[300], [0], [60] * 6])
def test_rows_that_see_large_drafted_keys(D, count, lens):
    """Keys 2^7 to 2^40 times as large as the others, scores of ordinary size (a small scale): rows that see them weigh them as the formula does.  At 2^20 and the usual scale a large key takes
    everything or nothing.  Rows four times, twice and once in a tile, and in both tiles."""
    c = make(lens, 2, D, seed=89)
    counts = [count] * len(lens)
    n, off, par = sum(counts), np.concatenate([[0], np.cumsum(counts)]), parents(counts, 14)
    Q, K, V = rows(n, 8, D, 1), rows(n, 2, D, 2), rows(n, 2, D, 3)
    cache = cache_once(c, D, *lens, 89)
    sees = [drafts.ancestors(par[a:b], b - a) for a, b in zip(off[:-1], off[1:])]
    for k in (7, 9, 12, 40):
        K2 = K.copy()
        for a, b in zip(off[:-1], off[1:]):
            for t, more in ((1, 0), (3, 1), (int(b - a) - 1, -1)):        # (of several sizes)
                K2[a + t] = scaled(K[a + t], k + more)
        scale = 2.0 ** (-k - 1) / np.sqrt(D)
        got = run(Q, K2, V, c, off, par, 8, 64, scale=scale)
        want, mass, reach = drafts.tree(Q, K2, V, cache, off, par, 4, None, float(np.float32(scale)))
        e = 2.0 ** -11 * reach + 2.0 ** -19 * np.abs(bf16_to_f64(Q)).sum(-1, keepdims=True) * 12 * scale
        bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -9 + 4 * e + 2.0 ** -20) * mass + 2.0 ** -17 * 12 + 1e-30
        assert (np.abs(got - want) <= bound).all(), (k, float((np.abs(got - want) / bound).max()))
    K2, first = K.copy(), off[:-1]
    K2[first + 2] = scaled(K[first + 2], 20)
    got = run(Q, K2, V, c, off, par, 8, 64)
    want, mass, _ = drafts.tree(Q, K2, V, cache, off, par, 4)
    _, _, reach = drafts.tree(Q, K, V, cache, off, par, 4)               # of the keys that decide where the large one is out
    e = 2.0 ** -11 * reach + 2.0 ** -19 * np.abs(bf16_to_f64(Q)).sum(-1, keepdims=True) * 12 / np.sqrt(D)
    bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -9 + 4 * e + 2.0 ** -20) * mass + 2.0 ** -17 * 12 + 1e-30
    taken = 0
    for s, a in enumerate(first):
        for i in range(counts[s]):
            for hq in range(8):
                x = bf16_to_f64(Q[a + i, hq]) @ bf16_to_f64(K2[a + 2, hq // 4]) / np.sqrt(D) if sees[s][i, 2] else -np.inf
                if abs(x) > 2.0 ** 12:                                    # (beyond what 2^-11 of 2^20 |q| |k| can turn)
                    assert (np.abs(got - want) <= bound)[a + i, hq].all(), (s, i, hq, x)
                    taken += bool(x > 0)
    assert taken


def test_a_wait_of_this_kernel_gives_up_and_leaves_the_device_usable():
    """A barrier that nothing signals: the wait ends by the SM's clock, 2^32 cycles at most here (of 1 GHz at least)."""
    st, waited = ag.wait_probe_clock()
    assert st == ag.AG_ERR_TIMEOUT and waited < 4.3e9
    c = make([100], 1, 64, seed=97)
    Q, K, V = rows(5, 2, 64, 1), rows(5, 1, 64, 2), rows(5, 1, 64, 3)
    check(run(Q, K, V, c, [0, 5], None, 2, 5), Q, K, V, c, [0, 5], None, 2)
