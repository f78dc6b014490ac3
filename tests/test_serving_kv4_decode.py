"""Single-token attention over the 4-bit cache against its 64-bit oracle.

Tolerance: an output is sum_j p_j v_j / sum_j p_j.  v_j is rounded to bf16 once, by at most half a step: 2^-8 relative; p_j is kept to 16 bits.
Scores are 32-bit sums that carry up to 1024 q s on the way: |error| <= 2^-23 * 1024 * sum |q| s / sqrt D =: e, and for the inputs here (sum |q| s < 200 at
D = 128, half at 64) e < 1.2 * 2^-9; an output moves by at most 2 e sum p |v| / sum p.  Together less than 5 * 2^-9 of sum p |v| / sum p (from the
oracle, with |v|); the output's own rounding adds 2^-8 |want|."""
import gc

import numpy as np
import pytest
import torch

from oracle import kv4
from oracle.attention import bf16_to_f64
from paper_2609_24270_b200 import binding as ag
from tests.test_serving_kv4 import Cache, dev

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def give_memory_back():
    """Tests that look at addresses or at free memory find torch's allocator without blocks of these."""
    yield
    gc.collect()
    torch.cuda.empty_cache()



def reference(Q, c, row=None):
    """(want, sum p |v| / sum p), vectorised: the oracle's definition on pages that are decoded once."""
    D, H_kv = c.D, c.pages.shape[1]
    n_pages = c.pages.shape[0]
    K, V = kv4.load(c.pages, D, np.arange(n_pages * 64)) if not hasattr(c, "kv") else c.kv
    c.kv = (K, V)
    Qf = bf16_to_f64(Q)
    B, H_q, _ = Qf.shape
    want, mass = np.zeros(Qf.shape), np.zeros(Qf.shape)
    for b in range(B):
        r = b if row is None else int(row[b])
        if r < 0 or r >= len(c.len):
            continue
        n = min(max(int(c.len[r]), 0), c.page_of.shape[1] * 64)
        pages = np.repeat(c.page_of[r], 64)[:n].astype(np.int64)
        slots = pages * 64 + np.arange(n) % 64
        slots = slots[(pages >= 0) & (pages < n_pages)]
        if not len(slots):
            continue
        G = H_q // H_kv
        for h in range(H_kv):
            s = Qf[b, h * G:(h + 1) * G] @ K[slots, h].T / np.sqrt(D)
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            want[b, h * G:(h + 1) * G] = p @ V[slots, h]
            mass[b, h * G:(h + 1) * G] = p @ np.abs(V[slots, h])
    return want, mass


def sensible_pages(c, seed):
    rng = np.random.default_rng(seed)
    n, H, D = c.pages.shape[0], c.pages.shape[1], c.D
    s = 0.25 * np.exp(0.3 * rng.standard_normal((n, H, 4 * D)))
    b = s * (-7.5 + rng.standard_normal(s.shape))
    pair = np.stack([s, b], -1).astype(np.float32)
    c.pages[:, :, 64 * D:] = kv4.bf16_bits(kv4.f32_to_bf16_value(pair)).reshape(n, H, -1).view(np.uint8)


def make(lens, H_kv, D, max_pages=None, seed=1, spare=2):
    need = [-(-x // 64) for x in lens]
    c = Cache(sum(need) + spare, H_kv, D, len(lens), max_pages or max(need + [1]), seed)
    sensible_pages(c, seed)
    order, at = np.random.default_rng(seed).permutation(sum(need) + spare), 0
    for r, x in enumerate(lens):
        c.page_of[r, :need[r]] = order[at:at + need[r]]
        at += need[r]
        c.len[r] = x
    c.push()
    return c


def queries(B, H_q, D, seed, peak=1.0):
    return kv4.bf16_bits(kv4.f32_to_bf16_value(peak * np.random.default_rng(seed).standard_normal((B, H_q, D)).astype(np.float32)))


def run(Q, c, row=None, stream=0, fill=float("nan")):
    B, H_q, D = Q.shape
    size = ag.attention_decode_kv4_workspace(B, H_q, c.pages.shape[1], D, c.page_of.shape[1])
    ws = torch.full((max(size, 16),), 255, dtype=torch.uint8, device="cuda")       # NaN where nothing is written
    dQ, d_row = dev(Q), None if row is None else dev(np.asarray(row, np.int32))
    O = torch.full((B, H_q, D), fill, dtype=torch.bfloat16, device="cuda")
    for _ in range(2):
        ag.attention_decode_kv4(dQ.data_ptr(), c.pool, c.table, None if row is None else d_row.data_ptr(), O.data_ptr(), B, H_q, ws.data_ptr(), size, stream)
    torch.cuda.synchronize()
    return O.float().cpu().numpy().astype(np.float64)


def check(got, want, mass):
    assert np.isfinite(got).all()
    bound = 2.0 ** -8 * np.abs(want) + 5 * 2.0 ** -9 * mass + 1e-30
    assert (np.abs(got - want) <= bound).all(), float((np.abs(got - want) / bound).max())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 4, 8, 9, 16, 21])
def test_heads_and_ragged_lengths(D, G):
    lens = [1, 0, 63, 64, 65, 15, 16, 17, 130, 700]
    c = make(lens, 2, D, seed=G)
    for peak in (1.0, 6.0):
        Q = queries(len(lens), 2 * G, D, 3, peak)
        got = run(Q, c)
        check(got, *reference(Q, c))
        assert not got[1].any()


@pytest.mark.parametrize("D,lens", [(128, [5000, 1, 2049]), (64, [9000]), (128, [512, 513, 0])])
def test_long_rows_are_split_and_joined(D, lens):
    c = make(lens, 1, D, seed=7, max_pages=150)
    Q = queries(len(lens), 4, D, 4, 3.0)
    assert ag.attention_decode_kv4_workspace(len(lens), 4, 1, D, 150) > 0
    check(run(Q, c), *reference(Q, c))
    # a row that selects itself twice, another order, rows outside the table
    row = [2, 0, -1, 3, 2] if len(lens) == 3 else [0, 0, 1]
    Q = queries(len(row), 4, D, 5)
    got = run(Q, c, row)
    check(got, *reference(Q, c, row))
    assert not got[row.index(-1) if -1 in row else 2].any()


def test_what_lies_behind_the_end_does_not_count():
    """Pages end inside a tile; the rest of the last page, free pages and table entries behind the end hold NaN or nonsense."""
    lens = [1, 20, 64 * 9 + 7, 100]
    c = make(lens, 2, 128, max_pages=20, seed=3)
    nan = np.array([0x7FC0, 0xFF80], np.uint16).view(np.uint8)
    for r, n in enumerate(lens):
        if n % 64:
            block = c.pages[c.page_of[r, n // 64]]
            for which in (0, 1):
                at = kv4.scale_byte(128, which, n % 64, 0)
                end = 72 * 128 + which * 8 * 128
                block[:, at:end] = np.tile(nan, (end - at) // 4)
    c.page_of[:, -1] = 1 << 29
    c.page_of[0, 1:] = -5
    c.push()
    Q = queries(4, 8, 128, 6)
    check(run(Q, c), *reference(Q, c))
    # pages that the pool does not have are left out, and lengths are clamped
    c.page_of[2, 3] = c.pages.shape[0]
    c.page_of[2, 5] = -1
    c.page_of[3, :2] = -1
    c.len[1] = -4
    c.push()
    got = run(Q, c)
    check(got, *reference(Q, c))
    assert not got[1].any() and not got[3].any()
    c.len[0] = 1 << 30
    c.page_of[0, :] = c.page_of[2, 0]
    c.push()
    check(run(Q, c), *reference(Q, c))


def test_values_that_are_not_finite_show():
    c = make([70, 70], 1, 64, seed=8)
    at = kv4.scale_byte(64, 0, 3, 0)
    c.pages[c.page_of[1, 0], :, at:at + 4] = np.array([0x7FC0, 0x7FC0], np.uint16).view(np.uint8)     # one key that was stored as NaN
    c.push()
    got = run(queries(2, 2, 64, 9), c, fill=0.0)
    assert np.isfinite(got[0]).all() and np.isnan(got[1]).all()
    c.pages[c.page_of[1], :, 64 * 64:72 * 64] = np.tile(np.array([0x7FC0, 0x7FC0], np.uint16).view(np.uint8), 128)[None, None]   # every key
    c.push()
    assert np.isnan(run(queries(2, 2, 64, 9), c, fill=0.0)[1]).all()


@pytest.mark.parametrize("step", [1.0, 4.0, 12.0])
@pytest.mark.parametrize("D", [64, 128])
def test_values_of_very_different_sizes(D, step):
    """Pages whose values grow (and shrink) by powers of two from one to the next: the common exponent has to follow.  Beside the usual bound a value
    may be off by 2^-32 of the row's largest: fp16 has steps of 2^-24 at its lower end, so s, taken 16 + u <= 31 times, b - 16 s and the sum are off by at most 33 half steps,
    33 * 2^-25 < 2^-19, where the largest value is kept at 2^13 or more."""
    c = make([700, 64 * 9 + 1], 1, D, seed=17)
    sb = c.pages[:, :, 72 * D:].reshape(c.pages.shape[0], 1, -1).copy().view(np.uint16)
    for r in range(2):
        for i, p in enumerate(c.page_of[r]):
            if p >= 0:
                f = 2.0 ** round((i if r == 0 else -i) * step)
                sb[p] = kv4.bf16_bits((bf16_to_f64(sb[p]) * f).astype(np.float32))
    c.pages[:, :, 72 * D:] = sb.view(np.uint8)
    c.push()
    Q = queries(2, 8, D, 18)
    got, (want, mass) = run(Q, c), reference(Q, c)
    V = c.kv[1]
    for r in range(2):
        n = int(c.len[r])
        slots = np.repeat(c.page_of[r].astype(np.int64), 64)[:n] * 64 + np.arange(n) % 64
        bound = 2.0 ** -8 * np.abs(want[r]) + 5 * 2.0 ** -9 * mass[r] + 2.0 ** -32 * np.abs(V[slots]).max()
        assert np.isfinite(got[r]).all() and (np.abs(got[r] - want[r]) <= bound).all()


def test_calls_side_by_side_and_in_a_graph():
    c = make([300, 4000, 64], 2, 128, seed=11, max_pages=80)
    Qs = [queries(3, 8, 128, 20 + i, 2.0) for i in range(3)]
    size = ag.attention_decode_kv4_workspace(3, 8, 2, 128, 80)
    bufs = [(dev(Q), torch.full((3, 8, 128), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.empty(size, dtype=torch.uint8, device="cuda"),
             torch.cuda.Stream()) for Q in Qs]
    torch.cuda.synchronize()
    for _ in range(20):
        for dQ, O, ws, s in bufs:
            ag.attention_decode_kv4(dQ.data_ptr(), c.pool, c.table, None, O.data_ptr(), 3, 8, ws.data_ptr(), size, s.cuda_stream)
    torch.cuda.synchronize()
    for Q, (_, O, _, _) in zip(Qs, bufs):
        check(O.float().cpu().numpy().astype(np.float64), *reference(Q, c))
    first = bufs[0][1].clone()
    dQ, O, ws, s = bufs[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        ag.attention_decode_kv4(dQ.data_ptr(), c.pool, c.table, None, O.data_ptr(), 3, 8, ws.data_ptr(), size, torch.cuda.current_stream().cuda_stream)
    O.fill_(float("nan"))
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(O, first)             # the same split every time: the same bits
    c.len[:] = [10, 3000, 0]                 # lengths are read when the graph runs
    c.push()
    graph.replay()
    torch.cuda.synchronize()
    check(O.float().cpu().numpy().astype(np.float64), *reference(Qs[0], c))


def test_against_the_oracles_loops():
    c = make([40, 100], 2, 64, seed=13)
    Q = queries(2, 6, 64, 14, 2.0)
    want = kv4.decode(Q, c.pages, 64, c.page_of, c.len)
    assert np.abs(want - reference(Q, c)[0]).max() <= 1e-12
    check(run(Q, c), want, reference(Q, c)[1])
