"""Attention over prompts whose values and keys are not finite here and there: a row's result follows from what the row sees, whatever later tokens hold.

The oracle: with the values that are not finite taken as zeros, the 64-bit attention; then, column by column, a NaN or infinities of both signs that the row sees
make a NaN, one kind of infinity stays; a key whose score is a NaN or infinite makes the whole row NaN, one of minus infinity has no weight.  Tolerance of the finite results: that of
tests/test_serving_prompt.py (derived there)."""
import gc

import numpy as np
import pytest
import torch

from oracle import attention as oa
from paper_2609_24270_b200 import binding as ag
from tests.test_serving_prompt import dev, offsets, plan_for, rows, run

pytestmark = pytest.mark.gpu
NAN, INF, NEG = 0x7FC0, 0x7F80, 0xFF80


@pytest.fixture(autouse=True, scope="module")
def give_memory_back():
    """Tests that look at addresses or at free memory find torch's allocator without blocks of these."""
    yield
    gc.collect()
    torch.cuda.empty_cache()


def odd(bits):
    return (bits & 0x7F80) == 0x7F80


def want_of(Q, K, V, q_off, kv_off):
    """(result, bound); rows of tokens that belong to a sequence."""
    Qf, Kf, Vf = oa.bf16_to_f64(Q), oa.bf16_to_f64(K), oa.bf16_to_f64(np.where(odd(V), 0, V).astype(np.uint16))
    want, mass = np.full(Qf.shape, 7.0), np.zeros(Qf.shape)
    G = Q.shape[1] // K.shape[1]
    for a, b, c, d in zip(q_off[:-1], q_off[1:], kv_off[:-1], kv_off[1:]):
        last = (d - c) - (b - a) + np.arange(b - a)
        visible = np.arange(d - c)[None] <= last[:, None]
        for hq in range(Q.shape[1]):
            v = V[c:d, hq // G]
            with np.errstate(invalid="ignore", over="ignore"):
                s = np.where(visible, Qf[a:b, hq] @ Kf[c:d, hq // G].T / np.sqrt(Q.shape[2]), -np.inf)
            lost = np.isnan(s).any(1) | (s == np.inf).any(1)                   # a key makes the row NaN, unless its score is minus infinity
            assert not (visible & (s == -np.inf))[:, odd(v).any(1)].any()      # (zero times infinity is not asked for)
            s[lost] = np.where(visible, 0.0, -np.inf)[lost]
            some = visible.any(1)
            p = np.exp(s - s.max(1, keepdims=True, initial=-1e300))
            p /= np.where(some, p.sum(1), 1)[:, None]
            w = p @ Vf[c:d, hq // G]
            mass[a:b, hq] = p @ np.abs(Vf[c:d, hq // G])

            def sees(where):                                                   # [queries][columns]: the row sees a key with `where` in the column
                first = np.where(where.any(0), where.argmax(0), 1 << 30) if d > c else np.full(Q.shape[2], 1 << 30)
                return last[:, None] >= first[None]

            nan, up, down = sees(odd(v) & ((v & 0x7F) != 0)), sees(v == INF), sees(v == NEG)
            w[up], w[down] = np.inf, -np.inf
            w[nan | (up & down) | lost[:, None]] = np.nan
            want[a:b, hq] = w
    return want, 2.0 ** -8 * np.abs(want) + 1.5 * 2.0 ** -8 * mass + 1e-30


def compare(got, want, bound):
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want))
    inf, fine = np.isinf(want), np.isfinite(want)
    assert (got[inf] == want[inf]).all()
    assert (np.abs(got[fine] - want[fine]) <= bound[fine]).all()


def spoil(x, n, seed, kinds=(NAN, INF, NEG)):
    rng, x = np.random.default_rng(seed), x.copy()
    for _ in range(n):
        x[rng.integers(x.shape[0]), rng.integers(x.shape[1]), rng.integers(x.shape[2])] = rng.choice(kinds)
    return x


@pytest.mark.parametrize("D,Hq,Hkv", [(128, 8, 2), (64, 8, 2), (128, 3, 1), (64, 21, 1), (128, 2, 2)])
def test_values_here_and_there(D, Hq, Hkv):
    q_lens, k_lens = [1, 70, 300, 0, 129, 64], [1, 70, 700, 5, 40, 128]
    q_off, kv_off = offsets(q_lens), offsets(k_lens)
    Q, K, V = rows(sum(q_lens), Hq, D, 1), rows(sum(k_lens), Hkv, D, 2), rows(sum(k_lens), Hkv, D, 3)
    for n, kinds in ((1, (NAN,)), (4, (INF,)), (30, (NAN, INF, NEG)), (300, (INF, NEG))):
        V2 = spoil(V, n, n, kinds)
        compare(run(Q, K, V2, q_off, kv_off), *want_of(Q, K, V2, q_off, kv_off))
    K2, V2 = spoil(K, 3, 5), spoil(V, 9, 6)
    compare(run(Q, K2, V2, q_off, kv_off), *want_of(Q, K2, V2, q_off, kv_off))


@pytest.mark.parametrize("D", [64, 128])
def test_rows_in_front_keep_their_bits(D):
    """A later token's values change nothing, not even a rounding."""
    n = 500
    Q, K, V = rows(n, 8, D, 7), rows(n, 2, D, 8), rows(n, 2, D, 9)
    clean = run(Q, K, V, offsets([n]))
    for at in (499, 300, 257, 256, 255, 1):
        V2, K2 = V.copy(), K.copy()
        V2[at:, :, ::3], K2[at:, 0, 5] = INF, NAN
        V2[at:, 1, 1::7] = NAN
        got = run(Q, K2, V2, offsets([n]))
        assert np.array_equal(got[:at], clean[:at])


@pytest.mark.parametrize("which", ["first", "last", "all", "every other"])
@pytest.mark.parametrize("budget", [None, 1, 3])
def test_units_that_are_run_again(budget, which):
    """On few SMs a block runs many units in turn: any of them, and the last one, may have to be run once more."""
    lens = [64] * 7 + [65, 200, 31]                # G = 4: units of 64 tokens
    off = offsets(lens)
    Q, K, V = rows(sum(lens), 4, 64, 10), rows(sum(lens), 1, 64, 11), rows(sum(lens), 1, 64, 12)
    for i, (a, b) in enumerate(zip(off[:-1], off[1:])):
        if which == "all" or (which == "first" and i == 8) or (which == "last" and i == 9) or (which == "every other" and i % 2):
            V[(a + b) // 2, 0, i] = (NAN, INF, NEG)[i % 3]
    plan = plan_for(budget)
    for _ in range(3):
        compare(run(Q, K, V, off, plan=plan, times=2), *want_of(Q, K, V, off, off))


@pytest.mark.parametrize("D", [64, 128])
def test_the_end_of_a_million_keys(D):
    """40 queries behind a million keys share a tile with a later token's NaN; every warp of the block has such rows."""
    n, m, G = 40, 1 << 20, 6
    gen = torch.Generator(device="cuda").manual_seed(D)
    Q, K, V = (torch.randn(t, h, D, device="cuda", generator=gen).bfloat16() for t, h in ((n, G), (m, 1), (m, 1)))
    V2 = V.clone()
    V2[m - 10] = float("nan")
    V2[m - 5:, 0, ::2] = float("inf")
    O = torch.full_like(Q, 7.0)
    off, koff, plan = dev(np.array([0, n], np.int32)), dev(np.array([0, m], np.int32)), plan_for()
    torch.cuda.synchronize()
    ag.attention_prompt(Q.data_ptr(), K.data_ptr(), V2.data_ptr(), O.data_ptr(), G, 1, D, off.data_ptr(), koff.data_ptr(), 1, n, m, plan)
    torch.cuda.synchronize()
    assert plan.last_status() == ag.AG_OK
    seen = torch.arange(m, device="cuda")[None] <= m - n + torch.arange(n, device="cuda")[:, None]
    for h in range(G):
        p = torch.where(seen, Q[:, h].double() @ K[:, 0].double().T / D ** 0.5, -float("inf")).softmax(1)
        want, mass = p @ V[:, 0].double(), p @ V[:, 0].double().abs()
        bound = 2.0 ** -8 * want.abs() + 1.5 * 2.0 ** -8 * mass
        assert ((O[:, h].double() - want).abs() <= bound)[: n - 10].all() and O[n - 10:, h].isnan().all()


def test_a_model_that_has_diverged():
    """Every value a NaN: every row is one, after a bounded multiple of the usual time (a row by row repair took hundreds of times as long)."""
    n, Hq, Hkv, D = 4096, 32, 8, 128
    gen = torch.Generator(device="cuda").manual_seed(3)
    Q, K, V = (torch.randn(n, h, D, device="cuda", generator=gen).bfloat16() for h in (Hq, Hkv, Hkv))
    bad, O, off, plan = torch.full_like(V, float("nan")), torch.zeros_like(Q), dev(offsets([n])), plan_for()
    took = []
    for v in (V, bad):
        best = float("inf")
        for _ in range(4):
            e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            e[0].record()
            ag.attention_prompt(Q.data_ptr(), K.data_ptr(), v.data_ptr(), O.data_ptr(), Hq, Hkv, D, off.data_ptr(), None, 1, n, n, plan,
                                stream=torch.cuda.current_stream().cuda_stream)
            e[1].record()
            torch.cuda.synchronize()
            best = min(best, e[0].elapsed_time(e[1]))
        assert plan.last_status() == ag.AG_OK
        took.append(best)
    assert O.isnan().all()
    print(f"finite {took[0] * 1000:.0f} us, all NaN {took[1] * 1000:.0f} us")
    assert took[1] < 20 * took[0]


def test_units_that_last_longer_than_two_seconds():
    """Twenty-five million keys, every value a NaN: a unit and its second pass take some 2.9 s, most of it the second pass, while the next one waits for its turn."""
    n, m, G, D = 130, 24 << 20, 4, 128
    Q = torch.ones(n, G, D, dtype=torch.bfloat16, device="cuda")
    K, V = torch.zeros(m, 1, D, dtype=torch.bfloat16, device="cuda"), torch.full((m, 1, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    O = torch.zeros_like(Q)
    off, koff, plan = dev(np.array([0, n], np.int32)), dev(np.array([0, m], np.int32)), plan_for(1)
    e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    s = torch.cuda.current_stream()
    e[0].record()
    ag.attention_prompt(Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(), G, 1, D, off.data_ptr(), koff.data_ptr(), 1, n, m, plan, stream=s.cuda_stream)
    e[1].record()
    torch.cuda.synchronize()
    print(f"three units, twice: {e[0].elapsed_time(e[1]) / 1000:.2f} s")
    assert plan.last_status() == ag.AG_OK and O.isnan().all()
