"""Attention over whole prompts against its 64-bit oracle.

Tolerance: the probabilities (relative to a reference, up to 2^8) are rounded to bf16, at most half a step: 2^-8 relative, so an output is off by
at most 2^-8 * sum p |v| / sum p.  Scores are exact bf16 products summed in 32 bits, off by at most 2^-16 * sum |q k| scale (128 adds), and sum |q k| scale < 60 for
the inputs here: below 2^-10, which moves an output by at most 2 * 2^-10 of the same sum; the exponential's 2^-22 is nothing beside it.
The output is rounded to bf16: 2^-8 |want|.  Together 2^-8 |want| + 1.5 * 2^-8 * sum p |v| / sum p."""
import gc

import numpy as np
import pytest
import torch

from oracle import attention as oa
from paper_2609_24270_b200 import binding as ag
from paper_2609_24270_b200 import inputs
from tests.gpu_util import device_topo

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def give_memory_back():
    """Tests that look at addresses or at free memory find torch's allocator without blocks of these."""
    yield
    gc.collect()
    torch.cuda.empty_cache()

_plans = {}


def plan_for(budget=None, **kw):
    key = (budget, tuple(sorted(kw.items())))
    if key not in _plans:
        topo = device_topo()
        _plans[key] = ag.sched_build(topo, None, budget or topo.n_sm, ag.make_policy(kind=ag.AG_DIE_COMPACT, M=128, N=256, K=64, **kw))
    return _plans[key]


def rows(n, h, d, seed, peak=1.0):
    x = np.random.default_rng(seed).standard_normal((n, h, d)).astype(np.float32) * peak
    return inputs.f32_to_bf16_bits(x)


def offsets(lens, lead=0):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32) + lead


def dev(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy((a.view(np.int16) if a.dtype == np.uint16 else a).copy()).cuda()


def run(Q, K, V, q_off, kv_off=None, causal=True, plan=None, scale=0.0, fill=7.0, stream=0, times=1):
    Tq, Hq, D = Q.shape
    Tk, Hkv, _ = K.shape
    plan = plan or plan_for()
    dQ, dK, dV, dqo = dev(Q), dev(K), dev(V), dev(q_off)
    dko = None if kv_off is None else dev(kv_off)
    O = torch.full((Tq, Hq, D), fill, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    for _ in range(times):
        ag.attention_prompt(dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), O.data_ptr(), Hq, Hkv, D, dqo.data_ptr(), None if dko is None else dko.data_ptr(),
                            len(q_off) - 1, Tq, Tk, plan, causal=causal, scale=scale, stream=stream)
    torch.cuda.synchronize()
    st = plan.last_status()
    assert st == ag.AG_OK, (ag.strerror(st), plan.last_status_where())
    return O.float().cpu().numpy().astype(np.float64)


def check(got, want, mass):
    assert np.isfinite(got).all()
    bound = 2.0 ** -8 * np.abs(want) + 1.5 * 2.0 ** -8 * mass + 1e-30
    assert (np.abs(got - want) <= bound).all(), float((np.abs(got - want) / bound).max())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 63, 64, 65, 127, 128, 129, 300])
def test_one_sequence(D, n):
    Q, K, V = rows(n, 4, D, 1), rows(n, 2, D, 2), rows(n, 2, D, 3)
    for causal in (True, False):
        check(run(Q, K, V, [0, n] and offsets([n]), causal=causal), *oa.prompt(Q, K, V, offsets([n]), causal=causal))


@pytest.mark.parametrize("D,Hq,Hkv", [(128, 3, 1), (64, 5, 1), (128, 2, 2), (128, 14, 2), (64, 32, 1), (128, 64, 1), (128, 7, 7)])
def test_head_groups(D, Hq, Hkv):
    lens = [70, 1, 200, 33]
    Q, K, V = rows(sum(lens), Hq, D, 4), rows(sum(lens), Hkv, D, 5), rows(sum(lens), Hkv, D, 6)
    check(run(Q, K, V, offsets(lens)), *oa.prompt(Q, K, V, offsets(lens)))


@pytest.mark.parametrize("D", [64, 128])
def test_packed_sequences_with_and_without_a_past(D):
    """Empty sequences, sequences without keys, more queries than keys (rows that see nothing), long pasts; tokens of no sequence keep what they held."""
    q_lens = [5, 0, 130, 1, 64, 300, 17, 2]
    k_lens = [5, 9, 700, 513, 0, 300, 9, 128]
    q_off, kv_off = offsets(q_lens, lead=3), offsets(k_lens, lead=11)
    Q, K, V = rows(int(q_off[-1]) + 4, 8, D, 7, 2.0), rows(int(kv_off[-1]) + 2, 2, D, 8), rows(int(kv_off[-1]) + 2, 2, D, 9)
    for causal in (True, False):
        got = run(Q, K, V, q_off, kv_off, causal)
        want, mass = oa.prompt(Q, K, V, q_off, kv_off, causal)
        a, b = int(q_off[0]), int(q_off[-1])
        check(got[a:b], want[a:b], mass[a:b])
        assert (got[:a] == 7.0).all() and (got[b:] == 7.0).all()


@pytest.mark.parametrize("k_lens", [[9, 0, 300], [0, 0, 0], [130, 1, 0]])
def test_far_more_queries_than_keys(k_lens):
    """Whole tiles, and whole units, whose rows see nothing."""
    q_lens = [700, 500, 1000]
    q_off, kv_off = offsets(q_lens), offsets(k_lens)
    Q, K, V = rows(2200, 8, 128, 33), rows(max(1, sum(k_lens)), 2, 128, 34), rows(max(1, sum(k_lens)), 2, 128, 35)
    for causal in (True, False):
        check(run(Q, K, V, q_off, kv_off, causal), *oa.prompt(Q, K, V, q_off, kv_off, causal))
    if not sum(k_lens):
        plan, dQ, off, koff = plan_for(), dev(Q), dev(q_off), dev(kv_off)
        O = torch.full((2200, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        ag.attention_prompt(dQ.data_ptr(), None, None, O.data_ptr(), 8, 2, 128, off.data_ptr(), koff.data_ptr(), 3, 2200, 0, plan)      # no keys at all
        torch.cuda.synchronize()
        assert plan.last_status() == ag.AG_OK and not O.any()


def test_growing_maxima_and_a_scale():
    """Scores that keep rising along the keys make the reference move again and again; so do peaked ones."""
    n, D = 700, 128
    Q, K, V = rows(n, 4, D, 10, 3.0), rows(n, 1, D, 11), rows(n, 1, D, 12)
    Kf = oa.bf16_to_f64(K) * np.linspace(0.01, 3, n)[:, None, None]
    K = inputs.f32_to_bf16_bits(Kf.astype(np.float32))
    Q[:, 2] = Q[0, 2]
    K[:, 0, :4] = inputs.f32_to_bf16_bits((np.sign(oa.bf16_to_f64(Q[0, 2, :4])) * np.linspace(0, 8, n)[:, None]).astype(np.float32))
    for scale in (0.0, 0.3):
        want, mass = oa.prompt(Q, K, V, offsets([n]), scale=scale or None)
        got = run(Q, K, V, offsets([n]), scale=scale)
        # scores reach 300 here: their 32-bit sums are off by up to 128 * 2^-23 * 300 < 2^-7.7, an output by twice that
        bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -6.7) * mass
        assert (np.abs(got - want) <= bound).all()


def test_foreign_values_never_enter():
    """NaN and infinities in other sequences' keys and values, and behind the last one, leave a sequence's result bit for bit as it is."""
    lens = [50, 129, 77]
    q_off = offsets(lens)
    Q, K, V = rows(300, 8, 128, 13), rows(300, 2, 128, 14), rows(300, 2, 128, 15)
    clean = run(Q, K, V, q_off)
    for bad in (0x7FC0, 0x7F80, 0xFF80, 0xFF7F):
        K2, V2, Q2 = K.copy(), V.copy(), Q.copy()
        for x in (K2, V2, Q2):
            x[:50], x[179:] = bad, bad
        got = run(Q2, K2, V2, q_off)
        assert np.array_equal(got[50:179], clean[50:179])
        assert (got[256:] == 7.0).all()
    V2 = V.copy()
    V2[60, 0, 5] = 0x7FC0                     # a NaN of its own shows, in the rows that see it
    got = run(Q, K, V2, q_off)
    assert np.isnan(got[60:179, :4, 5]).all() and np.isfinite(got[50:60]).all() and np.isfinite(got[50:179, 4:]).all()


def test_later_values_however_large_never_enter():
    """The largest finite values in later tokens of the same sequence: a masked probability has to be zero, not nearly zero."""
    n = 200
    Q, K, V = rows(n, 8, 128, 30), rows(n, 2, 128, 31), rows(n, 2, 128, 32)
    clean = run(Q, K, V, offsets([n]))
    V2 = V.copy()
    V2[150:] = 0x7F7F
    V2[150:, 0, ::2] = 0xFF7F
    got = run(Q, K, V2, offsets([n]))
    assert np.array_equal(got[:150], clean[:150])


@pytest.mark.parametrize("D", [64, 128])
def test_a_nan_behind_rows_with_a_long_past(D):
    """Rows that share a key tile with a later token's NaN, at the end of 65536 keys: computed again, in time, and right."""
    n, m, at = 40, 65536, 65536 - 10
    Q, K, V = rows(n, 4, D, 33), rows(m, 1, D, 34), rows(m, 1, D, 35)
    want, mass = oa.prompt(Q, K, V, [0, n], [0, m])
    V2 = V.copy()
    V2[at] = 0x7FC0
    got = run(Q, K, V2, np.array([0, n], np.int32), np.array([0, m], np.int32))
    check(got[: n - 10], want[: n - 10], mass[: n - 10])
    assert np.isnan(got[n - 10:]).all()


def test_parts_of_a_fused_projection():
    n, Hq, Hkv, D = 150, 6, 2, 64
    qkv = rows(n, Hq + 2 * Hkv, D, 16)
    d = dev(qkv)
    O = torch.full((n, Hq + 1, D), 7.0, dtype=torch.bfloat16, device="cuda")
    q_off = dev(offsets([100, 50]))
    plan, stride = plan_for(), (Hq + 2 * Hkv) * D
    ag.attention_prompt(d.data_ptr(), d.data_ptr() + 2 * Hq * D, d.data_ptr() + 2 * (Hq + Hkv) * D, O.data_ptr(), Hq, Hkv, D, q_off.data_ptr(), None, 2, n, n, plan,
                        q_stride=stride, k_stride=stride, v_stride=stride, o_stride=(Hq + 1) * D)
    torch.cuda.synchronize()
    assert plan.last_status() == ag.AG_OK
    got = O.float().cpu().numpy().astype(np.float64)
    check(got[:, :Hq], *oa.prompt(qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], offsets([100, 50])))
    assert (got[:, Hq] == 7.0).all()


def test_on_sm_budgets_and_again_and_again():
    lens = [900, 40, 333, 1, 128]
    Q, K, V = rows(sum(lens), 8, 128, 17), rows(sum(lens), 2, 128, 18), rows(sum(lens), 2, 128, 19)
    want = oa.prompt(Q, K, V, offsets(lens))
    first = None
    for plan in (plan_for(), plan_for(74), plan_for(5), plan_for(1), plan_for(static_assign=0)):
        got = run(Q, K, V, offsets(lens), plan=plan, times=3)
        check(got, *want)
        first = got if first is None else first
        assert np.array_equal(got, first)     # who computes a unit does not matter
    plan = plan_for()
    plan.set_grid(9)                          # fewer blocks than planned SMs (the whole chip: every block lands on one): they drain the queue
    got = run(Q, K, V, offsets(lens), plan=plan)
    plan.set_grid(0)
    assert np.array_equal(got, first)


def test_two_plans_side_by_side():
    topo = device_topo()
    left = ag.sched_build(topo, None, 74, ag.make_policy(kind=ag.AG_DIE_COMPACT, M=128, N=256, K=64))
    right = ag.sched_build(topo, None, 74, ag.make_policy(kind=ag.AG_DIE_COMPACT, M=128, N=256, K=64, avoid=left.parsed()["sm_list"].tolist()))
    lens = [400, 300]
    Q, K, V = rows(700, 8, 128, 20), rows(700, 2, 128, 21), rows(700, 2, 128, 22)
    dQ, dK, dV, off = dev(Q), dev(K), dev(V), dev(offsets(lens))
    outs = [torch.full((700, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for O, s, plan in zip(outs, streams, (left, right)):
            ag.attention_prompt(dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), O.data_ptr(), 8, 2, 128, off.data_ptr(), None, 2, 700, 700, plan, stream=s.cuda_stream)
    torch.cuda.synchronize()
    assert left.last_status() == ag.AG_OK and right.last_status() == ag.AG_OK
    want = oa.prompt(Q, K, V, offsets(lens))
    for O in outs:
        check(O.float().cpu().numpy().astype(np.float64), *want)


def test_more_sequences_than_one_launch_takes():
    rng = np.random.default_rng(23)
    lens = rng.integers(0, 6, 2500)
    lens[1030] = 400
    n = int(lens.sum())
    Q, K, V = rows(n, 2, 64, 24), rows(n, 1, 64, 25), rows(n, 1, 64, 26)
    before = ag.kernel_launch_count()
    got = run(Q, K, V, offsets(lens))
    assert ag.kernel_launch_count() == before + 3
    check(got, *oa.prompt(Q, K, V, offsets(lens)))


def test_offsets_that_lie_outside_are_clamped():
    Q, K, V = rows(100, 4, 64, 27), rows(80, 2, 64, 28), rows(80, 2, 64, 29)
    q_off, kv_off = np.array([-5, 40, 30, 2000], np.int32), np.array([-9, 20, 20, 1 << 30], np.int32)
    got = run(Q, K, V, q_off, kv_off)
    want, mass = oa.prompt(Q, K, V, [0, 40, 40], [0, 20, 20])
    check(got[:30], want[:30], mass[:30])
    want, mass = oa.prompt(Q, K, V, [30, 100], [20, 80])       # (tokens 30 to 39 belong to two sequences: either one's result)
    check(got[40:], want[40:], mass[40:])


def test_refuses_a_capturing_stream():
    s = torch.cuda.Stream()
    Q, off = torch.zeros(4, 2, 64, dtype=torch.int16, device="cuda"), dev(offsets([4]))
    plan = plan_for()
    plan_for().last_status()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with pytest.raises(ag.AgError) as e:
        with torch.cuda.graph(g, stream=s):
            ag.attention_prompt(Q.data_ptr(), Q.data_ptr(), Q.data_ptr(), Q.data_ptr(), 2, 2, 64, off.data_ptr(), None, 1, 4, 4, plan, stream=s.cuda_stream)
    assert e.value.status == ag.AG_ERR_ARG
