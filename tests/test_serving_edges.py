"""The serving operators at their far ends: caches and packed tokens beyond four gigabytes, more requests and KV heads than threads or blocks, and
every call of the cache captured into a graph.  Tolerances: those of the modules whose checks are used."""
import gc

import numpy as np
import pytest
import torch

from oracle import attention as oa
from oracle import kv4
from oracle.attention import bf16_to_f64
from paper_2609_24270_b200 import binding as ag
from tests.test_serving_kv4 import dev, special_rows
from tests.test_serving_kv4_decode import check as check_decode
from tests.test_serving_kv4_decode import make, queries, reference
from tests.test_serving_kv4_decode import run as run_decode
from tests.test_serving_prompt import check as check_prompt
from tests.test_serving_prompt import plan_for, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def give_memory_back():
    """Tests that look at addresses or at free memory find torch's allocator without blocks of these."""
    yield
    gc.collect()
    torch.cuda.empty_cache()


def test_pages_beyond_four_gigabytes():
    n_pages, H, D, n_rows, max_pages = 110000, 8, 64, 4, 16
    size = ag.kv4_page_bytes(H, D)
    assert (n_pages - 40) * size > 1 << 32
    pages = torch.empty(n_pages * size, dtype=torch.uint8, device="cuda")
    refs = np.ones(n_pages, np.int32)
    refs[-40:] = 0
    d_refs, d_len = dev(refs), torch.zeros(n_rows, dtype=torch.int32, device="cuda")
    page_of = torch.full((n_rows, max_pages), -1, dtype=torch.int32, device="cuda")
    pool, table = ag.KV4Pool(pages.data_ptr(), n_pages, H, D), ag.KV4Table(page_of.data_ptr(), d_len.data_ptr(), d_refs.data_ptr(), n_rows, max_pages)
    lens = [700, 100]
    T = sum(lens)
    row, off = dev(np.array([0, 1], np.int32)), dev(np.array([0, 700, 800], np.int32))
    slot, ok = torch.empty(T, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(3)
    K, V = (kv4.bf16_bits(kv4.f32_to_bf16_value(rng.standard_normal((T, H, D)).astype(np.float32))) for _ in range(2))
    dK, dV = dev(K), dev(V)
    back_k, back_v = torch.zeros_like(dK), torch.zeros_like(dV)
    ag.kv4_extend(pool, table, row.data_ptr(), off.data_ptr(), 2, slot.data_ptr(), T, ok.data_ptr())
    ag.kv4_store(pool, dK.data_ptr(), dV.data_ptr(), slot.data_ptr(), T)
    ag.kv4_load(pool, slot.data_ptr(), T, back_k.data_ptr(), back_v.data_ptr())
    src, dst = dev(np.array([0], np.int32)), dev(np.array([2], np.int32))
    ag.kv4_fork(pool, table, src.data_ptr(), dst.data_ptr(), 1, ok.data_ptr() + 4)
    torch.cuda.synchronize()
    assert ok.tolist() == [1, 1]
    assert page_of[0, 0].item() == n_pages - 40 and (slot.cpu().numpy() >= (n_pages - 40) * 64).all()
    values = [kv4.values(*kv4.quantise(x)) for x in (K, V)]
    for got, want in zip((back_k, back_v), values):
        want = kv4.bf16_bits(kv4.f32_to_bf16_value(want.astype(np.float32)))       # (s u + b has at most 24 bits for these rows: one rounding)
        assert (got.cpu().numpy().view(np.uint16) == want).all()
    # decode: rows 0, 1 and the fork
    Q = queries(3, 16, D, 5)
    dQ, O = dev(Q), torch.zeros(3, 16, D, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(ag.attention_decode_kv4_workspace(3, 16, H, D, max_pages), dtype=torch.uint8, device="cuda")
    ag.attention_decode_kv4(dQ.data_ptr(), pool, table, None, O.data_ptr(), 3, 16, ws.data_ptr(), ws.numel())
    torch.cuda.synchronize()
    before = O.float().cpu().numpy().astype(np.float64)
    Qf = bf16_to_f64(Q)
    want, mass = np.zeros(Qf.shape), np.zeros(Qf.shape)
    for b, (lo, hi) in enumerate(((0, 700), (700, 800), (0, 700))):
        for h in range(16):
            s = values[0][lo:hi, h // 2] @ Qf[b, h] / np.sqrt(D)
            p = np.exp(s - s.max())
            p /= p.sum()
            want[b, h], mass[b, h] = p @ values[1][lo:hi, h // 2], p @ np.abs(values[1][lo:hi, h // 2])
    check_decode(before, want, mass)
    # the pages set aside in front are given back, and all move to the front: the same bits come out
    d_refs[: n_pages - 40] = 0
    moved = torch.empty(n_pages, dtype=torch.int32, device="cuda")
    ag.kv4_compact(pool, table, moved.data_ptr())
    O.zero_()
    ag.attention_decode_kv4(dQ.data_ptr(), pool, table, None, O.data_ptr(), 3, 16, ws.data_ptr(), ws.numel())
    torch.cuda.synchronize()
    assert page_of.max().item() < 40
    assert (O.float().cpu().numpy() == before).all()


def test_packed_tokens_beyond_four_gigabytes():
    T, stride, Hq, Hkv, D = 41000, 65536, 4, 2, 64
    lo, hi = 40850, 40990
    assert lo * stride * 2 > 1 << 32
    Q, K, V = rows(hi - lo, Hq, D, 1), rows(hi - lo, Hkv, D, 2), rows(hi - lo, Hkv, D, 3)
    X = torch.empty(T, stride, dtype=torch.int16, device="cuda")
    O = torch.empty(T, stride, dtype=torch.bfloat16, device="cuda")
    X[lo - 200:] = 0x7FC0                    # NaN all around
    O[lo - 1:] = 7.0
    for part, at in ((Q, 0), (K, Hq * D), (V, (Hq + Hkv) * D)):
        X[lo:hi, at:at + part.shape[1] * D] = dev(part).view(hi - lo, -1)
    off = dev(np.array([lo, hi], np.int32))
    plan = plan_for()
    torch.cuda.synchronize()
    p = X.data_ptr()
    ag.attention_prompt(p, p + Hq * D * 2, p + (Hq + Hkv) * D * 2, O.data_ptr(), Hq, Hkv, D, off.data_ptr(), None, 1, T, T, plan, q_stride=stride, k_stride=stride,
                        v_stride=stride, o_stride=stride)
    torch.cuda.synchronize()
    assert plan.last_status() == ag.AG_OK
    want, mass = oa.prompt(Q, K, V, [0, hi - lo])
    check_prompt(O[lo:hi, :Hq * D].float().cpu().numpy().astype(np.float64).reshape(hi - lo, Hq, D), want, mass)
    assert (O[lo:hi, Hq * D:] == 7.0).all() and (O[lo - 1] == 7.0).all() and (O[hi:] == 7.0).all()


@pytest.mark.parametrize("offset,pad", [(0, 0), (8, 0), (0, 8), (8, 24), (16, 16)])
@pytest.mark.parametrize("D", [64, 128])
def test_outputs_on_sixteen_byte_boundaries(D, offset, pad):
    """Rows of O that begin on 16 but not on 32 bytes: what lies between them stays."""
    n, Hq, Hkv = 150, 6, 2
    Q, K, V = rows(n, Hq, D, 1), rows(n, Hkv, D, 2), rows(n, Hkv, D, 3)
    dQ, dK, dV, off = dev(Q), dev(K), dev(V), dev(np.array([0, 33, n], np.int32))
    width = Hq * D + pad
    buf = torch.full((offset + n * width + 8,), 7.0, dtype=torch.bfloat16, device="cuda")
    plan = plan_for()
    torch.cuda.synchronize()
    ag.attention_prompt(dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), buf.data_ptr() + 2 * offset, Hq, Hkv, D, off.data_ptr(), None, 2, n, n, plan, o_stride=width)
    torch.cuda.synchronize()
    assert plan.last_status() == ag.AG_OK
    O = buf[offset:offset + n * width].view(n, width)
    want, mass = oa.prompt(Q, K, V, [0, 33, n])
    check_prompt(O[:, :Hq * D].float().cpu().numpy().astype(np.float64).reshape(n, Hq, D), want, mass)
    assert (buf[:offset] == 7.0).all() and (O[:, Hq * D:] == 7.0).all() and (buf[offset + n * width:] == 7.0).all()


def test_more_requests_than_threads():
    """600 requests (the blocks count several requests a thread), every fifth without keys, and rows in another order with strangers among them."""
    rng = np.random.default_rng(6)
    lens = [0 if i % 5 == 0 else int(x) for i, x in enumerate(rng.integers(1, 150, 600))]
    c = make(lens, 1, 64, seed=9)
    Q = queries(600, 2, 64, 10)
    check_decode(run_decode(Q, c), *reference(Q, c))
    row = list(rng.integers(-3, 605, 700))
    Q = queries(700, 2, 64, 11)
    check_decode(run_decode(Q, c, row), *reference(Q, c, row))


@pytest.mark.parametrize("H,G", [(300, 1), (1024, 1), (37, 9)])
def test_many_heads(H, G):
    c = make([130, 5, 0], H, 64, seed=12)
    Q = queries(3, H * G, 64, 13)
    check_decode(run_decode(Q, c), *reference(Q, c))


def test_every_call_in_a_graph():
    """Fork, store, load, copy, free, compact and decode as one graph, replayed twice from the same state, against the same calls made one by one."""
    H, D, n_pages, n_rows, max_pages = 2, 128, 40, 6, 8
    c = make([200, 70, 3], H, D, seed=14, max_pages=max_pages, spare=30)
    state = {k: torch.cat([c.d[k], torch.full((n_rows - 3, *c.d[k].shape[1:]), -1 if k == "page_of" else 0, dtype=c.d[k].dtype, device="cuda")]) if k in ("page_of", "len")
             else c.d[k].clone() for k in c.d}
    state["refs"] = torch.zeros_like(state["refs"])
    used = state["page_of"][state["page_of"] >= 0].long()
    state["refs"][used] = 1
    n_pages = state["refs"].numel()
    live = {k: v.clone() for k, v in state.items()}
    pool = ag.KV4Pool(live["pages"].data_ptr(), n_pages, H, D)
    table = ag.KV4Table(live["page_of"].data_ptr(), live["len"].data_ptr(), live["refs"].data_ptr(), n_rows, max_pages)
    src, dst, gone = dev(np.array([0, 1], np.int32)), dev(np.array([4, 3], np.int32)), dev(np.array([0], np.int32))
    row, off = dev(np.array([4, 3, 2], np.int32)), dev(np.array([0, 1, 2, 70], np.int32))
    K, V = dev(special_rows(70, H, D, 15) & 0x3FFF), dev(special_rows(70, H, D, 16) & 0x3FFF)
    other = torch.empty_like(live["pages"])
    out = {k: torch.zeros(n, dtype=torch.int32, device="cuda") for k, n in (("ok", 2), ("ok2", 3), ("slot", 70), ("moved", n_pages))}
    back = torch.zeros(2, 70, H, D, dtype=torch.int16, device="cuda")
    Q, O = dev(queries(4, 8, D, 17)), torch.zeros(4, 8, D, dtype=torch.int16, device="cuda")
    order = dev(np.array([3, 4, 2, 0], np.int32))
    ws = torch.empty(ag.attention_decode_kv4_workspace(4, 8, H, D, max_pages), dtype=torch.uint8, device="cuda")

    def start():
        for k in live:
            live[k].copy_(state[k])
        other.copy_(state["pages"])
        for t in (*out.values(), back, O):
            t.zero_()

    def calls(s):
        ag.kv4_fork(pool, table, src.data_ptr(), dst.data_ptr(), 2, out["ok"].data_ptr(), s)
        ag.kv4_extend(pool, table, row.data_ptr(), off.data_ptr(), 3, out["slot"].data_ptr(), 70, out["ok2"].data_ptr(), s)
        ag.kv4_store(pool, K.data_ptr(), V.data_ptr(), out["slot"].data_ptr(), 70, stream=s)
        ag.kv4_load(pool, out["slot"].data_ptr(), 70, back[0].data_ptr(), back[1].data_ptr(), stream=s)
        ag.kv4_free(pool, table, gone.data_ptr(), 1, s)
        ag.kv4_compact(pool, table, out["moved"].data_ptr(), s)
        ag.kv4_copy(ag.KV4Pool(other.data_ptr(), n_pages, H, D), None, out["moved"].data_ptr(), n_pages, s)
        ag.attention_decode_kv4(Q.data_ptr(), pool, table, order.data_ptr(), O.data_ptr(), 4, 8, ws.data_ptr(), ws.numel(), s)

    def result():
        torch.cuda.synchronize()
        return [t.cpu().clone() for t in (*live.values(), other, *out.values(), back, O)]

    start()
    torch.cuda.synchronize()
    calls(0)
    want = result()
    assert out["ok"].tolist() == [1, 1] and out["ok2"].tolist() == [1, 1, 1] and O.any()
    start()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        calls(torch.cuda.current_stream().cuda_stream)
    for _ in range(2):
        start()
        graph.replay()
        for a, b in zip(result(), want):
            assert torch.equal(a, b)
