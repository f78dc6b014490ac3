"""A server's drafted steps from end to end: prompts are turned and stored in one call, trees are drafted, turned, attended over the cache and verified, what stands is committed to
the cache by the numbers that the verification left on the device, step after step and as one captured graph."""
import gc

import numpy as np
import pytest
import torch

from oracle import drafts, kv4
from oracle.attention import bf16_to_f64
from paper_2609_24270_b200 import binding as ag
from tests.test_serving_kv4 import Cache, dev
from tests.test_serving_rotary import rotary
from tests.test_serving_tree import check as check_tree
from tests.test_serving_tree import parents, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def give_memory_back():
    """Tests that look at addresses or at free memory find torch's allocator without blocks of these."""
    yield
    gc.collect()
    torch.cuda.empty_cache()


def softmax(x):
    e = np.exp(x - x.max(-1, keepdims=True))
    return (e / e.sum(-1, keepdims=True)).astype(np.float32)


@pytest.mark.parametrize("D,captured", [(64, False), (128, False), (128, True)])
def test_drafted_steps(D, captured):
    H_q, H_kv, V, most, counts = 8, 2, 500, 8, [8, 3, 5]
    S, n = len(counts), sum(counts)
    c = Cache(60, H_kv, D, 4, 12, seed=1)
    c.push()
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    freq, mag = drafts.frequencies(D // 2, 10000.0, drafts.BANDS, 4.0, 1000.0, 1.0, 4.0)
    r = rotary(D // 2, False, freq, mag)
    stream = torch.cuda.Stream()
    at = lambda t: t.data_ptr()  # noqa: E731

    # prompts: room, then keys turned and stored, queries turned, in one call
    lens = [100, 0, 333]
    m = sum(lens)
    qkv = torch.cat([dev(rows(m, h, D, 5 + i)).view(torch.bfloat16) for i, h in enumerate((H_q, H_kv, H_kv))], 1)
    pos = dev(np.concatenate([np.arange(x) for x in lens]).astype(np.int32))
    row, p_off = dev(np.array([2, 0, 3], np.int32)), dev(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32))
    slot, ok, qT = torch.empty(m, dtype=torch.int32, device="cuda"), torch.empty(S, dtype=torch.int32, device="cuda"), torch.empty(m, H_q, D, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    w = qkv.stride(0)
    ag.kv4_extend(c.pool, c.table, at(row), at(p_off), S, at(slot), m, at(ok), stream.cuda_stream)
    ag.kv4_append_rotary(c.pool, r, at(pos), at(slot), m, at(qkv[:, H_q:]), at(qkv[:, H_q + H_kv:]), q_ptr=at(qkv), q_out_ptr=at(qT), H_q=H_q, k_stride=w, v_stride=w, q_stride=w,
                         stream=stream.cuda_stream)
    torch.cuda.synchronize()
    assert ok.all()

    # one step's buffers; everything below is queued without the host's looking at anything
    buf = dict(qkv=torch.empty(n, H_q + 2 * H_kv, D, dtype=torch.bfloat16, device="cuda"), pos=torch.empty(n, dtype=torch.int32, device="cuda"),
               O=torch.empty(n, H_q, D, dtype=torch.bfloat16, device="cuda"), P=torch.empty(n, V, device="cuda"), Q=torch.empty(n, V, device="cuda"), token=torch.empty(n, dtype=torch.int32, device="cuda"),
               parent=torch.empty(n, dtype=torch.int32, device="cuda"), u=torch.empty(n, device="cuda"), u_next=torch.empty(S, device="cuda"), accepted=torch.empty(n, dtype=torch.int32, device="cuda"),
               next=torch.empty(S, dtype=torch.int32, device="cuda"), new_off=torch.empty(S + 1, dtype=torch.int32, device="cuda"), rows=torch.empty(n, dtype=torch.int32, device="cuda"),
               slot=torch.empty(n, dtype=torch.int32, device="cuda"))
    d_off, size = dev(off), ag.attention_tree_kv4_workspace(S, most, H_q, H_kv, D, 12)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def step(s):
        b = buf
        w = b["qkv"].stride(0)
        Q, K, V_ = b["qkv"], b["qkv"][:, H_q:], b["qkv"][:, H_q + H_kv:]
        ag.rotary_apply(r, at(b["pos"]), n, D, at(Q), at(Q), H_q, at(K), at(K), H_kv, q_stride=w, k_stride=w, q_out_stride=w, k_out_stride=w, stream=s)
        ag.attention_tree_kv4(at(Q), at(K), at(V_), at(b["O"]), c.pool, c.table, at(row), at(d_off), at(b["parent"]), S, n, most, H_q, at(ws), size, q_stride=w, k_stride=w, v_stride=w, stream=s)
        ag.verify_drafts(at(b["P"]), at(b["Q"]), V, at(b["token"]), at(b["parent"]), at(d_off), S, n, at(b["u"]), at(b["u_next"]), at(b["accepted"]), at(b["next"]), at(b["new_off"]),
                         at(b["rows"]), stream=s)
        ag.kv4_extend(c.pool, c.table, at(row), at(b["new_off"]), S, at(b["slot"]), n, at(ok), s)
        ag.kv4_append_rotary(c.pool, None, None, at(b["slot"]), n, at(K), at(V_), k_stride=w, v_stride=w, from_ptr=at(b["rows"]), n_rows=n, stream=s)

    graph = None
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step(torch.cuda.current_stream().cuda_stream)
    held, rng = {2: 100, 0: 0, 3: 333}, np.random.default_rng(D)
    for k in range(4):
        par = parents(counts, k)
        depth = np.zeros(n, int)
        for a, b in zip(off[:-1], off[1:]):
            for i in range(a + 1, b):
                depth[i] = depth[a + par[i]] + 1
        pos = np.concatenate([held[x] + depth[a:b] for x, a, b in zip((2, 0, 3), off[:-1], off[1:])]).astype(np.int32)
        raw = [rows(n, h, D, 50 * k + i, 1.2) for i, h in enumerate((H_q, H_kv, H_kv))]
        P, Qd = softmax(2 * rng.standard_normal((n, V))), softmax(2 * rng.standard_normal((n, V)))
        Qd = (0.7 * P + 0.3 * Qd).astype(np.float32)
        token = np.array([rng.choice(V, p=Qd[a + max(par[i], 0)].astype(np.float64) / Qd[a + max(par[i], 0)].astype(np.float64).sum())
                          for a, b in zip(off[:-1], off[1:]) for i in range(a, b)], np.int32)
        u, u_next = rng.random(n).astype(np.float32) * np.float32(.999), rng.random(S).astype(np.float32) * np.float32(.999)
        for name, x in dict(pos=pos, parent=par, token=token, u=u, u_next=u_next, P=P, Q=Qd).items():
            buf[name].copy_(torch.from_numpy(x))
        buf["qkv"].copy_(torch.cat([dev(x).view(torch.bfloat16) for x in raw], 1))
        c.pages, c.page_of, c.len, c.refs = (c.d[x].cpu().numpy() for x in ("pages", "page_of", "len", "refs"))
        before = {x: getattr(c, x).copy() for x in ("pages", "page_of", "len", "refs")}
        torch.cuda.synchronize()
        if captured:
            graph.replay()
        else:
            step(stream.cuda_stream)
        torch.cuda.synchronize()
        turned = buf["qkv"].view(torch.int16).cpu().numpy().view(np.uint16)
        tQ, tK, tV = turned[:, :H_q], turned[:, H_q:H_q + H_kv], turned[:, H_q + H_kv:]
        want = drafts.rotate(bf16_to_f64(raw[0]), pos, freq, mag)
        assert np.abs(bf16_to_f64(tQ) - want).max() <= 2.0 ** -8 * np.abs(want).max() and (tV == raw[2]).all()
        check_tree(buf["O"].float().cpu().numpy().astype(np.float64), tQ, tK, tV, c, off, par, H_q // H_kv, [2, 0, 3])
        acc, nxt, new_off, took = drafts.verify(P.astype(np.float64), Qd.astype(np.float64), token, par, off, u, u_next)
        for name, x in dict(accepted=acc, next=nxt, new_off=new_off, rows=took).items():
            assert (buf[name].cpu().numpy() == x).all(), name
        slots, fine = kv4.extend(before["page_of"], before["len"], before["refs"], [2, 0, 3], new_off, n)
        assert fine.all() and (buf["slot"].cpu().numpy() == slots).all()
        stands = took[took >= 0]
        kv4.store(before["pages"], D, tK[stands], tV[stands], slots[:len(stands)])
        for x in before:
            assert (c.d[x].cpu().numpy() == before[x]).all(), x
        for j, x in enumerate((2, 0, 3)):
            held[x] += int(new_off[j + 1] - new_off[j])
    assert sum(held.values()) > 433 + 4 * S                                # some drafts stood
