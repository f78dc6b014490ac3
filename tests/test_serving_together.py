"""The serving operators together, as a server uses them: prompts are attended and stored, a prompt's beginning is shared by forks, tokens are decoded and
stored one by one, a later chunk attends over its cached past, requests leave, the pages are put together.  Every attention is compared with its
64-bit oracle on the values that the cache holds."""
import gc

import numpy as np
import pytest
import torch

from oracle import attention as oa
from oracle import kv4
from paper_2609_24270_b200 import binding as ag
from tests.test_serving_kv4 import dev
from tests.test_serving_kv4_decode import check as check_decode
from tests.test_serving_prompt import check as check_prompt
from tests.test_serving_prompt import plan_for, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def give_memory_back():
    """Tests that look at addresses or at free memory find torch's allocator without blocks of these."""
    yield
    gc.collect()
    torch.cuda.empty_cache()



class Server:
    def __init__(self, H_q, H_kv, D, n_pages, n_rows, max_pages):
        self.H_q, self.H_kv, self.D = H_q, H_kv, D
        self.pages = torch.full((n_pages, H_kv, 80 * D), 255, dtype=torch.uint8, device="cuda")       # NaN wherever nothing has been stored
        self.page_of = torch.full((n_rows, max_pages), -1, dtype=torch.int32, device="cuda")
        self.len, self.refs = torch.zeros(n_rows, dtype=torch.int32, device="cuda"), torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        self.pool = ag.KV4Pool(self.pages.data_ptr(), n_pages, H_kv, D)
        self.table = ag.KV4Table(self.page_of.data_ptr(), self.len.data_ptr(), self.refs.data_ptr(), n_rows, max_pages)
        self.held = {}                              # row -> list of (K, V) values of its tokens, as the cache stands for them
        self.stream = torch.cuda.Stream()
        torch.cuda.synchronize()

    def at(self):
        return self.stream.cuda_stream

    def append(self, req, K, V, lens):
        n = len(K)
        row, off = dev(np.array(req, np.int32)), dev(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32))
        slot, ok = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(len(req), dtype=torch.int32, device="cuda")
        dK, dV = dev(K), dev(V)
        torch.cuda.synchronize()
        ag.kv4_extend(self.pool, self.table, row.data_ptr(), off.data_ptr(), len(req), slot.data_ptr(), n, ok.data_ptr(), self.at())
        ag.kv4_store(self.pool, dK.data_ptr(), dV.data_ptr(), slot.data_ptr(), n, stream=self.at())
        torch.cuda.synchronize()
        assert ok.all()
        k, v = (kv4.values(*kv4.quantise(x)) for x in (K, V))
        o = np.concatenate([[0], np.cumsum(lens)])
        for r, a, b in zip(req, o[:-1], o[1:]):
            self.held.setdefault(r, []).extend(zip(k[a:b], v[a:b]))
        return slot

    def decode(self, req, Q):
        size = ag.attention_decode_kv4_workspace(len(req), self.H_q, self.H_kv, self.D, self.page_of.shape[1])
        ws, row, dQ = torch.empty(size, dtype=torch.uint8, device="cuda"), dev(np.array(req, np.int32)), dev(Q)
        O = torch.empty(Q.shape, dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        ag.attention_decode_kv4(dQ.data_ptr(), self.pool, self.table, row.data_ptr(), O.data_ptr(), len(req), self.H_q, ws.data_ptr(), size, self.at())
        torch.cuda.synchronize()
        Qf, G = oa.bf16_to_f64(Q), self.H_q // self.H_kv
        want, mass = np.zeros(Qf.shape), np.zeros(Qf.shape)
        for i, r in enumerate(req):
            k, v = (np.stack([t[w] for t in self.held[r]]) for w in (0, 1))
            for h in range(self.H_kv):
                s = Qf[i, h * G:(h + 1) * G] @ k[:, h].T / np.sqrt(self.D)
                p = np.exp(s - s.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                want[i, h * G:(h + 1) * G], mass[i, h * G:(h + 1) * G] = p @ v[:, h], p @ np.abs(v[:, h])
        check_decode(O.float().cpu().numpy().astype(np.float64), want, mass)

    def fork(self, src, dst):
        s, d = dev(np.array(src, np.int32)), dev(np.array(dst, np.int32))
        ok = torch.empty(len(src), dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        ag.kv4_fork(self.pool, self.table, s.data_ptr(), d.data_ptr(), len(src), ok.data_ptr(), self.at())
        torch.cuda.synchronize()
        assert ok.all()
        for a, b in zip(src, dst):
            self.held[b] = list(self.held[a])

    def free(self, req):
        r = dev(np.array(req, np.int32))
        torch.cuda.synchronize()
        ag.kv4_free(self.pool, self.table, r.data_ptr(), len(req), self.at())
        torch.cuda.synchronize()
        for a in req:
            del self.held[a]

    def compact(self):
        moved = torch.empty(self.refs.numel(), dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        ag.kv4_compact(self.pool, self.table, moved.data_ptr(), self.at())
        torch.cuda.synchronize()
        used = int((self.refs > 0).sum())
        assert not (self.refs[used:] > 0).any() and int(self.page_of.max()) < used


@pytest.mark.parametrize("D", [64, 128])
def test_a_server_from_prompt_to_compaction(D):
    H_q, H_kv = 8, 2
    sv = Server(H_q, H_kv, D, 60, 8, 12)
    plan = plan_for(100)
    # two prompts, attended together and stored
    lens = [150, 333]
    n = sum(lens)
    Q, K, V = rows(n, H_q, D, 40, 1.5), rows(n, H_kv, D, 41), rows(n, H_kv, D, 42)
    off = np.array([0, 150, n], np.int32)
    dQ, dK, dV, d_off = dev(Q), dev(K), dev(V), dev(off)
    O = torch.empty(n, H_q, D, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    ag.attention_prompt(dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), O.data_ptr(), H_q, H_kv, D, d_off.data_ptr(), None, 2, n, n, plan, stream=sv.at())
    torch.cuda.synchronize()
    assert plan.last_status() == ag.AG_OK
    check_prompt(O.float().cpu().numpy().astype(np.float64), *oa.prompt(Q, K, V, off))
    sv.append([0, 1], K, V, lens)
    # four samples of the second prompt; every request decodes a few tokens, apart from one another
    sv.fork([1, 1, 1, 0], [2, 3, 4, 5])
    live = [0, 1, 2, 3, 4, 5]
    for step in range(5):
        k, v = rows(len(live), H_kv, D, 50 + step), rows(len(live), H_kv, D, 60 + step)
        sv.append(live, k, v, [1] * len(live))
        sv.decode(live, rows(len(live), H_q, D, 70 + step, 2.0))
        if step == 1:
            sv.free([1, 3])                       # the shared pages stay with the others
            live = [0, 2, 4, 5]
        if step == 2:
            sv.compact()
        if step == 3:
            sv.fork([4], [1])                     # a row that has been given up is used again
            live = [5, 1, 2, 4, 0]
    # a later chunk of a prompt: its past is read back from the cache, its own keys are taken as they are
    past = len(sv.held[2])
    k, v, q = rows(70, H_kv, D, 80), rows(70, H_kv, D, 81), rows(70, H_q, D, 82)
    slots = torch.tensor([int(sv.page_of[2, j // 64]) * 64 + j % 64 for j in range(past)], dtype=torch.int32, device="cuda")
    kv = torch.empty(2, past + 70, H_kv, D, dtype=torch.bfloat16, device="cuda")
    kv[0, past:], kv[1, past:] = dev(k).view(torch.bfloat16), dev(v).view(torch.bfloat16)
    dq, q_off, kv_off = dev(q), dev(np.array([0, 70], np.int32)), dev(np.array([0, past + 70], np.int32))
    O = torch.empty(70, H_q, D, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    ag.kv4_load(sv.pool, slots.data_ptr(), past, kv[0].data_ptr(), kv[1].data_ptr(), stream=sv.at())
    ag.attention_prompt(dq.data_ptr(), kv[0].data_ptr(), kv[1].data_ptr(), O.data_ptr(), H_q, H_kv, D, q_off.data_ptr(), kv_off.data_ptr(), 1, 70, past + 70, plan,
                        stream=sv.at())
    torch.cuda.synchronize()
    held = [kv4.bf16_bits(kv4.f32_to_bf16_value(np.stack([t[w] for t in sv.held[2]]).astype(np.float32))) for w in (0, 1)]
    check_prompt(O.float().cpu().numpy().astype(np.float64), *oa.prompt(q, np.concatenate([held[0], k]), np.concatenate([held[1], v]), [0, 70], [0, past + 70]))
    sv.append([2], k, v, [70])
    sv.decode([2, 0], rows(2, H_q, D, 90))
    # everybody leaves: no page is held any more
    sv.free(sorted(sv.held))
    assert not sv.refs.any() and not sv.len.any() and (sv.page_of == -1).all()


def test_prompts_and_decoding_share_the_chip():
    """Prompts on one part of the chip, decoding beside them on another stream; both results are those of calls alone."""
    H_q, H_kv, D = 8, 2, 128
    sv = Server(H_q, H_kv, D, 80, 16, 10)
    lens = [300] * 8
    K, V = rows(2400, H_kv, D, 43), rows(2400, H_kv, D, 44)
    sv.append(list(range(8)), K, V, lens)
    plan = plan_for(74)
    n = 1500
    Q, Kp, Vp = rows(n, H_q, D, 45), rows(n, H_kv, D, 46), rows(n, H_kv, D, 47)
    dQ, dK, dV, off = dev(Q), dev(Kp), dev(Vp), dev(np.array([0, 1000, n], np.int32))
    q = dev(rows(8, H_q, D, 48))
    size = ag.attention_decode_kv4_workspace(8, H_q, H_kv, D, 10)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    alone = [torch.empty(n, H_q, D, dtype=torch.bfloat16, device="cuda"), torch.empty(8, H_q, D, dtype=torch.bfloat16, device="cuda")]
    beside = [torch.zeros_like(x) for x in alone]
    other = torch.cuda.Stream()

    def prompt(out, s):
        ag.attention_prompt(dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), out.data_ptr(), H_q, H_kv, D, off.data_ptr(), None, 2, n, n, plan, stream=s.cuda_stream)

    def step(out, s):
        ag.attention_decode_kv4(q.data_ptr(), sv.pool, sv.table, None, out.data_ptr(), 8, H_q, ws.data_ptr(), size, s.cuda_stream)

    torch.cuda.synchronize()
    prompt(alone[0], other)
    torch.cuda.synchronize()
    step(alone[1], other)
    torch.cuda.synchronize()
    for _ in range(10):
        prompt(beside[0], other)
        step(beside[1], sv.stream)
    torch.cuda.synchronize()
    assert plan.last_status() == ag.AG_OK
    assert torch.equal(alone[0], beside[0]) and torch.equal(alone[1], beside[1])
