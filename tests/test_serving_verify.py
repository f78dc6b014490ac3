"""Verification of drafted tokens: whole numbers, equal to the oracle's.  Its sums are in 64 bits on both sides, in other orders: a border between two tokens lies within 2^-50 of the
same place, and the random numbers here are fixed."""
import gc

import numpy as np
import pytest
import torch

from oracle import drafts, kv4
from oracle.attention import bf16_to_f64
from paper_2609_24270_b200 import binding as ag
from tests.test_serving_kv4 import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def give_memory_back():
    """Tests that look at addresses or at free memory find torch's allocator without blocks of these."""
    yield
    gc.collect()
    torch.cuda.empty_cache()


def softmax(x):
    e = np.exp(x - x.max(-1, keepdims=True))
    return e / e.sum(-1, keepdims=True)


def trees(rng, counts, width):
    out = []
    for n in counts:
        kids, par = [0] * n, [-1] if n else []
        for i in range(1, n):
            p = int(rng.choice([j for j in range(i) if kids[j] < width]))
            kids[p] += 1
            par.append(p)
        out += par
    return np.array(out, np.int32)


class Step:
    """A batch: probabilities of both models, drafts drawn from the drafting one."""

    def __init__(self, counts, vocab, width=1, bits=32, far=1.0, distinct=False, seed=0, peak=1.5):
        rng = np.random.default_rng(seed)
        n = sum(counts)
        self.off, self.parent = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32), trees(rng, counts, width)
        logits = peak * rng.standard_normal((n, vocab))
        self.P, self.Q = (softmax(x).astype(np.float32) for x in (logits, logits + far * rng.standard_normal((n, vocab))))
        if bits == 16:
            self.P, self.Q = kv4.f32_to_bf16_value(self.P), kv4.f32_to_bf16_value(self.Q)
        self.token, tried = np.zeros(n, np.int32), {}
        for s in range(len(counts)):
            for i in range(self.off[s] + 1, self.off[s + 1]):
                p = self.off[s] + self.parent[i]
                w = self.Q[p].astype(np.float64)
                if distinct:
                    w[tried.get(p, [])] = 0
                self.token[i] = rng.choice(vocab, p=w / w.sum()) if w.sum() > 0 else 0
                tried.setdefault(p, []).append(self.token[i])
        self.u, self.u_next = rng.random(n).astype(np.float32), rng.random(len(counts)).astype(np.float32)
        self.u, self.u_next = np.minimum(self.u, np.float32(1 - 2 ** -24)), np.minimum(self.u_next, np.float32(1 - 2 ** -24))
        self.bits, self.distinct, self.vocab = bits, distinct, vocab

    def device(self, pad=0, q_pad=None, shift=0):
        """Rows `pad` entries apart more than they are long, from entry `shift` on; what lies between is NaN."""
        def put(x, more):
            if x is None:
                return None, None, 0
            kind = torch.bfloat16 if self.bits == 16 else torch.float32
            buf = torch.full((x.shape[0] * (self.vocab + more) + shift + 16,), float("nan"), dtype=kind, device="cuda")
            view = buf[shift:shift + x.shape[0] * (self.vocab + more)].view(x.shape[0], -1)[:, :self.vocab]
            view.copy_(torch.from_numpy(x).cuda().to(kind))
            return buf, view, self.vocab + more
        self.bufs = put(self.P, pad), put(self.Q, pad if q_pad is None else q_pad)
        self.d = {k: dev(getattr(self, k)) for k in ("off", "parent", "token", "u", "u_next")}

    def run(self, stream=0, chain=False, n_seq=None):
        n, S = len(self.token), len(self.off) - 1
        (_, p, ps), (_, q, qs) = self.bufs
        out = [torch.full((k,), -9, dtype=torch.int32, device="cuda") for k in (n, S, S + 1, n)]
        torch.cuda.synchronize()
        ag.verify_drafts(p.data_ptr(), None if q is None else q.data_ptr(), self.vocab, self.d["token"].data_ptr(), None if chain else self.d["parent"].data_ptr(), self.d["off"].data_ptr(),
                         S, n, self.d["u"].data_ptr(), self.d["u_next"].data_ptr(), *(o.data_ptr() for o in out), p_stride=ps, q_stride=qs, bf16=self.bits == 16, distinct=self.distinct,
                         stream=stream)
        torch.cuda.synchronize()
        return [o.cpu().numpy() for o in out]

    def want(self, chain=False):
        f = lambda x: None if x is None else x.astype(np.float64)  # noqa: E731
        return drafts.verify(f(self.P), f(self.Q), self.token, None if chain else self.parent, self.off, self.u, self.u_next, self.distinct)


def same(got, want):
    for g, w, name in zip(got, want, ("accepted", "next", "new_off", "rows")):
        assert (g == w).all(), (name, g, w)


@pytest.mark.parametrize("vocab", [1, 2, 7, 64, 1000, 4096, 33333])
@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("drawn", ["replace", "distinct", "certain"])
def test_trees_and_chains(vocab, bits, drawn):
    for width, seed in ((1, 1), (3, 2), (6, 3)):
        s = Step([1, 5, 9, 0, 16, 2], vocab, width, bits, 1.0, drawn == "distinct", seed)
        if drawn == "certain":
            s.Q = None
        s.device()
        same(s.run(), s.want())
    same(s.run(chain=True), s.want(chain=True))


@pytest.mark.parametrize("pad,q_pad,shift", [(0, 0, 1), (3, 3, 0), (5, 5, 2), (1, 2, 0), (8, 0, 3)])
@pytest.mark.parametrize("bits", [16, 32])
def test_strides_and_alignments(pad, q_pad, shift, bits):
    """Rows that do not begin on 16 bytes, or p's and q's differently; nothing between the rows counts."""
    for vocab in (129, 5000):
        s = Step([6, 11, 3], vocab, 2, bits, seed=pad + vocab)
        s.device(pad, q_pad, shift)
        same(s.run(), s.want())


def test_many_requests_of_all_block_counts():
    for S, vocab in ((40, 700), (80, 700), (160, 300), (400, 130)):
        rng = np.random.default_rng(S)
        s = Step(list(rng.integers(0, 7, S)), vocab, 2, seed=S)
        s.device()
        same(s.run(), s.want())


def test_long_chain_and_tokens_beyond_the_most():
    s = Step([64, 90, 3], 50, 1, far=0.2, seed=4)
    s.u[:] = 0.0                                     # everything with p > 0 is accepted
    s.parent = np.concatenate([np.arange(-1, n - 1) for n in (64, 90, 3)]).astype(np.int32)
    s.device()
    got = s.run()
    same(got, s.want())
    assert got[0][:64].all() and got[0][64:128].all() and not got[0][128:154].any()


def test_edges():
    """p = q; p below q everywhere; one-hot rows; a token outside the vocabulary; a parent behind its child; random numbers of 0; a row without weight."""
    V = 300
    s = Step([4, 4, 4, 4, 4, 4, 4], V, 3, seed=6)
    s.Q[0:4] = s.P[0:4]
    s.u[0:4] = 1 - 2.0 ** -24
    s.Q[4:8] = np.float32(2.0) * s.P[4:8]
    s.P[8:12] = 0
    s.P[8:12, 17] = 1
    s.token[13], s.token[14] = V, -3
    s.parent[16:20] = [-1, 2, 0, 3]
    s.u[20:24], s.u_next[5] = 0.0, 0.0
    s.P[24:28] = 0
    s.device()
    got = s.run()
    same(got, s.want())
    assert got[1][2] == 17 and got[1][6] == -1 and not got[0][13:15].any() and not got[0][17]
    s.distinct = True
    same(s.run(), s.want())
    s.Q, s.distinct = None, False
    s.device()
    same(s.run(), s.want())


def test_siblings_with_what_stays_when_nothing_is_left():
    """p lies below q everywhere: a rejected draft leaves r as it was, itself included."""
    rng = np.random.default_rng(8)
    s = Step([5] * 30, 40, 4, seed=9, distinct=True)
    s.parent = np.tile([-1, 0, 0, 0, 0], 30).astype(np.int32)
    s.P = (s.Q * np.float32(0.25)).astype(np.float32)
    s.token = np.concatenate([[0, *rng.permutation(40)[:4]] for _ in range(30)]).astype(np.int32)
    for distinct in (True, False):
        s.distinct = distinct
        s.device()
        got = s.run()
        same(got, s.want())
    assert got[0].sum() < 150


def test_the_same_draft_twice():
    s = Step([4] * 20, 12, 3, seed=10)
    s.parent = np.tile([-1, 0, 0, 0], 20).astype(np.int32)
    s.token[1::4] = s.token[2::4]
    s.token[3::4] = s.token[2::4]
    for distinct in (False, True):
        s.distinct = distinct
        s.device()
        same(s.run(), s.want())
    s.Q = None
    s.device()
    same(s.run(), s.want())


@pytest.mark.parametrize("distinct", [False, True])
def test_text_is_distributed_as_the_target_has_it(distinct):
    """40000 requests with the same p and q: the token behind the root comes up n p times, five deviations of sqrt(n p (1 - p)) allowed; two drafts each."""
    S, V, rng = 40000, 9, np.random.default_rng(11 + distinct)
    p, q = softmax(rng.standard_normal(V)).astype(np.float32), softmax(rng.standard_normal(V)).astype(np.float32)
    keys = np.log(q) + rng.gumbel(size=(S, V))
    first = keys.argmax(1)
    second = np.argsort(-keys, 1)[:, 1] if distinct else (np.log(q) + rng.gumbel(size=(S, V))).argmax(1)
    token = np.stack([np.zeros(S), first, second], 1).astype(np.int32)
    d = {k: dev(v) for k, v in dict(off=(3 * np.arange(S + 1)).astype(np.int32), token=token.reshape(-1), parent=np.tile([-1, 0, 0], S).astype(np.int32),
                                    u=rng.random(3 * S).astype(np.float32) * np.float32(1 - 2.0 ** -24), u_next=rng.random(S).astype(np.float32) * np.float32(1 - 2.0 ** -24)).items()}
    P, Q = (torch.from_numpy(x).cuda().repeat(3 * S, 1) for x in (p, q))
    out = [torch.empty(k, dtype=torch.int32, device="cuda") for k in (3 * S, S)]
    ag.verify_drafts(P.data_ptr(), Q.data_ptr(), V, d["token"].data_ptr(), d["parent"].data_ptr(), d["off"].data_ptr(), S, 3 * S, d["u"].data_ptr(), d["u_next"].data_ptr(),
                     out[0].data_ptr(), out[1].data_ptr(), distinct=distinct)
    torch.cuda.synchronize()
    acc, nxt = out[0].cpu().numpy().reshape(S, 3), out[1].cpu().numpy()
    text = np.where(acc[:, 1] > 0, token[:, 1], np.where(acc[:, 2] > 0, token[:, 2], nxt))
    seen, mean = np.bincount(text, minlength=V), S * p.astype(np.float64)
    assert (np.abs(seen - mean) <= 5 * np.sqrt(mean * (1 - p))).all(), (seen, mean)


def test_requests_that_own_no_tokens_and_tokens_that_no_request_owns():
    s = Step([3, 4], 100, 1, seed=12)
    s.off = np.array([2, 5, 5, 60], np.int32)           # tokens 0, 1 belong to nobody; offsets beyond the tokens are clamped
    s.u_next = np.array([.1, .2, .3], np.float32)
    s.parent = np.array([0, 0, -1, 0, 1, -1, 0], np.int32)
    s.device()
    got = s.run()
    s.off[3] = 7
    want = s.want()
    assert (got[0][:2] == -9).all() and (got[0][2:] == want[0][2:]).all() and got[1].tolist() == want[1].tolist() and got[1][1] == -1
    assert got[2].tolist() == want[2].tolist() and (got[3] == want[3]).all()


def test_streams_and_graphs():
    s, t = Step([5, 9, 2], 20000, 2, seed=13), Step([8] * 70, 900, 3, seed=14)
    s.device(), t.device()
    want = s.want(), t.want()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = []
    torch.cuda.synchronize()
    for _ in range(3):
        for x, st in zip((s, t), streams):
            n, S = len(x.token), len(x.off) - 1
            out = [torch.full((k,), -9, dtype=torch.int32, device="cuda") for k in (n, S, S + 1, n)]
            st.wait_stream(torch.cuda.current_stream())
            ag.verify_drafts(x.bufs[0][1].data_ptr(), x.bufs[1][1].data_ptr(), x.vocab, x.d["token"].data_ptr(), x.d["parent"].data_ptr(), x.d["off"].data_ptr(), S, n,
                             x.d["u"].data_ptr(), x.d["u_next"].data_ptr(), *(o.data_ptr() for o in out), stream=st.cuda_stream)
            outs.append(out)
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        same([x.cpu().numpy() for x in o], want[i % 2])
    out = outs[0]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=streams[0]):
        ag.verify_drafts(s.bufs[0][1].data_ptr(), s.bufs[1][1].data_ptr(), s.vocab, s.d["token"].data_ptr(), s.d["parent"].data_ptr(), s.d["off"].data_ptr(), 3, len(s.token),
                         s.d["u"].data_ptr(), s.d["u_next"].data_ptr(), *(o.data_ptr() for o in out), stream=torch.cuda.current_stream().cuda_stream)
    s.u = np.random.default_rng(15).random(len(s.u)).astype(np.float32)
    s.d["u"].copy_(torch.from_numpy(s.u))
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    same([x.cpu().numpy() for x in out], s.want())


def test_rows_beyond_two_to_the_32_bytes():
    V, n = 1 << 18, 4200                                 # 4.4 GB of p
    P = torch.zeros(n, V, dtype=torch.float32, device="cuda")
    P[:, 5], P[-1, 5], P[-1, V - 1] = 1.0, 0.25, 0.75
    token = dev(np.full(n, 5, np.int32))
    off, u, u_next = dev(np.array([0, 2, n - 2, n], np.int32)), dev(np.full(n, .5, np.float32)), dev(np.array([.3, .3, .3], np.float32))
    out = [torch.empty(k, dtype=torch.int32, device="cuda") for k in (n, 3, 4, n)]
    ag.verify_drafts(P.data_ptr(), None, V, token.data_ptr(), None, off.data_ptr(), 3, n, u.data_ptr(), u_next.data_ptr(), *(o.data_ptr() for o in out))
    torch.cuda.synchronize()
    assert out[1].tolist() == [5, 5, V - 1] and out[2].tolist() == [0, 2, 66, 68]


@pytest.mark.parametrize("vocab", [5, 200, 5003])
@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("kind", ["one", "nearly", "far", "several"])
def test_siblings_drawn_from_a_concentrated_q(kind, bits, vocab):
    """Without repetition, q all but used up by the first siblings: a token to which the target gives nothing is neither accepted nor sampled, whatever the random numbers are."""
    counts = [5, 5, 6, 4, 2, 5, 16] * 6
    s = Step(counts, vocab, 4, bits, distinct=True, seed=vocab + bits)
    rng, n = np.random.default_rng(vocab), sum(counts)
    logits = rng.standard_normal((n, vocab))
    if kind == "several":
        logits *= 6
    else:
        logits[np.arange(n), rng.integers(0, vocab, n)] += dict(one=300, nearly=7.5 if bits == 16 else 18, far=19 if bits == 16 else 40)[kind]
    s.Q = softmax(logits).astype(np.float32)
    s.P = softmax(2 * rng.standard_normal((n, vocab))).astype(np.float32) * (rng.random((n, vocab)) < .5)
    s.P[:, 0] += 2.0 ** -10                                                          # (no row without weight)
    s.P = (s.P / s.P.sum(1, keepdims=True, dtype=np.float64)).astype(np.float32)
    if bits == 16:
        s.P, s.Q = kv4.f32_to_bf16_value(s.P), kv4.f32_to_bf16_value(s.Q)
    s.token[:] = 0
    for a, b in zip(s.off[:-1], s.off[1:]):
        tried = {}
        for i in range(a + 1, b):
            w = s.Q[a + s.parent[i]].astype(np.float64)
            w[tried.setdefault(s.parent[i], [])] = 0
            s.token[i] = rng.choice(vocab, p=w / w.sum()) if w.sum() > 0 else rng.integers(0, vocab)
            tried[s.parent[i]].append(s.token[i])
    s.u[1::2] = 0.5
    s.device()
    got = s.run()
    same(got, s.want())
    first = np.repeat(s.off[:-1], counts)
    drafts_in = (got[0] > 0) & (s.parent >= 0)
    assert (s.P[(first + s.parent)[drafts_in], s.token[drafts_in]] > 0).all()
    for r, (a, b) in enumerate(zip(s.off[:-1], s.off[1:])):
        last = a + np.flatnonzero(got[0][a:b])[-1]
        assert s.P[last, got[1][r]] > 0
    s.d["parent"].fill_(0)                                                           # all of a request's drafts as siblings, tokens and random numbers as they are
    for a in s.off[:-1]:
        s.d["parent"][int(a)] = -1
    s.parent = s.d["parent"].cpu().numpy()
    same(s.run(), s.want())


@pytest.mark.parametrize("bits,peak,seed", [(16, 6, 3), (16, 6, 4), (16, 6, 5), (32, 20, 0), (32, 20, 4), (32, 12, 3)])
def test_text_of_a_concentrated_q_is_distributed_as_the_target_has_it(bits, peak, seed):
    """40000 requests of three siblings drawn without repetition: five deviations, and what the header says of rows that do not sum to 1."""
    S, V, rng = 40000, 6, np.random.default_rng(seed)
    p, q = (softmax(k * rng.standard_normal(V)).astype(np.float32) for k in (1, peak))
    if bits == 16:
        p, q = kv4.f32_to_bf16_value(p), kv4.f32_to_bf16_value(q)
    first = np.argsort(-(np.log(q.astype(np.float64)) + rng.gumbel(size=(S, V))), 1)[:, :3]
    token = np.concatenate([np.zeros((S, 1)), first], 1).astype(np.int32)
    d = {k: dev(v) for k, v in dict(off=(4 * np.arange(S + 1)).astype(np.int32), token=token.reshape(-1), parent=np.tile([-1, 0, 0, 0], S).astype(np.int32),
                                    u=rng.random(4 * S).astype(np.float32) * np.float32(1 - 2.0 ** -24), u_next=rng.random(S).astype(np.float32) * np.float32(1 - 2.0 ** -24)).items()}
    kind = torch.bfloat16 if bits == 16 else torch.float32
    P, Q = (torch.from_numpy(x).cuda().to(kind).repeat(4 * S, 1) for x in (p, q))
    out = [torch.empty(k, dtype=torch.int32, device="cuda") for k in (4 * S, S)]
    ag.verify_drafts(P.data_ptr(), Q.data_ptr(), V, d["token"].data_ptr(), d["parent"].data_ptr(), d["off"].data_ptr(), S, 4 * S, d["u"].data_ptr(), d["u_next"].data_ptr(),
                     out[0].data_ptr(), out[1].data_ptr(), bf16=bits == 16, distinct=True)
    torch.cuda.synchronize()
    acc, nxt = out[0].cpu().numpy().reshape(S, 4)[:, 1:], out[1].cpu().numpy()
    text = np.where(acc.any(1), first[np.arange(S), acc.argmax(1)], nxt)
    p, q = p.astype(np.float64), q.astype(np.float64)
    seen, mean = np.bincount(text, minlength=V), S * p / p.sum()
    off = abs(p.sum() - q.sum()) / max(p.sum(), q.sum()) + 2 * abs(1 - q.sum())
    assert (np.abs(seen - mean) <= 5 * np.sqrt(mean * (1 - p)) + S * off + 1).all(), (seen, mean)


@pytest.mark.parametrize("S", [1, 3, 700])
def test_no_tokens_at_all(S):
    off, u_next = torch.zeros(S + 1, dtype=torch.int32, device="cuda"), torch.zeros(S, device="cuda")
    nxt, new_off = torch.full((S,), -9, dtype=torch.int32, device="cuda"), torch.full((S + 1,), -9, dtype=torch.int32, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda").data_ptr() or None
    ag.verify_drafts(none, none, 100, none, none, off.data_ptr(), S, 0, none, u_next.data_ptr(), none, nxt.data_ptr(), new_off.data_ptr(), none)
    torch.cuda.synchronize()
    assert (nxt == -1).all() and (new_off == 0).all()


@pytest.mark.parametrize("pad,q_pad,shift", [(0, 0, 1), (3, 3, 0), (5, 5, 2), (1, 2, 0), (8, 0, 3)])
@pytest.mark.parametrize("bits", [16, 32])
def test_what_is_left_of_rows_at_any_stride(pad, q_pad, shift, bits):
    """Siblings without repetition over rows that begin anywhere, one entry at a time where p's and q's lie differently; tokens at a row's ends among them."""
    for vocab in (131, 2050):
        s = Step([6, 11, 3, 16, 9], vocab, 5, bits, distinct=True, seed=pad + vocab, peak=4.0)
        s.P = np.roll(s.P, 1, 1)                                                      # far from q: many are refused
        s.token[3::7], s.token[5::7] = 0, vocab - 1
        s.device(pad, q_pad, shift)
        same(s.run(), s.want())
