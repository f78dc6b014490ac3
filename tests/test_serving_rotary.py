"""Rotary positions and the append that turns keys on their way into the 4-bit cache, against the 64-bit oracle.

Tolerance: cosine and sine are rounded to 32 bits, a product is, and a multiply-add is: at most 2^-24 of what they are each, together below 2^-22 (|a| + |b|) magnitude; the output is
rounded to bf16, 2^-8 of itself (2^-133 below the smallest normal).  The angle, position * frequency in 64 bits, is off by 2^-53 of itself: 2^-33 for a million radians.
An append holds bit for bit what ag_rotary_apply and ag_kv4_store make one after the other."""
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


def rows(n, H, D, seed, stretch=1.0):
    return kv4.bf16_bits(kv4.f32_to_bf16_value(stretch * np.random.default_rng(seed).standard_normal((n, H, D)).astype(np.float32)))


def rotary(rot, pairs, freq, magnitude=1.0):
    d = torch.from_numpy(np.ascontiguousarray(freq)).cuda()
    r = ag.Rotary(d.data_ptr(), rot, ag.AG_ROTARY_PAIRS if pairs else ag.AG_ROTARY_HALVES, magnitude)
    r.keep = d
    return r


def check(got, x, pos, freq, magnitude, pairs):
    want = drafts.rotate(x, pos, freq, magnitude, pairs)
    rot, half = 2 * len(freq), len(freq)
    reach = np.zeros(x.shape)
    a, b = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if pairs else (np.arange(half), np.arange(half, rot))
    reach[..., a] = reach[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    bound = 2.0 ** -8 * np.abs(want) + 2.0 ** -21 * magnitude * reach + 2.0 ** -133
    got = got.float().cpu().numpy().astype(np.float64)
    assert (got[..., rot:] == x[..., rot:]).all()
    assert (np.abs(got - want) <= bound).all(), float((np.abs(got - want) / bound).max())


CASES = [(64, 16, False, 1), (64, 32, True, 3), (64, 48, False, 2), (64, 64, False, 7), (64, 64, True, 8), (128, 16, True, 1), (128, 48, False, 5), (128, 64, False, 4), (128, 80, True, 3),
         (128, 112, False, 1), (128, 128, False, 9), (128, 128, True, 2)]


@pytest.mark.parametrize("D,rot,pairs,H", CASES)
def test_turned_rows(D, rot, pairs, H):
    n, H_kv = 13, max(1, H // 3)
    pos = np.array([0, 1, 2, 7, 100, 4095, 131071, 999999, -1, -50000, 2 ** 31 - 1, -2 ** 31, 12], np.int32)
    freq, magnitude = drafts.frequencies(rot, 10000.0, drafts.RAMP, 16.0, 4096.0, 1.0, 32.0)
    Q, K = rows(n, H, D, 1, 3.0), rows(n, H_kv, D, 2)
    r, dQ, dK, dp = rotary(rot, pairs, freq, magnitude), dev(Q), dev(K), dev(pos)
    oQ, oK = (torch.full(x.shape, float("nan"), dtype=torch.bfloat16, device="cuda") for x in (Q, K))
    ag.rotary_apply(r, dp.data_ptr(), n, D, dQ.data_ptr(), oQ.data_ptr(), H, dK.data_ptr(), oK.data_ptr(), H_kv)
    torch.cuda.synchronize()
    # at 2^31 radians an angle is off by 2^-22: those two rows get twice the room
    x, y = bf16_to_f64(Q), bf16_to_f64(K)
    near = np.abs(pos.astype(np.int64)) < 2 ** 30
    check(oQ[torch.from_numpy(near).cuda()], x[near], pos[near], freq, magnitude, pairs)
    check(oK[torch.from_numpy(near).cuda()], y[near], pos[near], freq, magnitude, pairs)
    far = oQ.float().cpu().numpy().astype(np.float64)[~near]
    assert np.abs(far - drafts.rotate(x[~near], pos[~near], freq, magnitude, pairs)).max() <= 2.0 ** -8 * np.abs(far).max() + 1e-4
    # one of the two alone, in place; parts of a wider buffer
    assert dQ.data_ptr() % 16 == 0
    ag.rotary_apply(r, dp.data_ptr(), n, D, k_ptr=dK.data_ptr(), k_out_ptr=dK.data_ptr(), H_kv=H_kv)
    torch.cuda.synchronize()
    assert torch.equal(dK, oK.view(torch.int16))
    wide = torch.zeros(n, H + H_kv + 1, D, dtype=torch.bfloat16, device="cuda")
    wide[:, :H], wide[:, H:H + H_kv] = dev(Q).view(torch.bfloat16), dev(K).view(torch.bfloat16)
    ag.rotary_apply(r, dp.data_ptr(), n, D, wide.data_ptr(), wide.data_ptr(), H, wide[:, H:].data_ptr(), wide[:, H:].data_ptr(), H_kv, q_stride=wide.stride(0), k_stride=wide.stride(0),
                    q_out_stride=wide.stride(0), k_out_stride=wide.stride(0))
    torch.cuda.synchronize()
    assert torch.equal(wide[:, :H], oQ) and torch.equal(wide[:, H:H + H_kv], oK) and not wide[:, H + H_kv:].any()


def test_values_that_are_not_finite_stay_in_their_pairs():
    n, D, rot = 2, 64, 32
    X = rows(n, 3, D, 3)
    X[0, 1, 3], X[1, 2, 40], X[1, 0, 33] = 0x7FC0, 0x7F80, 0x8000
    freq, _ = drafts.frequencies(rot)
    for pairs in (False, True):
        d, out, pos = dev(X), torch.empty(n, 3, D, dtype=torch.bfloat16, device="cuda"), dev(np.array([5, 6], np.int32))
        ag.rotary_apply(rotary(rot, pairs, freq), pos.data_ptr(), n, D, d.data_ptr(), out.data_ptr(), 3)
        torch.cuda.synchronize()
        odd = ~torch.isfinite(out).cpu().numpy()
        where = {(0, 1, 3), (0, 1, 2 if pairs else 19), (1, 2, 40)}
        assert set(zip(*(a.tolist() for a in np.nonzero(odd)))) == where
        assert (out.view(torch.int16).cpu().numpy().view(np.uint16)[..., rot:] == X[..., rot:]).all()      # (a negative zero among them)


@pytest.mark.parametrize("D,rot,pairs,H_kv,H_q", [(64, 64, False, 1, 3), (64, 16, True, 5, 5), (64, 48, False, 8, 16), (128, 128, False, 8, 32), (128, 64, True, 3, 3), (128, 112, False, 2, 6),
                                                  (128, 128, True, 9, 0), (128, 0, False, 4, 4), (64, 0, False, 2, 0)])
@pytest.mark.parametrize("n", [1, 37, 700])
def test_append_is_turn_and_store(D, rot, pairs, H_kv, H_q, n):
    rng = np.random.default_rng(n + rot)
    n_pages = n // 64 + 3
    slots = rng.permutation(n_pages * 64)[:n].astype(np.int32)
    slots[rng.random(n) < 0.1] = -1
    if n > 1:
        slots[0], slots[1] = n_pages * 64, 2 ** 31 - 1                    # outside: nothing is stored
    K, V, Q = rows(n, H_kv, D, 5, 1.3), rows(n, H_kv, D, 6), rows(n, max(H_q, 1), D, 7)
    K[0, 0, 5] = 0x7F80
    pos = rng.integers(0, 200000, n).astype(np.int32)
    d = {k: dev(v) for k, v in dict(K=K, V=V, Q=Q, slot=slots, pos=pos).items()}
    fill = torch.from_numpy(rng.integers(0, 256, (n_pages, H_kv, 80 * D)).astype(np.uint8)).cuda()
    one, two = fill.clone(), fill.clone()
    r = rotary(rot, pairs, drafts.frequencies(rot)[0], 1.25) if rot else None
    kT, qT, kO, qO = (torch.empty(x.shape, dtype=torch.bfloat16, device="cuda") for x in (K, Q, K, Q))
    if rot:
        ag.rotary_apply(r, d["pos"].data_ptr(), n, D, *((d["Q"].data_ptr(), qT.data_ptr(), H_q) if H_q else (None, None, 0)), d["K"].data_ptr(), kT.data_ptr(), H_kv)
    else:
        kT, qT = d["K"].view(torch.bfloat16), d["Q"].view(torch.bfloat16)
    ag.kv4_store(ag.KV4Pool(one.data_ptr(), n_pages, H_kv, D), kT.data_ptr(), d["V"].data_ptr(), d["slot"].data_ptr(), n)
    for with_k in (False, True):
        two.copy_(fill)
        ask = dict(q_ptr=d["Q"].data_ptr(), q_out_ptr=qO.data_ptr(), H_q=H_q) if H_q else {}
        ag.kv4_append_rotary(ag.KV4Pool(two.data_ptr(), n_pages, H_kv, D), r, d["pos"].data_ptr() if rot else None, d["slot"].data_ptr(), n, d["K"].data_ptr(), d["V"].data_ptr(),
                             k_out_ptr=kO.data_ptr() if with_k else None, **ask)
        torch.cuda.synchronize()
        assert torch.equal(one, two)
        bits = lambda t: t.view(torch.int16)  # noqa: E731
        assert not H_q or torch.equal(bits(qO), bits(qT))
        assert not with_k or torch.equal(bits(kO), bits(kT))
    # the oracle's bytes, from the turned keys
    if n <= 37:
        want = fill.cpu().numpy()
        kv4.store(want, D, kT.view(torch.int16).cpu().numpy().view(np.uint16), V, slots)
        assert (two.cpu().numpy() == want).all()


def test_rows_by_index():
    """Chosen rows of wider buffers, as the commit of accepted drafts takes them; an index outside passes its token over."""
    D, H_kv, H_q, have, n = 128, 2, 4, 50, 20
    rng = np.random.default_rng(3)
    frm = rng.integers(0, have, n).astype(np.int32)
    frm[3], frm[7], frm[19] = -1, have, frm[0]
    slots, pos = np.arange(n, dtype=np.int32)[::-1].copy(), rng.integers(0, 5000, n).astype(np.int32)
    K, V, Q = rows(have, H_kv, D, 8), rows(have, H_kv, D, 9), rows(have, H_q, D, 10)
    qkv = torch.cat([dev(x).view(torch.bfloat16) for x in (Q, K, V)], 1)
    freq, _ = drafts.frequencies(64)
    r, d = rotary(64, False, freq), {k: dev(v) for k, v in dict(frm=frm, slot=slots, pos=pos).items()}
    pages = torch.zeros(1, H_kv, 80 * D, dtype=torch.uint8, device="cuda")
    qO = torch.full((n, H_q, D), -7.0, dtype=torch.bfloat16, device="cuda")
    ag.kv4_append_rotary(ag.KV4Pool(pages.data_ptr(), 1, H_kv, D), r, d["pos"].data_ptr(), d["slot"].data_ptr(), n, qkv[:, H_q:].data_ptr(), qkv[:, H_q + H_kv:].data_ptr(),
                         q_ptr=qkv.data_ptr(), q_out_ptr=qO.data_ptr(), H_q=H_q, k_stride=qkv.stride(0), v_stride=qkv.stride(0), q_stride=qkv.stride(0),
                         from_ptr=d["frm"].data_ptr(), n_rows=have)
    torch.cuda.synchronize()
    fine = (frm >= 0) & (frm < have)
    check(qO[torch.from_numpy(fine).cuda()], bf16_to_f64(Q)[frm[fine]], pos[fine], freq, 1.0, False)
    assert (qO[torch.from_numpy(~fine).cuda()] == -7.0).all()
    kT = torch.empty(n, H_kv, D, dtype=torch.bfloat16, device="cuda")
    picked = qkv[:, H_q:H_q + H_kv][torch.from_numpy(frm.clip(0, have - 1)).long().cuda()].contiguous()
    ag.rotary_apply(r, d["pos"].data_ptr(), n, D, k_ptr=picked.data_ptr(), k_out_ptr=kT.data_ptr(), H_kv=H_kv)
    torch.cuda.synchronize()
    want = np.zeros((1, H_kv, 80 * D), np.uint8)
    kv4.store(want, D, kT.view(torch.int16).cpu().numpy().view(np.uint16)[fine], V[frm[fine]], slots[fine])
    assert (pages.cpu().numpy() == want).all()


def test_other_streams_graphs_and_far_rows():
    """Two calls at once on streams of their own; a captured call sees what the buffers hold when it runs; rows beyond 2^32 bytes."""
    D, H, n = 128, 8, 300
    freq, _ = drafts.frequencies(128)
    r, X, pos = rotary(128, False, freq), rows(n, H, D, 11), np.arange(n, dtype=np.int32) * 17
    d, dp = dev(X), dev(pos)
    outs = [torch.zeros(n, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for o, s in zip(outs, streams):
        ag.rotary_apply(r, dp.data_ptr(), n, D, d.data_ptr(), o.data_ptr(), H, stream=s.cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])
    check(outs[0], bf16_to_f64(X), pos, freq, 1.0, False)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=streams[0]):
        ag.rotary_apply(r, dp.data_ptr(), n, D, d.data_ptr(), outs[2].data_ptr(), H, stream=torch.cuda.current_stream().cuda_stream)
    dp.add_(3)
    g.replay()
    torch.cuda.synchronize()
    check(outs[2], bf16_to_f64(X), pos + 3, freq, 1.0, False)
    wide = torch.zeros((1 << 32) // 2 * 2 + 4096, dtype=torch.bfloat16, device="cuda")        # 8 GB: three rows 2^31 elements apart
    step = (1 << 31) - 8 * 16
    for i in range(3):
        wide[i * step:i * step + H * D] = dev(X[i]).view(torch.bfloat16).reshape(-1)
    o = torch.empty(3, H, D, dtype=torch.bfloat16, device="cuda")
    ag.rotary_apply(r, dp.data_ptr(), 3, D, wide.data_ptr(), o.data_ptr(), H, q_stride=step)
    torch.cuda.synchronize()
    check(o, bf16_to_f64(X[:3]), (pos + 3)[:3], freq, 1.0, False)
