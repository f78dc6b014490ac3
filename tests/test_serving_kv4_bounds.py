"""What the header says of the roundings in single-token attention over the 4-bit cache, term by term, at inputs where each of them shows.

Per output, with v, s, b (value, scale, base) of the cache, p the exact probabilities, u = 2^-11 half a step of fp16:
  values          (16 + u) s + c with c = b - 16 s: c is rounded once (u |c|), the result once (u |v|), s is exact; at fp16's lower end 2^-32 of the row's largest
  probabilities   u p, or 2^-35 of the largest; the exponential, its argument and the sums in 32 bits: 2^-18 p
  scores          e = (2^-13 sum |q| s + 2^-21 sum |q| (15 s + |b|)) / sqrt D, largest over the keys: an output moves by at most (exp(2 e) - 1) sum p |v|
  output          rounded to bf16, 2^-8 of itself."""
import gc

import numpy as np
import pytest
import torch

from oracle import kv4
from oracle.attention import bf16_to_f64
from tests.test_serving_kv4_decode import make, queries, run

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def give_memory_back():
    """Tests that look at addresses or at free memory find torch's allocator without blocks of these."""
    yield
    gc.collect()
    torch.cuda.empty_cache()


def groups(c, which):
    """scale and base of every slot and group, as float64 [slots][H_kv][D / 32]."""
    at = 64 * c.D + which * 8 * c.D
    sb = bf16_to_f64(c.pages[:, :, at:at + 8 * c.D].copy().view(np.uint16)).reshape(c.pages.shape[0], c.pages.shape[1], 64, c.D // 32, 2)
    sb = sb.transpose(0, 2, 1, 3, 4).reshape(-1, c.pages.shape[1], c.D // 32, 2)
    return sb[..., 0], sb[..., 1]


def within_the_bounds(Q, c, got):
    D, H_kv, n_pages = c.D, c.pages.shape[1], c.pages.shape[0]
    K, V = kv4.load(c.pages, D, np.arange(n_pages * 64))
    (ks, kb), (vs, vb) = groups(c, 0), groups(c, 1)
    Qf, u = bf16_to_f64(Q), 2.0 ** -11
    G = Q.shape[1] // H_kv
    for r in range(len(Q)):
        n = int(c.len[r])
        slots = np.repeat(c.page_of[r].astype(np.int64), 64)[:n] * 64 + np.arange(n) % 64
        for hq in range(Q.shape[1]):
            h, q = hq // G, Qf[r, hq]
            k, v = K[slots, h], V[slots, h]
            x = k @ q / np.sqrt(D)
            p = np.exp(x - x.max())
            p /= p.sum()
            want, mass = p @ v, p @ np.abs(v)
            by_group = np.abs(q).reshape(-1, 32).sum(1)
            e = ((2.0 ** -13 * ks[slots, h] + 2.0 ** -21 * (15 * ks[slots, h] + np.abs(kb[slots, h]))) @ by_group).max() / np.sqrt(D)
            off = u * (1 + 2.0 ** -10) * (np.abs(v) + np.repeat(np.abs(vb[slots, h] - 16 * vs[slots, h]), 32, -1)) + 2.0 ** -32 * np.abs(v).max()
            bound = 2.0 ** -8 * np.abs(want) + p @ off + (u + 2.0 ** -18 + np.expm1(2 * e)) * mass + 2.0 ** -35 * p.max() * np.abs(v).sum(0) + 1e-30
            assert (np.abs(got[r, hq] - want) <= bound).all(), (r, hq, float((np.abs(got[r, hq] - want) / bound).max()))


def set_values(c, scale, base, codes=None):
    """All values of the cache: scale and base by [page][head][token][group], codes as they are or set."""
    n, H = c.pages.shape[:2]
    pair = kv4.bf16_bits(kv4.f32_to_bf16_value(np.stack(np.broadcast_arrays(scale, base), -1).astype(np.float32)))
    c.pages[:, :, 72 * c.D:] = pair.reshape(n, H, -1).view(np.uint8)
    if codes is not None:
        c.pages[:, :, 32 * c.D:64 * c.D] = codes
    c.push()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", [[1, 2, 64, 150], [3000, 700]])
def test_usual_values(D, lens):
    c = make(lens, 2, D, seed=31)
    for peak in (0.05, 1.0, 4.0):
        Q = queries(len(lens), 8, D, 32, peak)
        within_the_bounds(Q, c, run(Q, c))


@pytest.mark.parametrize("D", [64, 128])
def test_values_that_cancel(D):
    """Tokens in pairs with the same key and opposite values: what is left of the output is what the roundings leave."""
    c = make([64, 640, 1300], 1, D, seed=33)
    n = c.pages.shape[0]
    rng = np.random.default_rng(34)
    block = c.pages.reshape(n, 80 * D)
    for t in range(0, 64, 2):                                     # the odd token's key is the even one's
        for d in range(0, D, 2):                                  # (two elements a byte)
            a, b = kv4.byte_of(D, 0, t, d)[0], kv4.byte_of(D, 0, t + 1, d)[0]
            block[:, b] = block[:, a]
        for g in range(D // 32):
            a, b = kv4.scale_byte(D, 0, t, g), kv4.scale_byte(D, 0, t + 1, g)
            block[:, b:b + 4] = block[:, a:a + 4]
    s = np.abs(rng.standard_normal((n, 1, 64, D // 32))) + 0.1
    s = kv4.f32_to_bf16_value(s.astype(np.float32)).astype(np.float64)
    b = -7.5 * s
    for t in range(0, 64, 2):                                     # b + s u and -b + (-s) u: the same size, the other sign
        s[:, :, t + 1], b[:, :, t + 1] = -s[:, :, t], -b[:, :, t]
    for t in range(0, 64, 2):                                     # the same codes
        for d in range(D):
            (x, hx), (y, hy) = kv4.byte_of(D, 1, t, d), kv4.byte_of(D, 1, t + 1, d)
            nib = (block[:, x] >> (4 * hx)) & 15
            block[:, y] = (block[:, y] & (0x0F if hy else 0xF0)) | (nib << (4 * hy))
    set_values(c, s, b)
    Q = queries(3, 8, D, 35, 0.5)
    within_the_bounds(Q, c, run(Q, c))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("peak,channel", [(0.02, 0.0), (1.0, 0.0), (30.0, 0.0), (300.0, 0.0), (3.0, 200.0), (30.0, 4000.0)])
def test_probabilities_and_scores(D, peak, channel):
    """Values of exactly 1 and -1: the outputs are differences of probabilities.  Queries from tiny to huge, and one channel of keys and queries that outweighs the others."""
    c = make([130, 900], 1, D, seed=36)
    n = c.pages.shape[0]
    rng = np.random.default_rng(37)
    if channel:
        at = kv4.scale_byte(D, 0, 0, 0)
        for t in range(64):                                       # group 0 of every key is some 40 steps away from zero
            at = kv4.scale_byte(D, 0, t, 0)
            pair = c.pages[:, 0, at:at + 4].copy().view(np.uint16)
            pair[:, 1] = kv4.bf16_bits(kv4.f32_to_bf16_value((40 * bf16_to_f64(pair[:, 0])).astype(np.float32)))
            c.pages[:, 0, at:at + 4] = pair.view(np.uint8)
    set_values(c, np.zeros((n, 1, 64, D // 32)), rng.choice([-1.0, 1.0], (n, 1, 64, D // 32)))
    Q = queries(2, 8, D, 38, peak)
    if channel:
        Q[:, :, 5] = kv4.bf16_bits(np.float32(channel))
    within_the_bounds(Q, c, run(Q, c))
