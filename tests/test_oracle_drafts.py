"""CPU: the oracle of a drafted step against closed forms, and the host's rotary frequencies against the oracle."""
import math

import numpy as np
import pytest

from oracle import drafts, kv4
from oracle.attention import bf16_to_f64
from paper_2609_24270_b200 import binding as ag

SCALINGS = [dict(), dict(scaling=ag.AG_ROTARY_LINEAR, factor=4.0), dict(scaling=ag.AG_ROTARY_BANDS, factor=8.0, context=8192.0, low=1.0, high=4.0),
            dict(scaling=ag.AG_ROTARY_RAMP, factor=16.0, context=4096.0, low=1.0, high=32.0), dict(scaling=ag.AG_ROTARY_RAMP, factor=2.0, context=10.0, low=1.0, high=32.0)]


@pytest.mark.parametrize("kw", SCALINGS)
@pytest.mark.parametrize("rot,base", [(2, 10000.0), (64, 10000.0), (128, 500000.0), (96, 10.0)])
def test_frequencies(kw, rot, base):
    got, magnitude = ag.rotary_frequencies(rot, base, **kw)
    want, m = drafts.frequencies(rot, base, **kw)
    assert np.allclose(got, want, rtol=1e-13, atol=0) and abs(magnitude - m) < 1e-14
    assert got[0] <= 1.0 + 1e-12 and (got > 0).all() and (np.diff(got) <= 0).all()


def test_frequencies_refused():
    for bad in (dict(rot=3), dict(rot=0), dict(rot=2048), dict(rot=64, base=1.0), dict(rot=64, base=float("nan")), dict(rot=64, scaling=4), dict(rot=64, scaling=-1),
                dict(rot=64, scaling=ag.AG_ROTARY_LINEAR, factor=0.5), dict(rot=64, scaling=ag.AG_ROTARY_LINEAR, factor=float("inf")),
                dict(rot=64, scaling=ag.AG_ROTARY_BANDS, factor=2.0, context=0.0, low=1.0, high=4.0),
                dict(rot=64, scaling=ag.AG_ROTARY_RAMP, factor=2.0, context=4096.0, low=4.0, high=4.0)):
        with pytest.raises(ag.AgError) as e:
            ag.rotary_frequencies(**bad)
        assert e.value.status == ag.AG_ERR_ARG
    assert ag.lib().ag_rotary_frequencies(None, None, None) == ag.AG_ERR_ARG


@pytest.mark.parametrize("pairs", [False, True])
def test_a_rotation_keeps_what_a_rotation_keeps(pairs):
    rng = np.random.default_rng(1)
    x, y, freq = rng.standard_normal((3, 2, 64)), rng.standard_normal((3, 2, 64)), drafts.frequencies(32)[0]
    at = np.array([5, 700, -3])
    rx = drafts.rotate(x, at, freq, pairs=pairs)
    assert (rx[..., 32:] == x[..., 32:]).all() and np.allclose((rx ** 2).sum(-1), (x ** 2).sum(-1))
    # products depend on the distance alone
    one = (rx * drafts.rotate(y, at + 11, freq, pairs=pairs)).sum(-1)
    two = (drafts.rotate(x, at * 0, freq, pairs=pairs) * drafts.rotate(y, at * 0 + 11, freq, pairs=pairs)).sum(-1)
    assert np.allclose(one, two)
    assert np.allclose(drafts.rotate(x, [0, 0, 0], freq, pairs=pairs), x)


def test_who_sees_whom():
    assert (drafts.ancestors(None, 4) == np.tril(np.ones((4, 4), bool))).all()
    sees = drafts.ancestors([-1, 0, 0, 1, 9, 4], 6)
    assert [np.flatnonzero(r).tolist() for r in sees] == [[0], [0, 1], [0, 2], [0, 1, 3], [4], [4, 5]]


def test_a_tree_of_one_path_is_a_causal_prompt():
    from oracle import attention as oa
    rng = np.random.default_rng(2)
    bits = lambda *s: kv4.bf16_bits(kv4.f32_to_bf16_value(rng.standard_normal(s).astype(np.float32)))  # noqa: E731
    Q, K, V = bits(7, 4, 64), bits(7, 2, 64), bits(7, 2, 64)
    past = [(bits(5, 2, 64), bits(5, 2, 64)), (bits(0, 2, 64), bits(0, 2, 64))]
    cache = lambda r, h: tuple(bf16_to_f64(x[:, h]) for x in past[r])  # noqa: E731
    got, _, _ = drafts.tree(Q, K, V, cache, [0, 4, 7], None, 2)
    kk, vv = np.concatenate([past[0][0], K[:4], K[4:]]), np.concatenate([past[0][1], V[:4], V[4:]])
    want, _ = oa.prompt(Q, kk, vv, [0, 4, 7], [0, 9, 12])
    assert np.allclose(got, want)


def test_verification_by_hand():
    P = np.array([[.5, .3, .2], [.1, .2, .7], [.4, .4, .2]])
    Q = np.array([[.2, .6, .2], [.3, .3, .4], [1, 0, 0]])
    v = lambda tok, u, un, **k: drafts.verify(P, k.pop("Q", Q), [0] + tok, k.pop("parent", None), [0, 3], [0] + u, [un], **k)  # noqa: E731
    # 1 is accepted while u .6 < .3, then 2 while u .4 < .7
    a, n, off, rows = v([1, 2], [.49, .99], .5)
    assert a.tolist() == [1, 1, 1] and n[0] == 1 and off.tolist() == [0, 3] and rows.tolist() == [0, 1, 2]
    # rejected at once: max(p - q, 0) = .3 0 0
    a, n, off, rows = v([1, 2], [.51, .0], .999)
    assert a.tolist() == [1, 0, 0] and n[0] == 0 and off.tolist() == [0, 1] and rows.tolist() == [0, -1, -1]
    # two siblings: after 1, r = (1, 0, 0); 0 is accepted then whatever u is
    a, n, _, rows = v([1, 0], [.51, .999], .85, parent=[-1, 0, 0])
    assert a.tolist() == [1, 0, 1] and rows.tolist() == [0, 2, -1] and n[0] == 2
    # not drawn: 1 is accepted while u < .3; after that r = (.5, 0, .2) / .7
    a, n, _, _ = v([1, 2], [.31, .5], .72, Q=None)
    assert a.tolist() == [1, 0, 0] and n[0] == 2


@pytest.mark.parametrize("distinct", [False, True])
def test_verified_text_has_the_targets_distribution(distinct):
    """Over all pairs of drafts and a fine grid of random numbers: the first token behind the root is distributed as p."""
    p, q = np.array([.1, .25, .4, .25]), np.array([.4, .3, .2, .1])
    got, grid = np.zeros(4), (np.arange(25) + .5) / 25
    for x in range(4):
        for y in range(4):
            w = q[x] * ((q[y] / (1 - q[x]) if y != x else 0) if distinct else q[y])
            if w == 0:
                continue
            for u1 in grid:
                for u2 in grid:
                    for un in grid[::6]:
                        a, n, _, rows = drafts.verify(np.stack([p] * 3), np.stack([q] * 3), [0, x, y], [-1, 0, 0], [0, 3], [0, u1, u2], [un], distinct)
                        got[[x, y][rows[1] - 1] if rows[1] > 0 else n[0]] += w / 625 / len(grid[::6])
    assert abs(got.sum() - 1) < 1e-9 and np.abs(got - p).max() < 0.02      # (a grid of 25 steps)


def rounded(x, bits):
    e = np.exp(x - x.max())
    f = (e / e.sum()).astype(np.float32)
    return (kv4.f32_to_bf16_value(f) if bits == 16 else f).astype(np.float64)


@pytest.mark.parametrize("p,q", [
    ([0, 0, 0, 1.0], [.69921875, .302734375, .0009765625, 0]),                        # entries of bf16 that sum to more than 1
    ([0, .6, 0, .4], rounded(np.array([0, -7.9, -8.3, -9.0]), 16)),                   # the largest rounds to 1
    ([0, .6, 0, .4], rounded(np.array([0, -19.0, -19.5, -20.0]), 32)),
    ([0, .6, 0, .4], rounded(np.array([0, -60.0, -61.0, -62.0]), 32)),
    ([0, .5, .5, 0], [1.0, 0, 0, 0]), ([.25, .25, .25, .25], [1.0, 0, 0, 0])])
def test_siblings_of_a_concentrated_q(p, q):
    """What the target gives no weight is never accepted, nor sampled; what is left of q is what the entries that are left add up to."""
    P, Q = np.tile(np.array(p, np.float64), (4, 1)), np.tile(np.array(q, np.float64), (4, 1))
    for u in (.02, .5, .98):
        for un in (0.0, .3, .99):
            a, n, _, _ = drafts.verify(P, Q, [0, 0, 1, 2], [-1, 0, 0, 0], [0, 4], [0, u, u, u], [un], True)
            for i, x in ((1, 0), (2, 1), (3, 2)):
                if a[i]:
                    assert p[x] > 0
                    break
            else:
                assert p[n[0]] > 0
                if sum(q[1:]) > 0 and q[0] >= 1 and p[0] == 0:
                    # 0 is refused, r stays p; 1 is judged by its share of what is left
                    assert u * q[1] * sum(q) / sum(q[1:]) >= p[1]
    # nothing is left behind the only token with weight: its siblings are passed over
    if q[0] == 1 and not any(q[1:]):
        a, n, _, _ = drafts.verify(P, Q, [0, 0, 1, 2], [-1, 0, 0, 0], [0, 4], [0, .999, 0.0, 0.0], [0.0], True)
        assert a.tolist() == [1, 0, 0, 0] and n[0] == 1


@pytest.mark.parametrize("bits,peak,seed", [(16, 6, 3), (16, 6, 4), (16, 6, 5), (16, 6, 12), (32, 20, 0), (32, 20, 4), (32, 12, 3), (32, 20, 9)])
def test_text_of_a_concentrated_q_has_the_targets_distribution(bits, peak, seed):
    """4000 requests of three siblings drawn without repetition from logits far apart: five deviations, and the rows' own sums beside 1 (see the header) once for each sibling."""
    S, V, rng = 4000, 6, np.random.default_rng(seed)
    p, q = rounded(rng.standard_normal(V), bits), rounded(peak * rng.standard_normal(V), bits)
    with np.errstate(divide="ignore"):
        first = np.argsort(-(np.log(q) + rng.gumbel(size=(S, V))), 1)[:, :3]
    token = np.concatenate([np.zeros((S, 1), int), first], 1).reshape(-1)
    a, n, _, _ = drafts.verify(np.broadcast_to(p, (4 * S, V)), np.broadcast_to(q, (4 * S, V)), token, np.tile([-1, 0, 0, 0], S), 4 * np.arange(S + 1), rng.random(4 * S), rng.random(S), True)
    a = a.reshape(S, 4)[:, 1:]
    text = np.where(a.any(1), first[np.arange(S), a.argmax(1)], n)
    seen, mean = np.bincount(text, minlength=V), S * p / p.sum()
    off = abs(p.sum() - q.sum()) / max(p.sum(), q.sum()) + 2 * abs(1 - q.sum())
    assert (np.abs(seen - mean) <= 5 * np.sqrt(mean * (1 - p)) + S * off + 1).all(), (seen, mean)


@pytest.mark.parametrize("siblings,p,q", [(1, [.25, .25, 0], [.9, .1, 0]), (1, [.6, .3, .3], [.2, .3, .5]), (2, [.5, .2, .1], [.3, .4, .1]), (2, [.4, .4, .2], [.7, .2, .3]),
                                          (1, [.2, .3, .1], None), (2, [.5, .5, .2], None), (1, [.5, .5, 0], [.9, .1, 0])])
def test_rows_that_do_not_sum_to_one(siblings, p, q):
    """The text is off by no more than what the header says of the rows' sums, in total variation; five deviations of 3000 requests beside it."""
    S, rng = 3000, np.random.default_rng(5)
    p = np.array(p)
    drawn = np.array([.2, .5, .3] if q is None else q)
    first = rng.choice(3, p=drawn / drawn.sum(), size=(S, siblings))
    n = siblings + 1
    token = np.concatenate([np.zeros((S, 1), int), first], 1).reshape(-1)
    Q = None if q is None else np.broadcast_to(drawn, (n * S, 3))
    a, nxt, _, _ = drafts.verify(np.broadcast_to(p, (n * S, 3)), Q, token, np.tile([-1] + [0] * siblings, S), n * np.arange(S + 1), rng.random(n * S), rng.random(S))
    a = a.reshape(S, n)[:, 1:]
    text = np.where(a.any(1), first[np.arange(S), a.argmax(1)], nxt)
    seen, want = np.bincount(text, minlength=3) / S, p / p.sum()
    sa, sb = p.sum(), drawn.sum()
    bound = abs(1 - sa) if q is None else abs(sa - sb) / max(sa, sb) + (siblings - 1) * abs(1 - sb) / max(1, sb)
    assert np.abs(seen - want).sum() / 2 <= bound + 5 * math.sqrt(.25 * 3 / S)
    if q is not None and siblings == 1 and p.sum() == .5:
        assert np.abs(seen - [.25, .75, 0]).max() < .04                # by hand: .9 * .25 / .9, and all the rest
