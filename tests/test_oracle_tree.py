"""Pins of the oracle for drafted tokens: causal attention, the decode step, and the target's own distribution."""
import numpy as np
import pytest

from oracle import tree as ot
from oracle.attention import causal_attention, decode_attention
from oracle.cache import HeadCache


def chain(T):
    return np.arange(T) - 1


def test_a_chain_over_an_empty_cache_is_causal_attention():
    rng = np.random.default_rng(1)
    q, k, v = (rng.normal(size=(7, 16)) for _ in range(3))
    out, lse = ot.tree_attention(q[None], k, v, chain(7), np.zeros((0, 16)), np.zeros((0, 16)))
    ref, A = causal_attention(q, k, v)
    np.testing.assert_allclose(out[0], ref, atol=1e-12)
    np.testing.assert_allclose(np.exp((q[3] @ k[:4].T) / 4.0 - lse[0, 3]), A[3, :4], atol=1e-12)


def test_branches_do_not_see_each_other():
    rng = np.random.default_rng(2)
    parent = np.array([-1, 0, 0, 1, 2, -1])
    q, k, v, K, V = (rng.normal(size=s) for s in ((2, 6, 8), (6, 8), (6, 8), (5, 8), (5, 8)))
    out, _ = ot.tree_attention(q, k, v, parent, K, V)
    for i, seen in enumerate([[0], [0, 1], [0, 2], [0, 1, 3], [0, 2, 4], [5]]):
        ref, _ = decode_attention(q[:, i], np.concatenate([K, k[seen]]), np.concatenate([V, v[seen]]))
        np.testing.assert_allclose(out[:, i], ref, atol=1e-12)


def test_one_accepted_node_is_a_decode_step():
    rng = np.random.default_rng(3)
    for trial in range(20):
        C, D, g = 32, 8, 3
        caches = []
        n = C - 1 if trial % 2 else int(rng.integers(0, C - 1))
        K, V, pos, sc = rng.normal(size=(n, D)), rng.normal(size=(n, D)), np.arange(n), rng.random(n)
        for _ in range(2):
            hc = HeadCache(C, D, 2, 1, 2)
            hc.load(K, V, pos, sc)
            caches.append(hc)
        for t in range(5):                                    # steps in a row: holes move
            q, k, v = rng.normal(size=(g, D)), rng.normal(size=D), rng.normal(size=D)
            s = caches[1].valid_slots()
            _, lse = ot.tree_attention(q[:, None], k[None], v[None], [-1], caches[1].K[s], caches[1].V[s])
            caches[0].step(q, k, v, 100 + t)
            assert ot.commit(caches[1], q[:, None], k[None], v[None], lse, [0], 100 + t)
            a, b = (c.retained() for c in caches)
            for x, y in zip(a, b):
                np.testing.assert_allclose(x, y, atol=1e-12)


def test_commit_keeps_the_budget_and_what_the_policy_protects():
    rng = np.random.default_rng(4)
    for trial in range(50):
        C, a = 16 * int(rng.integers(1, 4)), int(rng.integers(1, 20))
        hc = HeadCache(C, 4, 4, int(rng.integers(0, 3)), 2)
        n = int(rng.integers(0, C))
        hc.load(rng.normal(size=(n, 4)), rng.normal(size=(n, 4)), np.arange(n), rng.random(n))
        q, k, v = rng.normal(size=(2, a, 4)), rng.normal(size=(a, 4)), rng.normal(size=(a, 4))
        ot.commit(hc, q, k, v, np.zeros((2, a)), list(range(a)), 1000)
        assert hc.length == min(n + a, C - 1) and 0 <= hc.free_slot <= hc.length
        assert set(range(min(4, n))) <= set(hc.pos[hc.valid_slots()].tolist())
        assert len(set(hc.valid_slots().tolist())) == hc.length


def test_a_path_that_does_not_fit_stays_out():
    hc = HeadCache(16, 4, 0, 1, 2)
    hc.load(np.zeros((14, 4)), np.zeros((14, 4)), np.arange(14), np.zeros(14))
    x = np.zeros((1, 3, 4))
    assert not ot.commit(hc, x, x[0], x[0], np.zeros((1, 3)), [0, 1, 2], 50, evict=False)
    assert hc.length == 14
    assert ot.commit(hc, x, x[0], x[0], np.zeros((1, 3)), [0, 1], 50, evict=False)
    assert (hc.length, hc.free_slot) == (16, 16)


@pytest.mark.parametrize("kind", ["one", "independent", "distinct", "points"])
def test_the_first_token_has_the_targets_distribution(kind):
    """Probability of the token behind the root, integrated over the uniform numbers on a grid (midpoints of N cells each;
    the integrand is a step function with a few steps, so the error is a few cells)."""
    p = np.array([0.5, 0.3, 0.15, 0.05])
    d = np.array([0.1, 0.2, 0.3, 0.4])
    N = 40
    mid = (np.arange(N) + 0.5) / N
    pairs = [(x, 1.0) for x in range(4)] if kind == "one" else None
    T = 2 if kind == "one" else 3
    parent = np.array([-1] + [0] * (T - 1))
    got = np.zeros(4)
    if kind == "one":
        draws = [((x,), d[x]) for x, _ in pairs]
    elif kind == "points":
        draws = [((3, 1), 1.0)]                               # children that were chosen, not drawn
    elif kind == "independent":
        draws = [((x, y), d[x] * d[y]) for x in range(4) for y in range(4)]
    else:
        draws = [((x, y), d[x] * d[y] / (1 - d[x])) for x in range(4) for y in range(4) if x != y]
    target = np.tile(p, (T, 1))
    draft = None if kind == "points" else np.tile(d, (T, 1))
    for toks, weight in draws:
        tokens = np.array([0] + list(toks))
        us = [(a,) for a in mid] if T == 2 else [(a, b) for a in mid for b in mid]
        for u in us:
            path, _ = ot.verify(target, draft, tokens, parent, T, np.array([0.0] + list(u)), 0.0, distinct=kind == "distinct")
            w = weight / len(us)
            if len(path) == 2:
                got[tokens[path[1]]] += w
            else:
                for s in mid:
                    got[ot.verify(target, draft, tokens, parent, T, np.array([0.0] + list(u)), s, distinct=kind == "distinct")[1]] += w / N
    np.testing.assert_allclose(got, p, atol=3.0 / N)
    assert abs(got.sum() - 1) < 1e-9


def test_verify_by_hand():
    p = np.array([[0.25, 0.75], [0.5, 0.5]])
    # q(1) = 1: accepted where u < 0.75; then the second row decides
    assert ot.verify(p, None, [0, 1], [-1, 0], 2, [0, 0.7], 0.6) == ([0, 1], 1)
    assert ot.verify(p, None, [0, 1], [-1, 0], 2, [0, 0.75], 0.99) == ([0], 0)
    assert ot.verify(p, None, [0, 1], [-1, 0], 1, [0, 0.0], 0.25) == ([0], 1)
    assert ot.verify(p, None, [0, 1], [-1, 0], 0, [0, 0.0], 0.25) == ([], -1)
    # the draft was the target: always accepted where it can be drawn
    assert ot.verify(p, p, [0, 0], [-1, 0], 2, [0, 0.9999], 0.1)[0] == [0, 1]
    assert ot.verify(np.zeros((1, 2)), None, [0], [-1], 1, [0], 0.5) == ([0], -1)
