"""Pins of the drafted-tree oracle (oracle/tree_oracle.py), on the CPU."""
import numpy as np
import pytest

from oracle import tkv_oracle as O
from oracle import tree_oracle as T


def _cache(rng, n, L=2, B=2, Hq=6, Hkv=2, D=64, extra=16, cls=T.TreeOracleCache, **kw):
    c = cls(L, B, Hq, Hkv, D, n + extra, kv_dtype="f32", **kw)
    for l in range(L):
        c.append(l, rng.standard_normal((B, n, Hkv, D)), rng.standard_normal((B, n, Hkv, D)))
    return c


def test_who_sees_whom():
    assert T.ancestors([-1, 0, 0, 1, -1, 4, 3]) == [[0], [0, 1], [0, 2], [0, 1, 3], [4], [4, 5], [0, 1, 3, 6]]
    assert T.ancestors([-1, -2, 1, 0, 4, 9]) == [[0], None, None, [0, 3], None, None]


@pytest.mark.parametrize("scorer", ["attention", "vatp"])
def test_a_line_is_a_chunk(scorer):
    """Nodes in a line, all kept: outputs and scores of a chunk of tokens."""
    rng = np.random.default_rng(1)
    a, b = (_cache(np.random.default_rng(2), 30, scorer=scorer) for _ in range(2))
    n = 5
    parents = np.tile(np.arange(n) - 1, (2, 1))
    for l in range(2):
        k, v, q = (rng.standard_normal((2, n, h, 64)) for h in (2, 2, 6))
        for c in (a, b):
            c.append(l, k, v)
        assert np.allclose(a.attend_tree(l, q, parents), b.attend_and_score_chunk(l, q), rtol=1e-12, atol=1e-12)
    assert a.accept_tree(n, [list(range(n))] * 2) == n
    assert np.allclose(a.score, b.score, rtol=1e-12, atol=1e-15)
    assert a.length == b.length and np.array_equal(a.tier, b.tier) and all(np.array_equal(a.K[l], b.K[l]) for l in range(2))


def test_a_kept_path_is_as_if_its_tokens_had_been_decoded():
    rng = np.random.default_rng(3)
    a, b = (_cache(np.random.default_rng(4), 20, B=1) for _ in range(2))
    parents, path = np.array([[-1, 0, 0, 2, 2, 4]]), [0, 2, 4]
    rows = [[rng.standard_normal((1, 6, h, 64)) for h in (2, 2, 6)] for _ in range(2)]
    for l, (k, v, q) in enumerate(rows):
        a.append(l, k, v)
        o = a.attend_tree(l, q, parents)
        for j in path:
            b.append(l, k[:, j:j + 1], v[:, j:j + 1])
            assert np.allclose(b.attend_and_score(l, q[:, j]), o[:, j], rtol=1e-12, atol=1e-12)
    assert a.accept_tree(6, [path]) == 3
    assert np.allclose(a.score, b.score, rtol=1e-12, atol=1e-15) and np.allclose(a.V[1], b.V[1])


def test_walks_by_hand():
    p = np.array([[.5, .3, .2, 0.], [.1, .1, .1, .7], [.25, .25, .25, .25]])
    # ranked children 0 and 1 of the root: u = .6 >= .5 rejects token 0, leaves total .5; u * .5 < .3 takes token 1; then p[2]
    assert T.walk([-1, 0, 0], [9, 0, 1], p, None, [0, .6, .59], .6) == ([0, 2], 2)
    # ... both rejected: what is left is token 2 alone
    assert T.walk([-1, 0, 0], [9, 0, 1], p, None, [0, .6, .61], .999) == ([0], 2)
    # drawn child: u * q < p takes it
    q = np.array([[.25, .25, .25, .25]] * 3)
    assert T.walk([-1, 0], [9, 1], p[:2], q[:2], [0, .99], .05) == ([0, 1], 0)
    # token 3 has p = 0: rejected; residual max(p - q, 0) = .25, .05, 0, 0
    assert T.walk([-1, 0], [9, 3], p[:2], q[:2], [0, 0.], .82) == ([0], 0)
    assert T.walk([-1, 0], [9, 3], p[:2], q[:2], [0, 0.], .84) == ([0], 1)
    # a node of another branch, a node that is not there, a token outside the vocabulary
    assert T.walk([-1, -1, -2, 5, 0], [9, 0, 0, 0, 7], np.tile(p[:1], (5, 1)), None, [0] * 5, .49) == ([0], 0)


@pytest.mark.parametrize("drawn", [False, True])
def test_the_walks_first_token_is_distributed_as_the_target(drawn):
    """Three children of the root, 40000 walks.  A share x of m walks has standard deviation sqrt(x (1 - x) / m); five of them."""
    rng = np.random.default_rng(5)
    V, m = 5, 40_000
    p = rng.dirichlet(np.ones(V), size=4)
    q = rng.dirichlet(np.ones(V), size=4) if drawn else None
    seen = np.zeros(V)
    for _ in range(m):
        kids = rng.choice(V, 3, p=q[0]) if drawn else rng.permutation(V)[:3]
        path, nxt = T.walk([-1, 0, 0, 0], [0, *kids], p, q, rng.random(4), rng.random())
        seen[nxt if len(path) == 1 else kids[path[1] - 1]] += 1
    assert np.all(np.abs(seen / m - p[0]) <= 5 * np.sqrt(p[0] * (1 - p[0]) / m))


def test_gaps_stay_evicted():
    c = _cache(np.random.default_rng(6), 40, L=1)
    c.append(0, np.ones((2, 4, 2, 64)), np.ones((2, 4, 2, 64)))
    assert c.accept_tree(4, [[0, 2, 3], [1]], scored=False) == 3
    assert c.length[0] == 43 and list(c.tier[1, 40:43]) == [0, 3, 3] and not c.tier[0, :43].any()
    new = c.classify((500_000, 300_000, 150_000, 50_000))
    assert list(new[1, 40:43]) == [0, 3, 3]
    c.migrate()
    assert {41, 42} <= set(c.index_lists(1)[O.T3].tolist())
