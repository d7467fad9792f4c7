"""Pins of the float64 definitions in oracle/draft_oracle.py: hand cases, and identities with the decode oracle."""
import numpy as np

from oracle import draft_oracle as do
from oracle import slim_oracle as so


def test_a_lone_token_is_a_decode_step():
    g = np.random.default_rng(1)
    d, H, L = 24, 3, 7
    K, q, W = g.standard_normal((L + 1, d)), g.standard_normal(d), g.standard_normal((d, d))
    o, _, _ = do.tree_attention(q[None], K[-1:], K[:-1], [-1], W, H, 1.0e4)
    assert np.allclose(o[0], so.oracle_slim(q, K, W, H, 1.0e4), atol=1e-12)


def test_a_chain_is_successive_steps_and_siblings_do_not_see_each_other():
    g = np.random.default_rng(2)
    d, H, L = 16, 2, 5
    K, q, kt, W = g.standard_normal((L, d)), g.standard_normal((4, d)), g.standard_normal((4, d)), g.standard_normal((d, d))
    o, _, _ = do.tree_attention(q, kt, K, [-1, 0, 0, 2], W, H, 1.0e4)      # 0 -> 1, 0 -> 2 -> 3
    for i, chain in ((0, [0]), (1, [0, 1]), (2, [0, 2]), (3, [0, 2, 3])):
        rows = np.concatenate([K, kt[chain]])
        assert np.allclose(o[i], so.oracle_slim(q[i], rows, W, H, 1.0e4), atol=1e-12)


def test_padding_and_broken_parents_give_zero_rows():
    assert do.tree_chains([-1, 0, -2, 2, 5, 9, 1]) == [[0], [0, 1], [], [], [], [], [0, 1, 6]]
    o, _, _ = do.tree_attention(np.ones((2, 4)), np.ones((2, 4)), np.ones((0, 4)), [-2, -1], np.eye(4), 2)
    assert np.all(o[0] == 0) and np.allclose(o[1], 1.0)


def test_verification_by_hand():
    p = np.array([[.5, .25, .25], [0., 0., 1.], [1., 0., 0.]])
    q = np.array([[.25, .5, .25], [1., 0., 0.], [1., 0., 0.]])
    # token 1 at node 1: p/q = 1/2
    assert do.verify(p, q, [0, 1, 0], [-1, 0, -2], [.9, .49, 0.]) == ([0, 1], 2)
    # rejected: the residual is max(p - q, 0) = (1/4, 0, 0): token 0 whatever the draw
    assert do.verify(p, q, [0, 1, 0], [-1, 0, -2], [.9, .51, 0.]) == ([0], 0)
    # a second child of the root, token 0, is tested on the residual: r S q = r / 16 < 1/4 always
    assert do.verify(p, q, [0, 1, 0], [-1, 0, 0], [.9, .51, .99]) == ([0, 2], 0)


def test_verified_tokens_follow_the_target():
    # two children drawn from q, then the accepted one, or the final draw, is the next token: its frequency is p
    g = np.random.default_rng(3)
    V, N = 4, 20000
    p, q = np.array([.1, .2, .3, .4]), np.array([.4, .3, .2, .1])
    hits = np.zeros(V)
    P, Q = np.tile(p, (3, 1)), np.tile(q, (3, 1))
    for _ in range(N):
        tok = [0, g.choice(V, p=q), g.choice(V, p=q)]
        path, nxt = do.verify(P, Q, tok, [-1, 0, 0], g.random(3))
        hits[tok[path[1]] if len(path) > 1 else nxt] += 1
    # five standard deviations of a binomial share
    assert np.all(np.abs(hits / N - p) < 5 * np.sqrt(p * (1 - p) / N))


def test_weights_sum_to_the_heads_and_evict_by_hand():
    g = np.random.default_rng(4)
    w, _ = do.weights(g.standard_normal(12), g.standard_normal((9, 12)), 3, 1.0e4)
    assert np.isclose(w.sum(), 3.0) and np.all(w > 0)
    acc = [5., 1., 5., float("nan"), 5., 0., 9.]
    assert do.evict(acc, 7, 4, 1) == [0, 2, 4, 6]
    assert do.evict(acc, 7, 3, 1) == [0, 2, 6]
    assert do.evict(acc, 7, 6, 0) == [0, 1, 2, 4, 5, 6]
    assert do.evict(acc, 7, 3, 3) == [4, 5, 6]
    assert do.evict(acc, 2, 3, 1) == [0, 1]
