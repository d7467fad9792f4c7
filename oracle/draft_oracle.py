"""CPU float64 definitions of the operators beside the decode step: attention for a tree of drafted tokens,
verification of drafted tokens, accumulated attention weights and eviction.  Test infrastructure only, plain numpy,
written from the formulas; it imports nothing from the CUDA package."""
from __future__ import annotations

import numpy as np

from oracle.slim_oracle import rope_encode, softmax

F64 = np.float64


def tree_chains(parents) -> list:
    """For every token of one sequence the list [root, .., token] of tokens it attends; [] for padding (a parent below
    -1, one that is not an earlier token, or one that is padding)."""
    chains = []
    for i, p in enumerate(parents):
        if p == -1:
            chains.append([i])
        elif 0 <= p < i and chains[p]:
            chains.append(chains[p] + [i])
        else:
            chains.append([])
    return chains


def tree_attention(q, k_tree, K, parents, W_KV, H: int, rope_theta: float = 0.0):
    """One sequence: q, k_tree [n, d], K [L, d] cached rows.  Returns (o [n, d], mass [n, d], arg [n]):
    o the output, mass = (sum_t p_t |k_t|) |W_KV| (what relative errors of the probabilities act on), arg the largest
    sum_j |q_j k_j| / sqrt(d_k) of a token (what relative errors of the products in its arguments act on)."""
    q, k_tree, K = (np.asarray(x, dtype=F64) for x in (q, k_tree, K))
    W_KV = np.asarray(W_KV, dtype=F64)
    n, d = q.shape
    L, d_k = K.shape[0], d // H
    out, mass, arg = np.zeros((n, d)), np.zeros((n, d)), np.zeros(n)
    for i, chain in enumerate(tree_chains(parents)):
        if not chain:
            continue
        rows = np.concatenate([K, k_tree[chain]], axis=0)
        pos = np.concatenate([np.arange(L), L + np.arange(len(chain))])
        for h in range(H):
            cols = slice(h * d_k, (h + 1) * d_k)
            qh = rope_encode(q[i, cols], L + len(chain) - 1, rope_theta)
            kh = rope_encode(rows[:, cols], pos, rope_theta)
            p = softmax(kh @ qh / np.sqrt(d_k))
            out[i, cols] = (p @ rows) @ W_KV[:, cols]
            mass[i, cols] = (p @ np.abs(rows)) @ np.abs(W_KV[:, cols])
            arg[i] = max(arg[i], np.max(np.abs(kh) @ np.abs(qh)) / np.sqrt(d_k))
    return out, mass, arg


def verify(p, q, tokens, parents, r):
    """One sequence: p, q [n, V], tokens, parents, r [n].  Returns (path, next_token)."""
    p, q, r = (np.asarray(x, dtype=F64) for x in (p, q, r))
    n, V = p.shape
    u, W, S, path = 0, p[0].copy(), 1.0, [0]
    for c in range(1, n):
        if parents[c] != u or not 0 <= tokens[c] < V:
            continue
        x = tokens[c]
        if r[c] * S * q[u, x] < W[x]:
            u, W, S = c, p[c].copy(), 1.0
            path.append(c)
        else:
            rest = np.maximum(W - S * q[u], 0.0)
            if not rest.sum() <= 0:         # (a NaN is not nothing)
                W, S = rest, rest.sum()
    cum = np.cumsum(W)
    if not cum[-1] > 0:
        return path, -1
    return path, int(np.argmax(cum > r[0] * cum[-1]))


def weights(q, K, H: int, rope_theta: float = 0.0):
    """Probabilities of every cached row, summed over the heads, for the query at the newest row; and the largest
    sum_j |q_j k_j| / sqrt(d_k)."""
    q, K = np.asarray(q, dtype=F64), np.asarray(K, dtype=F64)
    L, d = K.shape
    d_k = d // H
    total, arg = np.zeros(L), 0.0
    for h in range(H):
        cols = slice(h * d_k, (h + 1) * d_k)
        qh = rope_encode(q[cols], L - 1, rope_theta)
        kh = rope_encode(K[:, cols], np.arange(L), rope_theta)
        total += softmax(kh @ qh / np.sqrt(d_k))
        arg = max(arg, float(np.max(np.abs(kh) @ np.abs(qh)) / np.sqrt(d_k)))
    return total, arg


def evict(acc, length: int, budget: int, recent: int) -> list:
    """The rows of one sequence that stay, in order."""
    if length <= budget:
        return list(range(length))
    old = range(length - recent)
    key = {t: (np.inf if np.isnan(acc[t]) else -float(acc[t]), t) for t in old}
    return sorted(sorted(old, key=lambda t: key[t])[:budget - recent]) + list(range(length - recent, length))
