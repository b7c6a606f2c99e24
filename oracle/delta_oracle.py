"""CPU oracle for the gated delta rule.

TEST INFRASTRUCTURE ONLY: shares no code with the CUDA library and must not be reached from any
product path.  float64 numpy, token by token, straight from the rule:
    S <- e^g S;  S <- S + k (beta (v - S^T k))^T;  o = scale S^T q
per value head, value head h reading query and key head h // (v_heads // k_heads).
"""
from __future__ import annotations

import numpy as np

EPS = 1e-6


def normalised(x):
    """Rows divided by the root of their sum of squares plus EPS."""
    x = np.asarray(x, np.float64)
    return x / np.sqrt((x * x).sum(-1, keepdims=True) + EPS)


def sequence(q, k, v, g, beta, S, scale):
    """One sequence: q, k [T, k_heads, k_dim], v [T, v_heads, v_dim], g, beta [T, v_heads], S [v_heads, k_dim, v_dim].
    Returns o [T, v_heads, v_dim] and the state behind the last token."""
    q, k, v, g, beta, S = (np.asarray(a, np.float64) for a in (q, k, v, g, beta, S))
    each = v.shape[1] // k.shape[1]
    q, k = np.repeat(q, each, 1), np.repeat(k, each, 1)
    S, o = S.copy(), np.zeros(v.shape)
    for t in range(v.shape[0]):
        S *= np.exp(g[t])[:, None, None]
        seen = np.einsum("hkv,hk->hv", S, k[t])
        S += k[t][:, :, None] * (beta[t][:, None] * (v[t] - seen))[:, None, :]
        o[t] = scale * np.einsum("hkv,hk->hv", S, q[t])
    return o, S


def forward(q, k, v, g, beta, o, state, seq_begin, slot=None, fresh=None, scale=None, normalize=False):
    """Packed sequences; o and state (a pool, or None) as they are behind the call, what the call leaves alone unchanged."""
    o, pool = np.array(o, np.float64), None if state is None else np.array(state, np.float64)
    if normalize:
        q, k = normalised(q), normalised(k)
    scale = 1 / np.sqrt(np.shape(q)[2]) if scale is None else scale
    taken = set()
    for i in range(len(seq_begin) - 1):
        at = slice(seq_begin[i], seq_begin[i + 1])
        s = i if slot is None else int(slot[i])
        if pool is not None:
            out = not 0 <= s < len(pool) or s in taken
            taken.add(s)
            if out:
                continue
        if at.start == at.stop:
            continue
        S = np.zeros((np.shape(v)[1], np.shape(q)[2], np.shape(v)[2])) if pool is None or (fresh is not None and fresh[i]) else pool[s]
        o[at], S = sequence(q[at], k[at], v[at], g[at], beta[at], S, scale)
        if pool is not None:
            pool[s] = S
    return o, pool
