"""CPU oracle for the speculative step (draft trees).  TEST INFRASTRUCTURE ONLY.

Float64 restatements of what the three operators are defined by, in the most literal form:
* a node of a draft tree sees what token-by-token decoding would see after its path: the path is appended to a copy of
  the sequence, one token at a time, and the ordinary decode attention is run there;
* committing a path is appending and encoding its tokens one at a time;
* the verification walks the tree and forms every residual distribution as a whole row.
"""
from __future__ import annotations

import copy

import numpy as np

from .ptenc_oracle import F64, OracleCache


def path_of(parent, i):
    """Ancestors of node i and i itself, root first."""
    line = []
    while i >= 0:
        line.insert(0, int(i))
        i = parent[i]
    return line


def _alone(cache, layer, b):
    """A one-layer, one-sequence cache holding a copy of sequence b."""
    c = OracleCache(n_layers=1, batch=1, n_q_heads=cache.Hq, n_kv_heads=cache.Hkv, head_dim=cache.D, window=cache.W,
                    evict_chunk=cache.E, n_global=1, rank=1, encode_enabled=0)
    c.seqs[0][0] = copy.deepcopy(cache.seqs[layer][b])
    return c


def tree_attn(cache, layer, q, k, v, parent, n_nodes=None, active=None):
    """q [B, T, Hq, D]; k, v [B, T, Hkv, D]; parent [B, T].  Returns out [B, T, Hq, D], lse [B, T, Hq] and done [B, T], which
    rows are defined."""
    q, k, v = (np.asarray(a, F64) for a in (q, k, v))
    B, T = parent.shape
    out = np.zeros((B, T, cache.Hq, cache.D), F64)
    lse = np.zeros((B, T, cache.Hq), F64)
    done = np.zeros((B, T), bool)
    for b in range(B):
        if active is not None and not active[b]:
            continue
        for i in range(T if n_nodes is None else int(n_nodes[b])):
            c = _alone(cache, layer, b)
            for j in path_of(parent[b], i):
                c.append_evict(0, k[b, j][None], v[b, j][None])
            o, s = c.decode_attn(0, q[b, i][None])
            out[b, i], lse[b, i], done[b, i] = o[0], s[0], True
    return out, lse, done


def commit_path(cache, layer, k, v, path, n_path, active=None):
    """Appends and encodes path[b][:n_path[b]] token by token.  Returns tokens evicted per sequence."""
    k, v = np.asarray(k, F64), np.asarray(v, F64)
    B = path.shape[0]
    gone = np.zeros(B, np.int64)
    for b in range(B):
        if active is not None and not active[b]:
            continue
        only = np.arange(B) == b
        for i in path[b, :int(n_path[b])]:
            _, toks, _ = cache.append_evict(layer, k[:, i], v[:, i], only)
            cache.encode(layer)
            gone[b] += len(toks[b])
    return gone


def verify_tree(p, q, tokens, parent, u, n_nodes=None):
    """One sequence: p, q [T, V] (q None: certain drafts), tokens, parent, u [T].  Returns (accepted path, next token, the
    distance of the closest decision from going the other way, as a probability)."""
    p = np.asarray(p, F64)
    n = len(parent) if n_nodes is None else int(n_nodes)
    line, margin = [0], np.inf
    while True:
        at = line[-1]
        r, moved = p[at], False
        for i in (j for j in range(1, n) if parent[j] == at):
            x = int(tokens[i])
            qrow = np.zeros_like(r)
            if q is None:
                qrow[x] = 1.0
            else:
                qrow[:] = q[at]
            margin = min(margin, abs(F64(u[i]) * qrow[x] - r[x]))
            if F64(u[i]) * qrow[x] < r[x]:
                line.append(i)
                moved = True
                break
            left = np.maximum(r - qrow, 0.0)
            r = left / left.sum() if left.sum() > 0 else p[at]
        if not moved:
            break
    if not r.sum() > 0:
        return line, -1, margin
    acc = np.cumsum(r)
    border = F64(u[0]) * acc[-1]
    nxt = int(np.flatnonzero(acc > border)[0])
    return line, nxt, min(margin, np.abs(acc / acc[-1] - F64(u[0])).min())
