"""Plain fp64 definitions of the tree-drafted decoding calls.

TEST INFRASTRUCTURE ONLY, like the rest of this package: numpy loops over
requests and nodes, straight from the definitions, sharing no code with the
CUDA path.  Inputs are numpy arrays (or CPU tensors, bf16 among them).
"""
from __future__ import annotations

import math

import numpy as np


def _f64(x):
    return x.double().numpy() if hasattr(x, "double") else np.asarray(x, np.float64)


def _int(x):
    return x.numpy() if hasattr(x, "numpy") else np.asarray(x)


def paths(parent, n):
    """Each of the first n nodes' path from the anchor, itself last."""
    out = []
    for i in range(n):
        at = int(parent[i])
        out.append((out[at] if at >= 0 else []) + [i])
    return out


def tree_softmax(q, k_blk, v_blk, k_pool, v_pool, page_table, prefix_len, parent, node_len,
                 scale=None, requests=None):
    """(out, lse) of shape [requests, N, Hq, D] and [requests, N, Hq]."""
    q, kb, vb = _f64(q), _f64(k_blk), _f64(v_blk)
    table, prefix, parent, node_len = map(_int, (page_table, prefix_len, parent, node_len))
    R, N, Hq, D = q.shape
    Hkv, page = k_pool.shape[1], k_pool.shape[2]
    G = Hq // Hkv
    s = 1.0 / math.sqrt(D) if scale is None else scale
    req = range(R) if requests is None else requests
    out = np.zeros((len(req), N, Hq, D))
    lse = np.full((len(req), N, Hq), -np.inf)
    for a, r in enumerate(req):
        P, n = int(prefix[r]), int(node_len[r])
        ids = [int(table[r, j]) for j in range(-(-P // page))]
        kp = _f64(k_pool[ids]).transpose(0, 2, 1, 3).reshape(-1, Hkv, D)[:P]
        vp = _f64(v_pool[ids]).transpose(0, 2, 1, 3).reshape(-1, Hkv, D)[:P]
        for i, line in enumerate(paths(parent[r], n)):
            k = np.concatenate([kp, kb[r, line]])
            v = np.concatenate([vp, vb[r, line]])
            for h in range(Hq):
                x = s * (k[:, h // G] @ q[r, i, h])
                m = x.max()
                e = np.exp(x - m)
                out[a, i, h] = (e @ v[:, h // G]) / e.sum()
                lse[a, i, h] = m + math.log(e.sum())
    return out, lse


def _step(S, k, v, g, b):
    """One token of the gated delta rule, all value heads: S [Hv, dk, dv], k [Hv, dk], v [Hv, dv]."""
    S = S * np.exp(g)[:, None, None]
    u = b[:, None] * (v - np.einsum("hkv,hk->hv", S, k))
    return S + k[:, :, None] * u[:, None, :]


def tree_linear(q, k, v, log_decay, beta, state_pool, state_slot, parent, node_len, scale=None,
                requests=None):
    """out [requests, N, Hv, dv]: every node's state from its parent's, read by its own query."""
    q, k, v, g, b, pool = map(_f64, (q, k, v, log_decay, beta, state_pool))
    slot, parent, node_len = map(_int, (state_slot, parent, node_len))
    R, N, Hk, dk = q.shape
    Hv = v.shape[2]
    s = 1.0 / math.sqrt(dk) if scale is None else scale
    heads = np.arange(Hv) // (Hv // Hk)
    req = range(R) if requests is None else requests
    out = np.zeros((len(req), N, Hv, v.shape[3]))
    for a, r in enumerate(req):
        states = []
        for i in range(int(node_len[r])):
            at = int(parent[r, i])
            S = _step(states[at] if at >= 0 else pool[slot[r]], k[r, i, heads], v[r, i], g[r, i],
                      b[r, i])
            states.append(S)
            out[a, i] = s * np.einsum("hkv,hk->hv", S, q[r, i, heads])
    return out


def tree_commit(k, v, log_decay, beta, state_pool, src_slot, path, path_len, requests=None):
    """The state after each accepted path, [requests, Hv, dk, dv]."""
    k, v, g, b, pool = map(_f64, (k, v, log_decay, beta, state_pool))
    src, path, n = map(_int, (src_slot, path, path_len))
    heads = np.arange(v.shape[2]) // (v.shape[2] // k.shape[2])
    req = range(len(n)) if requests is None else requests
    out = []
    for r in req:
        S = pool[src[r]]
        for i in path[r, :int(n[r])]:
            S = _step(S, k[r, i, heads], v[r, i], g[r, i], b[r, i])
        out.append(S)
    return np.stack(out)


def tree_append(blk, pool, page_table, prefix_len, path, path_len):
    """The pool (a copy, of any dtype) with every accepted row in its place."""
    pool = pool.clone() if hasattr(pool, "clone") else np.array(pool)
    page = pool.shape[2]
    table, prefix, path, n = map(_int, (page_table, prefix_len, path, path_len))
    for r in range(len(n)):
        for t in range(int(n[r])):
            pos = int(prefix[r]) + t
            pool[int(table[r, pos // page]), :, pos % page] = blk[r, int(path[r, t])]
    return pool


def tree_verify(logits, draft_probs, token, parent, node_len, uniform, noise, greedy=False,
                inv_temperature=1.0):
    """dict(path, path_len, next_token, node_logp, margin): margin[r] is how far, relatively, the
    request's closest decision was from going the other way."""
    token, parent, node_len = map(_int, (token, parent, node_len))
    R, N = token.shape
    t = 1.0 if greedy else inv_temperature
    path = np.full((R, N), -1, np.int64)
    count = np.zeros(R, np.int64)
    nxt = np.full(R, -1, np.int64)
    logp = np.zeros((R, N))
    margin = np.full(R, np.inf)
    for r in range(R):
        n = int(node_len[r])
        if n == 0:
            continue
        x = _f64(logits[r]) * t
        dist = {}

        def row(i):
            if i not in dist:
                m = x[i].max()
                dist[i] = x[i] - m - math.log(np.exp(x[i] - m).sum())
            return dist[i]

        for i in range(1, n):
            logp[r, i] = row(int(parent[r, i]))[token[r, i]]
        line = [0]
        while True:
            at = line[-1]
            w = np.exp(row(at))
            step = None
            for i in (j for j in range(1, n) if parent[r, j] == at):
                y = int(token[r, i])
                if greedy:
                    ok = y == int(np.argmax(x[at]))
                else:
                    d = _f64(draft_probs[r, at]) if draft_probs is not None else None
                    left = float(_f64(uniform)[r, i]) * (d[y] if d is not None else 1.0) * w.sum()
                    ok = left < w[y]
                    margin[r] = min(margin[r], abs(left - w[y]) / max(left, w[y], 1e-300))
                if ok:
                    step = i
                    break
                if not greedy:
                    if d is not None:
                        w = np.maximum(w / w.sum() - d, 0.0)
                    else:
                        w[y] = 0.0
            if step is None:
                break
            line.append(step)
        if greedy:
            nxt[r] = int(np.argmax(x[line[-1]]))
        else:
            if not w.sum() > 0:
                w = np.exp(row(line[-1]))
            race = w / _f64(noise[r])
            nxt[r] = int(np.argmax(race))
            if race.size > 1:
                two = np.partition(race, -2)[-2:]
                margin[r] = min(margin[r], (two[1] - two[0]) / two[1])
        path[r, :len(line)] = line
        count[r] = len(line)
    return dict(path=path, path_len=count, next_token=nxt, node_logp=logp, margin=margin)
