"""Plain fp64 definitions of the calls between the matrix products and the attention calls.

TEST INFRASTRUCTURE ONLY, like the rest of this package: numpy, straight from
the definitions, sharing no code with the CUDA path.  Inputs are numpy arrays (or CPU tensors,
bf16 among them).  Where a tolerance depends on what cancels, a function also returns the same
sum with every term's magnitude.
"""
from __future__ import annotations

import math

import numpy as np

from .tree import _f64, _int, paths


# ------------------------------------------------------------------ rotary positions


def rotary_freqs(rotary_dim, base=10000.0, scaling="plain", factor=1.0, original_len=0.0,
                 low_turns=1.0, high_turns=32.0):
    """Radians a position of every pair, in extended precision."""
    L = np.longdouble
    j = np.arange(rotary_dim // 2).astype(L)
    base, factor = L(base), L(factor)
    if scaling == "base":
        base = base * factor ** (L(rotary_dim) / L(rotary_dim - 2))
    f = base ** (-2 * j / L(rotary_dim))
    if scaling == "linear":
        f = f / factor
    if scaling == "by_parts":
        two_pi = 8 * np.arctan(L(1))
        n = L(original_len) * f / two_pi
        g = np.clip((n - L(low_turns)) / (L(high_turns) - L(low_turns)), 0, 1)
        f = g * f + (1 - g) * f / factor
    return f


def angles(table, pos):
    """Radians [len(pos), pairs] of whole positions by a table of 2^64ths of a turn, exactly reduced."""
    out = np.empty((len(pos), len(table)))
    for j, t in enumerate(table):
        for i, p in enumerate(pos):
            x = int(p) * (int(t) % 2 ** 64) % 2 ** 64
            out[i, j] = 2 * math.pi * ((x - 2 ** 64 if x >= 2 ** 63 else x) / 2.0 ** 64)
    return out


def rotate(x, angle, layout="half", inverse=False, amplitude=1.0):
    """x [rows, heads, D] by angle [rows, pairs]; and the magnitudes that enter each element."""
    x = _f64(x).copy()
    size = np.abs(x)
    pairs = angle.shape[1]
    c = amplitude * np.cos(angle)[:, None]
    s = amplitude * np.sin(angle)[:, None] * (-1 if inverse else 1)
    if layout == "half":
        i, j = slice(0, pairs), slice(pairs, 2 * pairs)
    else:
        i, j = slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)
    a, b = x[..., i].copy(), x[..., j].copy()
    x[..., i], x[..., j] = a * c - b * s, b * c + a * s
    size[..., i] = size[..., j] = abs(amplitude) * (np.abs(a) + np.abs(b))
    return x, size


# ------------------------------------------------------------------ logits


def tree_logits(logits, node_len, token=None, parent=None, history=None, output_start=None,
                repetition=None, presence=None, frequency=None, bias=None, mask=None):
    """history: a list of token lists; bias: a list of [(token, value), ...]; mask [R, N, V] bool.

    Returns (out, size): rows past node_len are NaN in `out`."""
    x = _f64(logits)
    R, N, V = x.shape
    out, size = np.full(x.shape, np.nan), np.zeros(x.shape)
    one = lambda a, r, d: d if a is None else float(a[r])  # noqa: E731
    for r in range(R):
        n = N if node_len is None else int(node_len[r])
        text = [] if history is None else list(history[r])
        start = 0 if output_start is None else int(output_start[r])
        lines = paths(parent[r], n) if token is not None else [[] for _ in range(n)]
        rep, pres, freq = one(repetition, r, 1.0), one(presence, r, 0.0), one(frequency, r, 0.0)
        for i in range(n):
            said = text[start:] + [int(token[r][k]) for k in lines[i]]
            count, seen = np.zeros(V), np.zeros(V, bool)
            for t in said:
                count[t] += 1
            seen[text + said] = True
            y = x[r, i].copy()
            with np.errstate(invalid="ignore", over="ignore"):
                y[seen] = np.where(y[seen] > 0, y[seen] / rep, y[seen] * rep)
                s = np.abs(y) + abs(freq) * count + abs(pres) * (count > 0)
                y = y - freq * count - pres * (count > 0)
                for t, b in ([] if bias is None else bias[r]):
                    y[t] += b
                    s[t] += abs(b)
            if mask is not None:
                y[~mask[r, i]] = -np.inf
            out[r, i], size[r, i] = y, s
    return out, size


# ------------------------------------------------------------------ block norms


def _act(kind, z):
    if z is None:
        return 1.0, None
    if kind == "none":
        return z, np.ones_like(z)
    a = 1 / (1 + np.exp(-z))
    return (a, a * (1 - a)) if kind == "sigmoid" else (z * a, a * (1 + z * (1 - a)))


def _stages(x, gate, residual, post_weight, pre_weight, group, shared, post, act, eps, alpha):
    x = _f64(x)
    T, W = x.shape
    G = group or W
    parts = x.reshape(T, W // G, G)
    q = 1 / np.sqrt((parts ** 2).mean(-1, keepdims=True) + eps) if post else np.ones((T, W // G, 1))
    w = np.ones(W) if post_weight is None else _f64(post_weight)
    w = np.tile(w, W // G) if shared and post_weight is not None else w
    n = (parts * q).reshape(T, W) * w
    a, slope = _act(act, None if gate is None else _f64(gate))
    u = alpha * n * a
    y = u if residual is None else _f64(residual) + u
    return parts, q, w, n, a, slope, u, y


def block_norm(x, gate=None, residual=None, post_weight=None, pre_weight=None, group=0,
               shared=False, post=True, pre=True, act="none", eps=1e-6, alpha=1.0):
    """(y, h, sizes of both)."""
    u, y = _stages(x, gate, residual, post_weight, pre_weight, group, shared, post, act, eps,
                   alpha)[-2:]
    size = np.abs(u) + (0 if residual is None else np.abs(_f64(residual)))
    if not pre:
        return y, None, size, None
    r = 1 / np.sqrt((y ** 2).mean(-1, keepdims=True) + eps)
    w = 1.0 if pre_weight is None else _f64(pre_weight)
    return y, y * r * w, size, size * r * np.abs(w)


def block_norm_bwd(x, gate, residual, post_weight, pre_weight, dy, dh, group=0, shared=False,
                   post=True, pre=True, act="none", eps=1e-6, alpha=1.0):
    """Gradients {dx, dgate, dresidual, dpost_weight, dpre_weight} and their sizes."""
    parts, q, w, n, a, slope, u, y = _stages(x, gate, residual, post_weight, pre_weight, group,
                                             shared, post, act, eps, alpha)
    T, W = y.shape
    grad, size = {}, {}
    g = np.zeros((T, W)) if dy is None else _f64(dy)
    gs = np.abs(g)
    ys = np.abs(u) + (0 if residual is None else np.abs(_f64(residual)))
    if pre:
        r = 1 / np.sqrt((y ** 2).mean(-1, keepdims=True) + eps)
        wp = np.ones(W) if pre_weight is None else _f64(pre_weight)
        m = _f64(dh) * wp
        g = g + r * (m - y * r * r * (y * m).mean(-1, keepdims=True))
        gs = gs + r * (np.abs(m) + ys * r * r * (ys * np.abs(m)).mean(-1, keepdims=True))
        grad["dpre_weight"] = (_f64(dh) * y * r).sum(0)
        size["dpre_weight"] = (np.abs(_f64(dh)) * ys * r).sum(0)
    grad["dresidual"], size["dresidual"] = g, gs
    if gate is not None:
        grad["dgate"] = alpha * g * n * slope
        size["dgate"] = abs(alpha) * gs * np.abs(n) * (np.abs(slope) + np.abs(a) + 1)
    dn, dns = alpha * g * a, abs(alpha) * gs * np.abs(a)
    if post:
        xq = (parts * q).reshape(T, W)
        by, bys = (dn * xq).sum(0), (dns * np.abs(xq)).sum(0)
        G = parts.shape[-1]
        grad["dpost_weight"] = by.reshape(-1, G).sum(0) if shared else by
        size["dpost_weight"] = bys.reshape(-1, G).sum(0) if shared else bys
        mp, mps = (dn * w).reshape(parts.shape), (dns * np.abs(w)).reshape(parts.shape)
        dn = (q * (mp - parts * q * q * (parts * mp).mean(-1, keepdims=True))).reshape(T, W)
        dns = (q * (mps + np.abs(parts) * q * q *
                    (np.abs(parts) * mps).mean(-1, keepdims=True))).reshape(T, W)
    grad["dx"], size["dx"] = dn, dns
    return grad, size
