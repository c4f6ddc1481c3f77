"""CPU pins of the tree calls' definitions (oracle/tree.py): a chain is a causal block, a
branch is the chain of its path, and verification returns the target's distribution."""
import numpy as np
import pytest

import oracle
from oracle import tree
from tests.tree_helpers import make_tree


def chain(R, N):
    return np.tile(np.arange(-1, N - 1, dtype=np.int32), (R, 1)), np.full(R, N, np.int32)


def gdr(seed, R=3, N=7, Hk=2, Hv=4, dk=16, dv=24, slots=5):
    g = np.random.default_rng(seed)
    k = g.standard_normal((R, N, Hk, dk))
    k /= np.linalg.norm(k, axis=-1, keepdims=True)
    return (g.standard_normal((R, N, Hk, dk)), k, g.standard_normal((R, N, Hv, dv)),
            -np.log1p(np.exp(g.standard_normal((R, N, Hv)))),
            1 / (1 + np.exp(-g.standard_normal((R, N, Hv)))),
            g.standard_normal((slots, Hv, dk, dv)), g.permutation(slots)[:R].astype(np.int32))


def paged(seed, R=3, N=6, Hq=4, Hkv=2, D=16, page=4, prefix=(0, 5, 12)):
    g = np.random.default_rng(seed)
    cols = 5
    pages = R * cols + 2
    table = g.permutation(pages)[:R * cols].reshape(R, cols).astype(np.int32)
    return (g.standard_normal((R, N, Hq, D)), g.standard_normal((R, N, Hkv, D)),
            g.standard_normal((R, N, Hkv, D)), g.standard_normal((pages, Hkv, page, D)),
            g.standard_normal((pages, Hkv, page, D)), table, np.array(prefix, np.int32))


def branching(seed, R, N):
    import random

    rng = random.Random(seed)
    return np.array([make_tree(rng, N) for _ in range(R)], np.int32), np.full(R, N, np.int32)


def test_a_chain_is_a_causal_block():
    x = gdr(0)
    parent, n = chain(3, 7)
    ref = oracle.gdr_per_token(*x, blockend=False, causal=True)
    assert np.allclose(tree.tree_linear(*x, parent, n), ref["causal"], rtol=1e-12, atol=1e-12)
    y = paged(1)
    parent, n = chain(3, 6)
    out, lse = tree.tree_softmax(*y, parent, n)
    want, wlse = oracle.block_softmax(*y, mask_mode=1)
    assert np.allclose(out, want, rtol=1e-12, atol=1e-12)
    assert np.allclose(lse, wlse, rtol=1e-12, atol=1e-12)


def test_a_whole_path_commits_and_appends_like_a_block():
    q, k, v, g, b, pool, slot = gdr(2)
    accept = np.array([0, 3, 7], np.int32)
    path = np.tile(np.arange(7, dtype=np.int32), (3, 1))
    ref = oracle.gdr_per_token(None, k, v, g, b, pool, slot, accept, blockend=False)["state"]
    got = tree.tree_commit(k, v, g, b, pool, slot, path, accept)
    assert np.allclose(got, ref, rtol=1e-12, atol=1e-12)
    _, kb, vb, kp, vp, table, prefix = paged(3)
    n = np.array([6, 0, 2], np.int32)
    path = np.tile(np.arange(6, dtype=np.int32), (3, 1))
    want = oracle.append_kv(kb, vb, kp, vp, table, prefix, n)
    for blk, pool, ref in ((kb, kp, want[0]), (vb, vp, want[1])):
        assert np.array_equal(tree.tree_append(blk, pool, table, prefix, path, n), ref)


@pytest.mark.parametrize("seed", range(4))
def test_a_branch_is_the_chain_of_its_path(seed):
    """Every node's outputs are the last row of the causal block of its path's tokens."""
    x = gdr(10 + seed)
    parent, n = branching(seed, 3, 7)
    got = tree.tree_linear(*x, parent, n)
    y = paged(20 + seed)
    parent_s, n_s = branching(seed, 3, 6)
    out, lse = tree.tree_softmax(*y, parent_s, n_s)
    for r in range(3):
        for i, line in enumerate(tree.paths(parent[r], 7)):
            part = [a[r:r + 1, line] for a in x[:5]]
            ref = oracle.gdr_per_token(*part, x[5], x[6][r:r + 1], blockend=False, causal=True)
            assert np.allclose(got[r, i], ref["causal"][0, -1], rtol=1e-12, atol=1e-12)
        for i, line in enumerate(tree.paths(parent_s[r], 6)):
            part = [a[r:r + 1, line] for a in y[:3]]
            ref, rl = oracle.block_softmax(*part, y[3], y[4], y[5][r:r + 1], y[6][r:r + 1],
                                           mask_mode=1)
            assert np.allclose(out[r, i], ref[0, -1], rtol=1e-12, atol=1e-12)
            assert np.allclose(lse[r, i], rl[0, -1], rtol=1e-12, atol=1e-12)


def test_the_committed_state_reads_what_the_last_node_read():
    """The state after a path, read by its last node's query, is that node's output."""
    q, k, v, g, b, pool, slot = gdr(4)
    parent, n = branching(4, 3, 7)
    out = tree.tree_linear(q, k, v, g, b, pool, slot, parent, n)
    lines = [tree.paths(parent[r], 7)[-1] for r in range(3)]
    path = np.full((3, 7), -1, np.int32)
    for r, line in enumerate(lines):
        path[r, :len(line)] = line
    S = tree.tree_commit(k, v, g, b, pool, slot, path, np.array([len(x) for x in lines]))
    read = np.einsum("rhkv,rhk->rhv", S, q[:, 6, np.arange(4) // 2]) / 4.0
    assert np.allclose(read, out[:, 6], rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("fixed", [False, True])
def test_verification_returns_the_target_distribution(fixed):
    """Two siblings tried against p = (1/2, 1/3, 1/6): the token after the anchor, summed over a
    grid of random numbers whose cells no decision cuts, has distribution p exactly."""
    p = np.array([1 / 2, 1 / 3, 1 / 6])
    q = np.array([1 / 6, 1 / 6, 2 / 3])
    cells = (np.arange(12) + 0.5) / 12
    tenths = (np.arange(10) + 0.5) / 10  # the second fixed draft is accepted below 2/5
    ratio = cells / (1 - cells)  # of two Exp(1) numbers, at its quantiles
    drafts = [(2, 1)] if fixed else [(a, b) for a in range(3) for b in range(3)]
    rows, weight = [], []
    for a, b in drafts:
        for u in cells:
            for w in tenths:
                for e in ratio:
                    rows.append((a, b, u, w, e))
                    weight.append(1.0 if fixed else q[a] * q[b])
    R = len(rows)
    rows, weight = np.array(rows), np.array(weight) / (12 * 10 * 12)
    token = np.concatenate([np.zeros((R, 1)), rows[:, :2]], 1).astype(np.int32)
    uniform = np.concatenate([np.zeros((R, 1)), rows[:, 2:4]], 1)
    noise = np.ones((R, 3))
    noise[:, 0] = rows[:, 4]
    logits = np.log(np.broadcast_to(p, (R, 3, 3)))
    res = tree.tree_verify(logits, None if fixed else np.broadcast_to(q, (R, 3, 3)), token,
                           np.tile(np.array([-1, 0, 0]), (R, 1)), np.full(R, 3), uniform, noise)
    first = np.where(res["path_len"] > 1,
                     token[np.arange(R), np.maximum(res["path"][:, 1], 0)], res["next_token"])
    got = np.array([weight[first == t].sum() for t in range(3)])
    assert np.allclose(got, p, atol=1e-9)


def test_greedy_walks_the_argmax():
    logits = np.zeros((1, 4, 5))
    logits[0, 0, 3] = logits[0, 2, 1] = logits[0, 3, 4] = 2.0
    token = np.array([[0, 1, 3, 1]])
    res = tree.tree_verify(logits, None, token, np.array([[-1, 0, 0, 2]]), np.array([4]), None,
                           None, greedy=True)
    assert res["path"][0].tolist() == [0, 2, 3, -1] and res["path_len"][0] == 3
    assert res["next_token"][0] == 4
    want = 2 - np.log(np.exp(2) + 4)
    assert np.allclose(res["node_logp"][0], [0, want - 2, want, want])
