"""Seeded inputs for the tree-drafted decoding calls, and the calls on them.

Everything a call must not use is poisoned: unused pages, page rows past a
prefix, unused nodes' activations (NaN), their parents, tokens and path
entries (far out of range), unused page-table entries (-1)."""
from __future__ import annotations

import math
import random
from types import SimpleNamespace

import torch

from paper_2606_01774_gb300 import flare

FAR = 1 << 30
DTYPES = {"bf16": (torch.bfloat16, flare.FLARE_DT_BF16), "f32": (torch.float32, flare.FLARE_DT_F32)}


def make_tree(rng, n, shape="mixed"):
    """Parents of n nodes: "chain", "star" (all children of the anchor) or "mixed"."""
    if shape == "chain":
        return [i - 1 for i in range(n)]
    if shape == "star":
        return [-1] + [0] * (n - 1) if n else []
    return [-1 if i == 0 else (i - 1 if rng.random() < 0.4 else rng.randrange(max(0, i - 7), i))
            for i in range(n)]


def trees(seed, R, N, nodes=None, shape="mixed", device="cuda"):
    rng = random.Random(seed)
    nodes = [rng.randint(0, N) for _ in range(R)] if nodes is None else nodes
    par = [make_tree(rng, n, shape) + [FAR] * (N - n) for n in nodes]
    return (torch.tensor(par, dtype=torch.int32, device=device).reshape(R, N),
            torch.tensor(nodes, dtype=torch.int32, device=device))


def poison_nodes(x, node_len):
    """NaN in the rows of nodes that are not used."""
    N = x.shape[1]
    off = torch.arange(N, device=x.device) >= node_len[:, None]
    x[off] = float("nan")
    return x


def softmax_inputs(seed, R, N, Hq, Hkv, D, page, prefix, dtype="bf16", nodes=None, shape="mixed",
                   room=0, device="cuda"):
    """prefix: a list of R lengths; room: tokens past each prefix that the table has pages for."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    dt, code = DTYPES[dtype]
    s = SimpleNamespace(R=R, N=N, Hq=Hq, Hkv=Hkv, D=D, page=page, dtype=dtype)
    s.parent, s.node_len = trees(seed, R, N, nodes, shape, device)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=device).to(dt)

    used = [-(-(P + room) // page) for P in prefix]
    pages = sum(used) + 2
    ids = torch.randperm(pages, generator=g, device=device).to(torch.int32)
    s.cols = max([1] + used)
    s.page_table = torch.full((R, s.cols), -1, dtype=torch.int32, device=device)
    s.k_pool, s.v_pool = normal(pages, Hkv, page, D), normal(pages, Hkv, page, D)
    hidden = torch.ones(pages, page, dtype=torch.bool, device=device)
    at = 0
    for r, n in enumerate(used):
        mine = ids[at:at + n]
        s.page_table[r, :n] = mine
        full = torch.arange(n * page, device=device).reshape(n, page) >= prefix[r]
        hidden[mine.long()] = full
        at += n
    for pool in (s.k_pool, s.v_pool):
        pool.permute(0, 2, 1, 3)[hidden] = float("nan")
    s.prefix_len = torch.tensor(prefix, dtype=torch.int32, device=device)
    s.q = poison_nodes(normal(R, N, Hq, D), s.node_len)
    s.k_blk = poison_nodes(normal(R, N, Hkv, D), s.node_len)
    s.v_blk = poison_nodes(normal(R, N, Hkv, D), s.node_len)
    s.desc = flare.softmax_desc(R, N, Hq, Hkv, D, page, pages, s.cols, code, 1.0 / math.sqrt(D))
    return s


def run_softmax(s, expect_bits=0, out=None, lse=None, stream=None):
    need = flare.flare_tree_softmax_workspace_size(s.desc)
    ws = torch.full((max(need, 1),), 0xFF, dtype=torch.uint8, device=s.q.device)
    out = torch.full_like(s.q, 7.0) if out is None else out
    lse = torch.full(s.q.shape[:3], 7.0, device=s.q.device) if lse is None else lse
    st = torch.zeros(1, dtype=torch.int32, device=s.q.device)
    flare.check(flare.flare_tree_softmax_attn(s.desc, s.q, s.k_blk, s.v_blk, s.k_pool, s.v_pool,
                                              s.page_table, s.prefix_len, s.parent, s.node_len,
                                              out, lse, ws, need, st, stream))
    _, bits = flare.flare_read_status(st, stream)
    assert bits == expect_bits, hex(bits)
    return out, lse


def linear_inputs(seed, R, N, Hk, Hv, dk, dv, dtype="bf16", nodes=None, shape="mixed",
                  decay=None, device="cuda"):
    """decay: the log-gate of every token, or None for -softplus(N(0, 1))."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    dt, code = DTYPES[dtype]
    s = SimpleNamespace(R=R, N=N, Hk=Hk, Hv=Hv, dk=dk, dv=dv, dtype=dtype)
    s.parent, s.node_len = trees(seed, R, N, nodes, shape, device)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=device)

    def unit(*shape):
        x = normal(*shape)
        return (x / x.norm(dim=-1, keepdim=True)).to(dt)

    s.q, s.k, s.v = unit(R, N, Hk, dk), unit(R, N, Hk, dk), normal(R, N, Hv, dv).to(dt)
    s.log_decay = -torch.nn.functional.softplus(normal(R, N, Hv))
    if decay is not None:
        s.log_decay.fill_(decay)
    s.beta = torch.sigmoid(normal(R, N, Hv))
    for x in (s.q, s.k, s.v, s.log_decay, s.beta):
        poison_nodes(x, s.node_len)
    slots = 2 * R + 3
    s.state_pool = normal(slots, Hv, dk, dv) * 0.3
    ids = torch.randperm(slots, generator=g, device=device).to(torch.int32)
    s.slot, s.dst_slot = ids[:R].contiguous(), ids[R:2 * R].contiguous()
    s.state_pool[ids[R:].long()] = float("nan")
    s.desc = flare.linear_desc(R, N, Hk, Hv, dk, dv, slots, code, 1.0 / math.sqrt(dk))
    return s


def run_linear(s, expect_bits=0, out=None, stream=None):
    out = torch.full_like(s.v, 7.0) if out is None else out
    st = torch.zeros(1, dtype=torch.int32, device=s.v.device)
    flare.check(flare.flare_tree_linear_attn(s.desc, s.q, s.k, s.v, s.log_decay, s.beta,
                                             s.state_pool, s.slot, s.parent, s.node_len, out, st,
                                             stream))
    _, bits = flare.flare_read_status(st, stream)
    assert bits == expect_bits, hex(bits)
    return out


def random_paths(seed, R, N, lens, device="cuda"):
    rng = random.Random(seed)
    rows = []
    for n in lens:
        p = sorted(rng.sample(range(N), n))
        rows.append(p + [FAR] * (N - n))
    return (torch.tensor(rows, dtype=torch.int32, device=device).reshape(R, N),
            torch.tensor(lens, dtype=torch.int32, device=device))


def verify_inputs(seed, R, N, V, dtype="bf16", drafts="sampled", greedy=False, inv_temp=1.25,
                  nodes=None, shape="mixed", close=0.7, offset=0, device="cuda"):
    """close: how far the drafter's logits are from the target's; offset: elements by which the
    logits start past their allocation (their rows then sit off any alignment)."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    dt, code = DTYPES[dtype]
    s = SimpleNamespace(R=R, N=N, V=V, dtype=dtype, greedy=greedy, inv_temp=inv_temp)
    s.parent, s.node_len = trees(seed, R, N, nodes, shape, device)
    raw = torch.empty(R * N * V + offset, dtype=dt, device=device)
    s.logits = raw[offset:].view(R, N, V)
    s.logits.copy_(3.0 * torch.randn(R, N, V, generator=g, device=device))
    x = (s.logits.float() + close * torch.randn(R, N, V, generator=g, device=device)) * inv_temp
    at = s.parent.long().clamp(min=0, max=N - 1)
    rows = torch.arange(R, device=device)[:, None]
    if drafts == "sampled":
        q = torch.softmax(x, -1)
        e = torch.empty(R, N, V, device=device).exponential_(generator=g).clamp_(min=1e-12)
        s.token = (q[rows, at] / e).argmax(-1).to(torch.int32)
        s.draft_probs = q.contiguous()
    else:
        best = x.topk(min(V, 8), dim=-1).indices
        order = torch.arange(N, device=device).expand(R, N) % best.shape[-1]
        s.token = torch.gather(best[rows, at], 2, order[:, :, None])[..., 0].to(torch.int32)
        s.draft_probs = None
    off = torch.arange(N, device=device) >= s.node_len[:, None]
    s.token[off] = FAR
    s.token[:, 0] = FAR
    s.logits[off] = float("nan")
    if s.draft_probs is not None:
        s.draft_probs[off] = float("nan")
    s.uniform = torch.rand(R, N, generator=g, device=device)
    s.noise = torch.empty(R, V, device=device).exponential_(generator=g).clamp_(min=1e-12)
    mode = flare.FLARE_VERIFY_GREEDY if greedy else flare.FLARE_VERIFY_SAMPLE
    s.desc = flare.tree_verify_desc(R, N, V, code, mode, inv_temp)
    return s


def run_verify(s, expect_bits=0, stream=None):
    need = flare.flare_tree_verify_workspace_size(s.desc)
    dev = s.logits.device
    ws = torch.full((max(need, 1),), 0xFF, dtype=torch.uint8, device=dev)
    got = dict(path=torch.full((s.R, s.N), 99, dtype=torch.int32, device=dev),
               path_len=torch.full((s.R,), 99, dtype=torch.int32, device=dev),
               next_token=torch.full((s.R,), 99, dtype=torch.int32, device=dev),
               node_logp=torch.full((s.R, s.N), 99.0, device=dev))
    st = torch.zeros(1, dtype=torch.int32, device=dev)
    flare.check(flare.flare_tree_verify(s.desc, s.logits, s.draft_probs, s.token, s.parent,
                                        s.node_len, None if s.greedy else s.uniform,
                                        None if s.greedy else s.noise, got["path"],
                                        got["path_len"], got["next_token"], got["node_logp"], ws,
                                        need, st, stream))
    _, bits = flare.flare_read_status(st, stream)
    assert bits == expect_bits, hex(bits)
    return got
