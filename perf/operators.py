"""One round of tree-drafted decoding on the hybrid backbone, measured call by call.

A round takes a tree of drafted tokens per request: node 0 is the anchor (the
token sampled last, not yet in the cache or the recurrent state), and
parent[i] < i for the others.  Five calls serve it:

  tree_softmax       the nodes' queries over the paged prefix and their own
                     ancestors in the tree (softmax layers)
  tree_linear        the gated delta rule along every root path (linear layers)
  tree_verify        which drafts the target accepts, and the next token
  tree_commit_state  the recurrent state after the accepted path
  tree_append_kv     the accepted path's keys and values into the paged cache

Each case has the plain form in elementary torch operations in fp32 and the
library's calls; `exact` restates the definitions in fp64.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
NEG = float("-inf")


# ------------------------------------------------------------------ the cases


def listed():
    return [
        # plain single-token decoding of one long request on the serving shapes
        dict(name="softmax_one_token_16k", op="tree_softmax", requests=1, nodes=1, nodes_lo=1,
             q_heads=16, kv_heads=2, head_dim=256, page=64, prefix_lo=16384, prefix_hi=16384,
             dtype="bf16"),
        # the concurrent serving batch with a 16-node tree per request
        dict(name="softmax_batch64_tree16", op="tree_softmax", requests=64, nodes=16, nodes_lo=16,
             q_heads=16, kv_heads=2, head_dim=256, page=64, prefix_lo=512, prefix_hi=8192,
             dtype="bf16"),
        # many requests of the small model, large ragged trees, small pages
        dict(name="softmax_batch96_tree61_p16", op="tree_softmax", requests=96, nodes=61,
             nodes_lo=23, q_heads=16, kv_heads=4, head_dim=128, page=16, prefix_lo=251,
             prefix_hi=2048, dtype="bf16"),
        # the fp32 layer, empty prefix among them
        dict(name="softmax_f32_tree13", op="tree_softmax", requests=12, nodes=13, nodes_lo=5,
             q_heads=6, kv_heads=2, head_dim=64, page=32, prefix_lo=0, prefix_hi=1021,
             dtype="f32"),
        # linear layers of the serving batch with the same 16-node trees
        dict(name="linear_batch64_tree16", op="tree_linear", requests=64, nodes=16, nodes_lo=16,
             qk_heads=16, v_heads=32, dk=128, dv=128, dtype="bf16"),
        # few requests, large ragged trees
        dict(name="linear_batch6_tree61", op="tree_linear", requests=6, nodes=61, nodes_lo=37,
             qk_heads=16, v_heads=32, dk=128, dv=128, dtype="bf16"),
        # a serving batch sampled against a drafter's distributions
        dict(name="verify_batch64_sampled", op="tree_verify", requests=64, nodes=16, nodes_lo=16,
             vocab=32000, dtype="bf16", drafts="sampled", mode="sample", temperature=0.8),
        # one user, greedy, top-k drafts, an odd vocabulary (rows off the 16-byte grid)
        dict(name="verify_one_greedy_odd", op="tree_verify", requests=1, nodes=9, nodes_lo=9,
             vocab=50257, dtype="bf16", drafts="top", mode="greedy", temperature=1.0),
        # the serving batch's commit after a round of short accepted paths
        dict(name="commit_batch64_path8", op="tree_commit_state", requests=64, nodes=16, path_lo=1,
             path_hi=8, qk_heads=16, v_heads=32, dk=128, dv=128, dtype="bf16"),
        # one request of the fp32 layer, a long accepted chain
        dict(name="commit_one_f32_path33", op="tree_commit_state", requests=1, nodes=40,
             path_lo=33, path_hi=33, qk_heads=2, v_heads=2, dk=64, dv=64, dtype="f32"),
        # all softmax layers' caches of a serving batch after a round
        dict(name="append_batch64_12layers", op="tree_append_kv", requests=64, nodes=16, path_lo=1,
             path_hi=8, layers=12, kv_heads=2, head_dim=256, page=64, prefix_lo=0, prefix_hi=2040,
             dtype="bf16"),
        # one request, one layer
        dict(name="append_one", op="tree_append_kv", requests=1, nodes=7, path_lo=3, path_hi=3,
             layers=1, kv_heads=4, head_dim=128, page=16, prefix_lo=509, prefix_hi=509,
             dtype="bf16"),
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def _drawn(rng, op):
    if op == "tree_softmax":
        c = dict(op=op, requests=_spread(rng, 1, 256), nodes=_spread(rng, 1, 64),
                 head_dim=rng.choice([64, 128, 256]), kv_heads=rng.choice([1, 2, 3, 4, 8]),
                 page=rng.choice([16, 32, 64, 128]), prefix_hi=_spread(rng, 16, 16384),
                 dtype=rng.choice(["bf16"] * 5 + ["f32"]))
        c["q_heads"] = c["kv_heads"] * rng.choice([1, 2, 3, 4, 5, 8])
        c["prefix_lo"] = rng.randint(0, c["prefix_hi"])
    elif op == "tree_linear":
        hk = rng.choice([1, 2, 4, 8, 16])
        d = rng.choice([64, 128, 128, 128])
        c = dict(op=op, requests=_spread(rng, 1, 128), nodes=_spread(rng, 1, 64), qk_heads=hk,
                 v_heads=hk * rng.choice([1, 2]), dk=d, dv=d,
                 dtype=rng.choice(["bf16"] * 5 + ["f32"]))
    elif op == "tree_verify":
        c = dict(op=op, requests=_spread(rng, 1, 128), nodes=_spread(rng, 1, 64),
                 vocab=_spread(rng, 1000, 160000), dtype=rng.choice(["bf16", "bf16", "f32"]),
                 drafts=rng.choice(["sampled", "top"]), mode=rng.choice(["sample", "sample", "greedy"]),
                 temperature=rng.choice([0.6, 0.8, 1.0]))
    elif op == "tree_commit_state":
        hk = rng.choice([1, 2, 4, 8, 16])
        d = rng.choice([64, 128, 128, 128])
        c = dict(op=op, requests=_spread(rng, 1, 128), nodes=_spread(rng, 1, 64), qk_heads=hk,
                 v_heads=hk * rng.choice([1, 2]), dk=d, dv=d,
                 dtype=rng.choice(["bf16"] * 3 + ["f32"]))
    else:
        c = dict(op=op, requests=_spread(rng, 1, 128), nodes=_spread(rng, 1, 64),
                 layers=rng.choice([1, 2, 5, 12]), kv_heads=rng.choice([1, 2, 3, 4, 8]),
                 head_dim=rng.choice([64, 128, 256]), page=rng.choice([16, 32, 64, 128]),
                 prefix_hi=_spread(rng, 16, 2048), dtype=rng.choice(["bf16"] * 3 + ["f32"]))
        c["prefix_lo"] = rng.randint(0, c["prefix_hi"])
    if "path" in op or op in ("tree_commit_state", "tree_append_kv"):
        c["path_hi"] = rng.randint(1, c["nodes"])
        c["path_lo"] = rng.randint(0, c["path_hi"])
    else:
        c["nodes_lo"] = rng.randint(1, c["nodes"])
    return c


def draw(rng):
    """Every call over its own range, the whole of a drawn case at most as large as the call's
    largest listed case (by bytes, by operations and by what its inputs hold)."""
    op = rng.choice(["tree_softmax", "tree_softmax", "tree_softmax", "tree_linear", "tree_linear",
                     "tree_verify", "tree_verify", "tree_commit_state", "tree_append_kv"])
    c = _drawn(rng, op)
    most = [max(f(x) for x in listed() if x["op"] == op) for f in (_bytes, _flops, _held)]
    while c["requests"] > 1 and any(f(c) > m for f, m in zip((_bytes, _flops, _held), most)):
        c["requests"] = c["requests"] * 4 // 5
    while c["nodes"] > 1 and any(f(c) > m for f, m in zip((_bytes, _flops, _held), most)):
        c["nodes"] = c["nodes"] * 4 // 5
        for k in ("nodes_lo", "path_lo", "path_hi"):
            if k in c:
                c[k] = min(c[k], c["nodes"])
    return c


def _bytes(c):
    return work(c)["bytes"]


def _flops(c):
    return work(c)["flops"]


def _held(c):
    """Bytes of the inputs that grow with the batch, used or not."""
    e = DTYPES[c["dtype"]].itemsize
    if c["op"] == "tree_softmax":
        return c["requests"] * c["prefix_hi"] * c["kv_heads"] * c["head_dim"] * 2 * e
    if c["op"] == "tree_verify":
        return c["requests"] * c["nodes"] * c["vocab"] * (e + 4)
    if c["op"] == "tree_append_kv":
        return (c["requests"] * (c["prefix_hi"] + c["nodes"]) * c["kv_heads"] * c["head_dim"] * 2 *
                e * c["layers"])
    return c["requests"] * c["v_heads"] * c["dk"] * c["dv"] * 4


def _lens(lo, hi, n):
    """n whole numbers spread evenly over [lo, hi]."""
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _sizes(c):
    """Per request: its prefix length, node count or path length, and tree, from the case alone
    (another seed deals them to other requests).  The draft trees mix chains with up to four
    siblings, as drafters make them."""
    rng = random.Random("%d/%d" % (c["requests"], c["nodes"]))
    n = c["requests"]
    out = []
    nodes = _lens(c.get("nodes_lo", 1), c["nodes"], n)
    paths = _lens(c.get("path_lo", 1), c.get("path_hi", 1), n)
    prefix = _lens(c.get("prefix_lo", 0), c.get("prefix_hi", 0), n)
    rng.shuffle(nodes)
    rng.shuffle(paths)
    for r in range(n):
        parent, kids = [-1], [0] * c["nodes"]
        for i in range(1, nodes[r]):
            at = i - 1 if rng.random() < 0.4 else rng.randint(max(0, i - 6), i - 1)
            at = at if kids[at] < 4 else i - 1
            kids[at] += 1
            parent.append(at)
        path = [0] + sorted(rng.sample(range(1, c["nodes"]), max(0, paths[r] - 1)))
        out.append(dict(nodes=nodes[r], path=path[:paths[r]], prefix=prefix[r], parent=parent,
                        inner=len(set(parent[1:]))))
    return out


def work(case):
    """What one pass cannot do without: every input that the result depends on read once, every
    output written once; products of the visible pairs only."""
    c, e = case, DTYPES[case["dtype"]].itemsize
    sizes = _sizes(c)
    if c["op"] == "tree_softmax":
        row = c["head_dim"] * e
        b = f = 0
        for s in sizes:
            pairs = s["nodes"] * s["prefix"] + sum(_depths(s["parent"]))
            b += 2 * (s["prefix"] + s["nodes"]) * c["kv_heads"] * row
            b += c["q_heads"] * (s["nodes"] * row + c["nodes"] * (row + 4))
            f += 4 * pairs * c["q_heads"] * c["head_dim"]
        return {"bytes": b, "flops": f}
    if c["op"] == "tree_linear":
        state = c["v_heads"] * c["dk"] * c["dv"]
        b = f = 0
        for s in sizes:
            n, p = s["nodes"], sum(_depths(s["parent"]))
            b += state * 4 + n * (2 * c["qk_heads"] * c["dk"] + c["v_heads"] * c["dv"]) * e
            b += n * c["v_heads"] * 8 + c["nodes"] * c["v_heads"] * c["dv"] * e
            f += n * 4 * state + p * c["v_heads"] * (4 * c["dk"] + 4 * c["dv"])
        return {"bytes": b, "flops": f}
    if c["op"] == "tree_verify":  # rows of nodes without children matter only where a path ends
        rows = sum(max(1, s["inner"]) for s in sizes)
        b = rows * c["vocab"] * e + (c["requests"] * c["vocab"] * 4 if c["mode"] == "sample" else 0)
        return {"bytes": b, "flops": 4 * rows * c["vocab"]}
    if c["op"] == "tree_commit_state":
        state = c["v_heads"] * c["dk"] * c["dv"]
        b = f = 0
        for s in sizes:
            n = len(s["path"])
            b += 2 * state * 4
            b += n * ((c["qk_heads"] * c["dk"] + c["v_heads"] * c["dv"]) * e + c["v_heads"] * 8)
            f += n * 4 * state
        return {"bytes": b, "flops": f}
    n = sum(len(s["path"]) for s in sizes)
    return {"bytes": 4 * n * c["layers"] * c["kv_heads"] * c["head_dim"] * e + 4 * n, "flops": 0}


def _depths(parent):
    d = []
    for at in parent:
        d.append(1 if at < 0 else d[at] + 1)
    return d


# ------------------------------------------------------------------ inputs


def prepare(case, seed):
    c = case
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    sizes = _sizes(c)
    random.Random(seed).shuffle(sizes)
    s = dict(case=c, sizes=sizes)
    R, N, dt = c["requests"], c["nodes"], DTYPES[c["dtype"]]

    def normal(*shape, dtype=dt):
        return torch.randn(shape, generator=g, device=dev).to(dtype)

    def whole(rows):
        return torch.tensor(rows, dtype=torch.int32, device=dev)

    s["node_len"] = whole([x["nodes"] for x in sizes])
    s["parent"] = whole([x["parent"] + [-1] * (N - x["nodes"]) for x in sizes])
    s["path_len"] = whole([len(x["path"]) for x in sizes])
    s["path"] = whole([x["path"] + [-1] * (N - len(x["path"])) for x in sizes])
    s["prefix_len"] = whole([x["prefix"] for x in sizes])
    s["dev_status"] = torch.zeros(1, dtype=torch.int32, device=dev)
    if c["op"] in ("tree_softmax", "tree_append_kv"):
        Hkv, D, page = c["kv_heads"], c["head_dim"], c["page"]
        room = N if c["op"] == "tree_append_kv" else 0
        used = [-(-(x["prefix"] + room) // page) for x in sizes]
        cols, pages = max(1, -(-(c["prefix_hi"] + room) // page)), sum(used) + 3
        ids = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
        table = torch.full((R, cols), -1, dtype=torch.int32, device=dev)
        first = 0
        for r, n in enumerate(used):
            table[r, :n] = ids[first:first + n]
            first += n
        s["page_table"] = table
        layers = c.get("layers", 1)
        s["k_pool"] = [normal(pages, Hkv, page, D) for _ in range(layers)]
        s["v_pool"] = [normal(pages, Hkv, page, D) for _ in range(layers)]
        s["k_blk"] = [normal(R, N, Hkv, D) for _ in range(layers)]
        s["v_blk"] = [normal(R, N, Hkv, D) for _ in range(layers)]
        if c["op"] == "tree_softmax":
            s["q"] = normal(R, N, c["q_heads"], D)
            s["out"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty(R, N, c["q_heads"], device=dev)
    elif c["op"] in ("tree_linear", "tree_commit_state"):
        Hk, Hv, dk, dv = c["qk_heads"], c["v_heads"], c["dk"], c["dv"]

        def unit(*shape):
            x = normal(*shape, dtype=torch.float32)
            return x / x.norm(dim=-1, keepdim=True)

        s["q"], s["k"] = unit(R, N, Hk, dk).to(dt), unit(R, N, Hk, dk).to(dt)
        s["v"] = normal(R, N, Hv, dv)
        s["log_decay"] = -torch.nn.functional.softplus(normal(R, N, Hv, dtype=torch.float32))
        s["beta"] = torch.sigmoid(normal(R, N, Hv, dtype=torch.float32))
        # committed states: the delta rule over a few random tokens; slots in random order, as
        # many again for commits that leave the source as it is
        slots = 2 * R + 1
        S = torch.zeros(slots, Hv, dk, dv, device=dev)
        for _ in range(6):
            k, v = unit(slots, Hv, dk, 1), normal(slots, Hv, 1, dv, dtype=torch.float32)
            b = torch.rand(slots, Hv, 1, 1, generator=g, device=dev)
            S *= 0.5 + 0.5 * torch.rand(slots, Hv, 1, 1, generator=g, device=dev)
            S += k * (b * (v - (k * S).sum(2, keepdim=True)))
        s["state_pool"] = S
        ids = torch.randperm(slots, generator=g, device=dev).to(torch.int32)
        s["slot"], s["dst_slot"] = ids[:R].contiguous(), ids[R:2 * R].contiguous()
        s["out"] = torch.empty_like(s["v"])
    else:
        V = c["vocab"]
        s["logits"] = normal(R, N, V, dtype=torch.float32).mul_(3.0).to(dt)
        x = s["logits"].float().add_(normal(R, N, V, dtype=torch.float32), alpha=0.7)
        x = x.mul_(1.0 / c["temperature"])
        at = s["parent"].long().clamp(min=0)
        if c["drafts"] == "sampled":  # siblings drawn independently from the drafter's distribution
            q = torch.softmax(x, -1)
            tok = torch.empty(R, N, dtype=torch.int32, device=dev)
            for r in range(R):
                e = torch.empty(N, V, device=dev).exponential_(generator=g).clamp_(min=1e-12)
                tok[r] = (q[r][at[r]] / e).argmax(-1)
            s["draft_probs"], s["token"] = q, tok
        else:  # the drafter's most likely tokens, one sibling after the other
            best = x.topk(4, dim=-1).indices
            sib = [[x_["parent"][:i].count(p) for i, p in enumerate(x_["parent"])] +
                   [0] * (N - x_["nodes"]) for x_ in sizes]
            rows = torch.gather(best, 1, at[:, :, None].expand(R, N, 4))
            s["token"] = torch.gather(rows, 2, whole(sib).long()[:, :, None])[:, :, 0].int()
            s["draft_probs"] = None
        del x
        s["uniform"] = torch.rand(R, N, generator=g, device=dev)
        s["noise"] = torch.empty(R, V, device=dev).exponential_(generator=g).clamp_(min=1e-12)
        s["path"] = torch.empty(R, N, dtype=torch.int32, device=dev)
        s["path_len"] = torch.empty(R, dtype=torch.int32, device=dev)
        s["next_token"] = torch.empty(R, dtype=torch.int32, device=dev)
        s["node_logp"] = torch.empty(R, N, device=dev)
    if own:
        s["desc"], s["workspace"] = _handle(s)
    return s


def _handle(s):
    """The descriptor and the workspace that a user's program keeps beside its buffers."""
    from paper_2606_01774_gb300 import flare

    c = s["case"]
    dt = flare.FLARE_DT_BF16 if c["dtype"] == "bf16" else flare.FLARE_DT_F32
    R, N = c["requests"], c["nodes"]
    need = 0
    if c["op"] in ("tree_softmax", "tree_append_kv"):
        desc = flare.softmax_desc(R, N, c.get("q_heads", c["kv_heads"]), c["kv_heads"],
                                  c["head_dim"], c["page"], s["k_pool"][0].shape[0],
                                  s["page_table"].shape[1], dt, 1.0 / math.sqrt(c["head_dim"]))
        if c["op"] == "tree_softmax":
            need = flare.flare_tree_softmax_workspace_size(desc)
    elif c["op"] == "tree_verify":
        mode = flare.FLARE_VERIFY_GREEDY if c["mode"] == "greedy" else flare.FLARE_VERIFY_SAMPLE
        desc = flare.tree_verify_desc(R, N, c["vocab"], dt, mode, 1.0 / c["temperature"])
        need = flare.flare_tree_verify_workspace_size(desc)
    else:
        desc = flare.linear_desc(R, N, c["qk_heads"], c["v_heads"], c["dk"], c["dv"],
                                 s["state_pool"].shape[0], dt, 1.0 / math.sqrt(c["dk"]))
    return desc, torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")


def run(state):
    return (_own if own else _plain)[state["case"]["op"]](state)


# ------------------------------------------------------------------ the library's calls


def _own_softmax(s):
    from paper_2606_01774_gb300 import flare

    flare.check(flare.flare_tree_softmax_attn(
        s["desc"], s["q"], s["k_blk"][0], s["v_blk"][0], s["k_pool"][0], s["v_pool"][0],
        s["page_table"], s["prefix_len"], s["parent"], s["node_len"], s["out"], s["lse"],
        s["workspace"], s["workspace"].numel(), s["dev_status"]))
    return {"out": s["out"], "lse": s["lse"]}


def _own_linear(s):
    from paper_2606_01774_gb300 import flare

    flare.check(flare.flare_tree_linear_attn(
        s["desc"], s["q"], s["k"], s["v"], s["log_decay"], s["beta"], s["state_pool"], s["slot"],
        s["parent"], s["node_len"], s["out"], s["dev_status"]))
    return {"out": s["out"]}


def _own_verify(s):
    from paper_2606_01774_gb300 import flare

    flare.check(flare.flare_tree_verify(
        s["desc"], s["logits"], s["draft_probs"], s["token"], s["parent"], s["node_len"],
        s["uniform"], s["noise"], s["path"], s["path_len"], s["next_token"], s["node_logp"],
        s["workspace"], s["workspace"].numel(), s["dev_status"]))
    return {k: s[k] for k in ("path", "path_len", "next_token", "node_logp")}


def _own_commit(s):
    from paper_2606_01774_gb300 import flare

    flare.check(flare.flare_tree_commit_state(
        s["desc"], s["k"], s["v"], s["log_decay"], s["beta"], s["state_pool"], s["slot"],
        s["dst_slot"], s["path"], s["path_len"], s["dev_status"]))
    return {"state_pool": s["state_pool"]}


def _own_append(s):
    from paper_2606_01774_gb300 import flare

    flare.check(flare.flare_tree_append_kv(
        s["desc"], s["k_blk"], s["v_blk"], s["k_pool"], s["v_pool"], s["page_table"],
        s["prefix_len"], s["path"], s["path_len"], s["dev_status"]))
    return {"k_pool": s["k_pool"], "v_pool": s["v_pool"]}


_own = dict(tree_softmax=_own_softmax, tree_linear=_own_linear, tree_verify=_own_verify,
            tree_commit_state=_own_commit, tree_append_kv=_own_append)


# ------------------------------------------------------------------ the plain forms


def _sees(parent, node_len):
    """[R, N, N]: whether node i sees node j (itself and its ancestors)."""
    R, N = parent.shape
    own_ = torch.eye(N, dtype=torch.bool, device=parent.device)
    sees = torch.zeros(R, N, N, dtype=torch.bool, device=parent.device)
    rows = torch.arange(R, device=parent.device)
    for i in range(N):
        at = parent[:, i].long()
        sees[:, i] = (sees[rows, at.clamp(min=0)] & (at >= 0)[:, None]) | own_[i]
    return sees & (torch.arange(N, device=parent.device) < node_len[:, None])[:, :, None]


def _plain_softmax(s):
    c = s["case"]
    R, N, Hq, Hkv, D = c["requests"], c["nodes"], c["q_heads"], c["kv_heads"], c["head_dim"]
    G = Hq // Hkv
    table = s["page_table"].long().clamp(min=0)
    L = table.shape[1] * c["page"]

    def keys(pool, blk):  # [R, Hkv, L + N, D]
        x = pool[table].permute(0, 2, 1, 3, 4).reshape(R, Hkv, L, D)
        return torch.cat([x, blk.permute(0, 2, 1, 3)], 2).float()

    q = s["q"].float().reshape(R, N, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(R, Hkv, N * G, D)
    x = torch.matmul(q, keys(s["k_pool"][0], s["k_blk"][0]).transpose(2, 3)) / math.sqrt(D)
    live = torch.arange(N, device=q.device) < s["node_len"][:, None]
    past = torch.arange(L, device=q.device) < s["prefix_len"][:, None]
    seen = torch.cat([past[:, None, :] & live[:, :, None], _sees(s["parent"], s["node_len"])], 2)
    seen = seen.repeat_interleave(G, 1)[:, None]
    x = x.masked_fill_(~seen, NEG)
    m = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(m == NEG, torch.zeros_like(m), m))
    total = x.sum(-1, keepdim=True)
    y = torch.matmul(x, keys(s["v_pool"][0], s["v_blk"][0]))
    y = torch.where(total > 0, y / total, torch.zeros_like(y))
    lse = (torch.log(total) + m)[..., 0]
    y = y.reshape(R, Hkv, N, G, D).permute(0, 2, 1, 3, 4).reshape(R, N, Hq, D)
    lse = lse.reshape(R, Hkv, N, G).permute(0, 2, 1, 3).reshape(R, N, Hq)
    return {"out": y.to(s["q"].dtype), "lse": lse}


def _heads(s):
    """q, k per value head and v, as [R, Hv, N, d] in fp32; gates as [R, Hv, N]."""
    rep = s["case"]["v_heads"] // s["case"]["qk_heads"]
    q, k = (s[x].float().repeat_interleave(rep, 2).permute(0, 2, 1, 3) for x in ("q", "k"))
    return (q, k, s["v"].float().permute(0, 2, 1, 3), s["log_decay"].permute(0, 2, 1),
            s["beta"].permute(0, 2, 1))


def _plain_linear(s):
    c = s["case"]
    N = c["nodes"]
    q, k, v, g, b = _heads(s)
    sees = _sees(s["parent"], s["node_len"])[:, None]
    total = torch.matmul(sees.float(), g[..., None])[..., 0]  # the log-decay along the root path
    decay = total[..., :, None] - total[..., None, :]
    decay = torch.where(sees, torch.exp(torch.where(sees, decay, torch.zeros_like(decay))),
                        torch.zeros_like(decay))
    S = s["state_pool"][s["slot"].long()]
    gate = torch.exp(total)[..., None]
    kk = decay * torch.matmul(k, k.transpose(2, 3))
    x = v - gate * torch.matmul(k, S)
    delta = torch.zeros_like(x)
    for i in range(N):
        late = torch.matmul(kk[:, :, i:i + 1, :i], delta[:, :, :i])[:, :, 0]
        delta[:, :, i] = b[:, :, i:i + 1] * (x[:, :, i] - late)
    y = gate * torch.matmul(q, S) + torch.matmul(decay * torch.matmul(q, k.transpose(2, 3)), delta)
    live = (torch.arange(N, device=y.device) < s["node_len"][:, None])[:, None, :, None]
    y = torch.where(live, y, torch.zeros_like(y)) / math.sqrt(c["dk"])
    return {"out": y.permute(0, 2, 1, 3).to(s["v"].dtype).contiguous()}


def _plain_verify(s):
    c = s["case"]
    R, N, V = c["requests"], c["nodes"], c["vocab"]
    dev = s["token"].device
    rows = torch.arange(R, device=dev)
    greedy = c["mode"] == "greedy"
    x = s["logits"].float() / c["temperature"] if not greedy else s["logits"].float()
    m = x.amax(-1, keepdim=True)
    z = torch.exp(x - m)
    total = z.sum(-1, keepdim=True)
    at = s["parent"].long().clamp(min=0)
    tok = s["token"].long()
    live = torch.arange(N, device=dev) < s["node_len"][:, None]
    picked = torch.gather(x[rows[:, None], at], 2, tok[:, :, None])[..., 0]
    stats = (m + torch.log(total))[..., 0]
    logp = picked - stats[rows[:, None], at]
    logp = torch.where(live & (s["parent"] >= 0), logp, torch.zeros_like(logp))
    prob = z.div_(total)
    best = x.argmax(-1)  # the lowest index among equals
    cur = torch.zeros(R, dtype=torch.long, device=dev)
    count = torch.ones(R, dtype=torch.long, device=dev)
    path = torch.full((R, N), -1, dtype=torch.int32, device=dev)
    path[:, 0] = 0
    taken = torch.zeros(R, device=dev)  # how often the siblings' distribution was taken off
    mass = torch.ones(R, device=dev)
    gone = torch.zeros(R, V, dtype=torch.bool, device=dev)
    for i in range(1, N):
        here = live[:, i] & (s["parent"][:, i] == cur)
        t = tok[:, i]
        if greedy:
            ok = here & (t == best[rows, cur])
        else:
            p = prob[rows, cur]
            if s["draft_probs"] is not None:
                d = s["draft_probs"][rows, cur]
                left = (p - taken[:, None] * d).clamp_(min=0)
                ok = here & (s["uniform"][:, i] * d[rows, t] * mass < left[rows, t])
                off = here & ~ok
                taken = torch.where(off, taken + mass, taken)
                rest = (p - taken[:, None] * d).clamp_(min=0).sum(-1)
            else:
                left = torch.where(gone[rows, t], torch.zeros_like(mass), p[rows, t])
                ok = here & (s["uniform"][:, i] * mass < left)
                off = here & ~ok
                gone[rows, t] |= off
                rest = p.masked_fill(gone, 0.0).sum(-1)
            mass = torch.where(off, rest, mass)
            taken = torch.where(ok, torch.zeros_like(taken), taken)
            mass = torch.where(ok, torch.ones_like(mass), mass)
            gone &= ~ok[:, None]
        cur = torch.where(ok, torch.full_like(cur, i), cur)
        path[rows, torch.where(ok, count, torch.zeros_like(count))] = torch.where(
            ok, torch.full_like(cur, i), torch.zeros_like(cur)).int()
        count += ok
    if greedy:
        nxt = best[rows, cur]
    else:
        p = prob[rows, cur]
        if s["draft_probs"] is not None:
            left = (p - taken[:, None] * s["draft_probs"][rows, cur]).clamp_(min=0)
        else:
            left = p.masked_fill(gone, 0.0)
        left = torch.where(left.sum(-1, keepdim=True) > 0, left, p)
        nxt = (left / s["noise"]).argmax(-1)
    return {"path": path, "path_len": count.int(), "next_token": nxt.int(), "node_logp": logp}


def _plain_commit(s):
    c = s["case"]
    q, k, v, g, b = _heads(s)
    S = s["state_pool"][s["slot"].long()]
    rows = torch.arange(c["requests"], device=S.device)
    for t in range(c["path_hi"]):
        at = s["path"][:, t].long().clamp(min=0)
        kt, vt = k[rows, :, at, :, None], v[rows, :, at, None, :]
        alpha, beta = torch.exp(g[rows, :, at])[..., None, None], b[rows, :, at][..., None, None]
        new = alpha * S
        new = new + kt * (beta * (vt - torch.matmul(kt.transpose(2, 3), new)))
        S = torch.where((t < s["path_len"])[:, None, None, None], new, S)
    s["state_pool"][s["dst_slot"].long()] = S
    return {"state_pool": s["state_pool"]}


def _plain_append(s):
    c = s["case"]
    N, page = c["nodes"], c["page"]
    t = torch.arange(N, device=s["path"].device)
    keep = t < s["path_len"][:, None]
    pos = (s["prefix_len"][:, None] + t)[keep].long()
    r = torch.arange(c["requests"], device=t.device)[:, None].expand(-1, N)[keep]
    node = s["path"][keep].long()
    where = s["page_table"][r, pos // page].long()
    for pools, blks in ((s["k_pool"], s["k_blk"]), (s["v_pool"], s["v_blk"])):
        for pool, blk in zip(pools, blks):
            pool[where, :, pos % page] = blk[r, node]
    return {"k_pool": s["k_pool"], "v_pool": s["v_pool"]}


_plain = dict(tree_softmax=_plain_softmax, tree_linear=_plain_linear, tree_verify=_plain_verify,
              tree_commit_state=_plain_commit, tree_append_kv=_plain_append)


# ------------------------------------------------------------------ the definitions in fp64


def exact(case, seed):
    s = prepare(case, seed)
    return dict(tree_softmax=_exact_softmax, tree_linear=_exact_linear, tree_verify=_exact_verify,
                tree_commit_state=_exact_commit, tree_append_kv=_exact_append)[case["op"]](s)


def _roots(parent):
    """Each node's path from the root, itself last."""
    out = []
    for i, at in enumerate(parent):
        out.append((out[at] if at >= 0 else []) + [i])
    return out


def _exact_softmax(s):
    c = s["case"]
    G = c["q_heads"] // c["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    lse = torch.full(s["lse"].shape, NEG, dtype=torch.float64, device=s["q"].device)
    for r, x in enumerate(s["sizes"]):
        P, n = x["prefix"], x["nodes"]
        ids = s["page_table"][r, :-(-P // c["page"])].long()

        def dense(pool):  # [P, Hkv, D]
            return pool[ids].double().transpose(1, 2).reshape(-1, c["kv_heads"], c["head_dim"])[:P]

        kp, vp = dense(s["k_pool"][0]), dense(s["v_pool"][0])
        kb, vb = s["k_blk"][0][r].double(), s["v_blk"][0][r].double()
        qn = s["q"][r, :n].double().reshape(n, c["kv_heads"], G, c["head_dim"])
        scale = c["head_dim"] ** -0.5
        far = torch.einsum("nhgd,phd->nhgp", qn, kp) * scale
        near = torch.einsum("nhgd,mhd->nhgm", qn, kb[:n]) * scale
        hide = torch.ones(n, n, dtype=torch.bool)
        for i, line in enumerate(_roots(x["parent"])):
            hide[i, line] = False
        near = near.masked_fill(hide.to(near.device)[:, None, None, :], NEG)
        total = torch.logsumexp(torch.cat([far, near], -1), -1)
        y = torch.einsum("nhgp,phd->nhgd", torch.exp(far - total[..., None]), vp)
        y = y + torch.einsum("nhgm,mhd->nhgd", torch.exp(near - total[..., None]), vb[:n])
        out[r, :n], lse[r, :n] = y.flatten(1, 2), total.flatten(1, 2)
    return {"out": out, "lse": lse}


def _exact_linear(s):
    """The recurrence itself: every node's state from its parent's."""
    c = s["case"]
    rep = c["v_heads"] // c["qk_heads"]
    out = torch.zeros(s["v"].shape, dtype=torch.float64, device=s["v"].device)
    for r, x in enumerate(s["sizes"]):
        S0 = s["state_pool"][int(s["slot"][r])].double()
        states = []
        q, k = (s[n][r].double().repeat_interleave(rep, 1) for n in ("q", "k"))
        v, g, b = s["v"][r].double(), s["log_decay"][r].double(), s["beta"][r].double()
        for i, at in enumerate(x["parent"]):
            S = (states[at] if at >= 0 else S0) * torch.exp(g[i])[:, None, None]
            u = b[i][:, None] * (v[i] - torch.einsum("hkv,hk->hv", S, k[i]))
            states.append(S + k[i][:, :, None] * u[:, None, :])
            out[r, i] = torch.einsum("hkv,hk->hv", states[i], q[i]) * c["dk"] ** -0.5
    return {"out": out}


def _exact_verify(s):
    c = s["case"]
    path = torch.full(s["path"].shape, -1, dtype=torch.int32)
    counts, nexts = [], []
    logps = torch.zeros(s["node_logp"].shape, dtype=torch.float64)
    temp = 1.0 if c["mode"] == "greedy" else c["temperature"]
    for r, x in enumerate(s["sizes"]):
        logp = torch.log_softmax(s["logits"][r].double() / temp, -1)
        tok, u = s["token"][r].tolist(), s["uniform"][r].double().tolist()
        kids = [[] for _ in range(c["nodes"])]
        for i, at in enumerate(x["parent"]):
            if at >= 0:
                kids[at].append(i)
        ends = torch.tensor([[at, tok[i]] for i, at in enumerate(x["parent"]) if at >= 0] or [[0, 0]])
        ends = ends.to(logp.device)
        got = logp[ends[:, 0], ends[:, 1]].cpu()
        if len(x["parent"]) > 1:
            logps[r, 1:x["nodes"]] = got
        line, done = [0], False
        while not done:
            at = line[-1]
            p = torch.exp(logp[at])
            done = True
            for i in kids[at]:
                if c["mode"] == "greedy":
                    ok = tok[i] == int((s["logits"][r, at] == s["logits"][r, at].max()).nonzero()[0])
                elif s["draft_probs"] is not None:
                    d = s["draft_probs"][r, at].double()
                    ok = u[i] * float(d[tok[i]]) < float(p[tok[i]])
                else:
                    ok = u[i] < float(p[tok[i]])
                if ok:
                    line.append(i)
                    done = False
                    break
                if c["mode"] != "greedy":  # the target without what the draft stands for
                    if s["draft_probs"] is not None:
                        p = (p - d).clamp(min=0)
                    else:
                        p[tok[i]] = 0
                    p = p / p.sum()
        path[r, :len(line)] = torch.tensor(line, dtype=torch.int32)
        counts.append(len(line))
        at = line[-1]
        if c["mode"] == "greedy":
            nexts.append(int((s["logits"][r, at] == s["logits"][r, at].max()).nonzero()[0]))
        else:
            nexts.append(int((p / s["noise"][r].double()).argmax()))
    return {"path": path, "path_len": torch.tensor(counts, dtype=torch.int32),
            "next_token": torch.tensor(nexts, dtype=torch.int32), "node_logp": logps}


def _exact_commit(s):
    """The state as a product of the tokens' linear maps and what they add."""
    c = s["case"]
    rep = c["v_heads"] // c["qk_heads"]
    pool = s["state_pool"].double()
    eye = torch.eye(c["dk"], dtype=torch.float64, device=pool.device)
    for r, x in enumerate(s["sizes"]):
        S = s["state_pool"][int(s["slot"][r])].double()
        for i in x["path"]:
            k = s["k"][r, i].double().repeat_interleave(rep, 0)[:, :, None]
            v, b = s["v"][r, i].double()[:, None, :], s["beta"][r, i].double()[:, None, None]
            step = torch.exp(s["log_decay"][r, i].double())[:, None, None] * (eye - b * k * k.transpose(1, 2))
            S = torch.matmul(step, S) + b * k * v
        pool[int(s["dst_slot"][r])] = S
    return {"state_pool": pool}


def _exact_append(s):
    page = s["case"]["page"]
    for r, x in enumerate(s["sizes"]):
        table = s["page_table"][r].tolist()
        for t, node in enumerate(x["path"]):
            p, row = table[(x["prefix"] + t) // page], (x["prefix"] + t) % page
            for i in range(s["case"]["layers"]):
                s["k_pool"][i][p, :, row] = s["k_blk"][i][r, node]
                s["v_pool"][i][p, :, row] = s["v_blk"][i][r, node]
    return {"k_pool": s["k_pool"], "v_pool": s["v_pool"]}
