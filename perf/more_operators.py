"""What stands between the matrix products and the attention, state and verification calls of
the hybrid stack, measured call by call.

  rotary       queries and keys rotated to their positions (and back: the gradient)
  append       the same for tokens that enter the paged cache, their keys and values written there
  logits       penalties for repeated tokens, biases and grammar masks on the target's logits
  norm         the norm, gate and scaled residual after a block and the norm before the next one
  norm_bwd     its gradients

Each case has the plain form in elementary torch operations in fp32 (angles in fp64) and the
library's calls; `exact` restates the definitions in fp64.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
NEG = float("-inf")
BASE = 1e6
EPS = 1e-6


# ------------------------------------------------------------------ the cases


def listed():
    return [
        # plain single-token decoding of one request on the serving heads: latency
        dict(name="rotary_one_token", op="rotary", requests=1, block=1, len_lo=1, len_hi=1,
             q_heads=16, kv_heads=2, head_dim=256, rotary_dim=64, layout="half", scaling="plain",
             inverse=False, tree=False, prefix_lo=16384, prefix_hi=16384, fused=True, dtype="bf16"),
        # training rows of the serving heads, views of the fused projection, long-context scaling
        dict(name="rotary_train_32k", op="rotary", requests=8, block=0, len_lo=4093, len_hi=4096,
             q_heads=16, kv_heads=2, head_dim=256, rotary_dim=256, layout="half",
             scaling="by_parts", inverse=False, tree=False, prefix_lo=0, prefix_hi=0, fused=True,
             dtype="bf16"),
        # the gradient of fp32 rows: odd lengths, pairs side by side, part of the head
        dict(name="rotary_f32_inverse", op="rotary", requests=5, block=0, len_lo=1, len_hi=2039,
             q_heads=6, kv_heads=2, head_dim=128, rotary_dim=96, layout="pairs", scaling="linear",
             inverse=True, tree=False, prefix_lo=0, prefix_hi=0, fused=False, dtype="f32"),
        # one new token of each request of a serving batch, ahead of the attention call
        dict(name="append_batch64_token", op="append", requests=64, block=1, len_lo=1, len_hi=1,
             q_heads=16, kv_heads=2, head_dim=256, rotary_dim=64, layout="half", scaling="plain",
             page=64, prefix_lo=512, prefix_hi=8192, fused=True, dense_k=True, dtype="bf16"),
        # ragged prompts packed one behind the other, small pages
        dict(name="append_prompts_p16", op="append", requests=7, block=0, len_lo=1, len_hi=8191,
             q_heads=16, kv_heads=4, head_dim=128, rotary_dim=128, layout="half", scaling="base",
             page=16, prefix_lo=0, prefix_hi=1021, fused=True, dense_k=False, dtype="bf16"),
        # one user, one token a round, an odd vocabulary (rows off the 16-byte grid)
        dict(name="logits_one_odd", op="logits", requests=1, nodes=1, nodes_lo=1, vocab=50257,
             history=1200, bias=12, masked=0.5, dtype="bf16"),
        # a serving batch of drafted trees under a grammar, long histories
        dict(name="logits_batch64_tree16", op="logits", requests=64, nodes=16, nodes_lo=16,
             vocab=32000, history=8192, bias=64, masked=0.9, dtype="bf16"),
        # fp32 logits of ragged trees, penalties alone
        dict(name="logits_f32_tree13", op="logits", requests=9, nodes=13, nodes_lo=5,
             vocab=50257, history=777, bias=0, masked=0.0, dtype="f32"),
        # the residual stream of a serving batch's single tokens
        dict(name="norm_batch64_token", op="norm", tokens=64, width=2048, group=0, shared=False,
             post=True, pre=True, gate="sigmoid", residual=True, strided=True, dtype="bf16"),
        # the residual stream in training
        dict(name="norm_train_16k", op="norm", tokens=16384, width=4096, group=0, shared=False,
             post=True, pre=True, gate="none", residual=True, strided=False, dtype="bf16"),
        # its gradients
        dict(name="norm_bwd_train_16k", op="norm_bwd", tokens=16384, width=4096, group=0,
             shared=False, post=True, pre=True, gate="none", residual=True, strided=False,
             dtype="bf16"),
        # gradients of a linear layer's output norm (a weight for all heads) and gate, odd rows
        dict(name="norm_bwd_heads_1021", op="norm_bwd", tokens=1021, width=2048, group=128,
             shared=True, post=True, pre=False, gate="silu", residual=False, strided=True,
             dtype="f32"),
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def _drawn(rng, op):
    if op in ("rotary", "append"):
        D = rng.choice([64, 128, 256])
        kv = rng.choice([1, 2, 3, 4, 8])
        c = dict(op=op, requests=_spread(rng, 1, 256), q_heads=kv * rng.choice([1, 2, 3, 4, 5, 8]),
                 kv_heads=kv, head_dim=D, rotary_dim=rng.choice([D // 4, D // 2, D * 3 // 4, D, D]),
                 layout=rng.choice(["half", "half", "pairs"]),
                 scaling=rng.choice(["plain", "linear", "base", "by_parts"]),
                 prefix_hi=_spread(rng, 1, 200000 if op == "rotary" else 8192),
                 fused=rng.random() < 0.6, dtype=rng.choice(["bf16"] * 3 + ["f32"]))
        c["prefix_lo"] = rng.randint(0, c["prefix_hi"])
        kind = rng.choice(["packed", "padded", "token"])
        c["len_hi"] = 1 if kind == "token" else _spread(rng, 1, 8191 if kind == "packed" else 64)
        c["len_lo"] = rng.randint(0 if kind == "packed" else 1, c["len_hi"])
        c["block"] = 0 if kind == "packed" else c["len_hi"]
        if op == "rotary":
            c["inverse"] = rng.random() < 0.4
            c["tree"] = kind == "padded" and rng.random() < 0.5
        else:
            c["page"] = rng.choice([16, 32, 64, 128])
            c["dense_k"] = rng.random() < 0.5
    elif op == "logits":
        c = dict(op=op, requests=_spread(rng, 1, 128), nodes=_spread(rng, 1, 64),
                 vocab=_spread(rng, 1000, 160000), history=rng.choice([0, _spread(rng, 1, 32768)]),
                 bias=rng.choice([0, _spread(rng, 1, 300)]), masked=rng.choice([0.0, 0.5, 0.9, 0.999]),
                 dtype=rng.choice(["bf16", "bf16", "f32"]))
        c["nodes_lo"] = rng.randint(1, c["nodes"])
    else:
        group = rng.choice([0, 0, 64, 128, 256])
        width = group * rng.randint(1, 8192 // group) if group else 8 * _spread(rng, 8, 1024)
        c = dict(op=op, tokens=_spread(rng, 1, 32768), width=width, group=group,
                 shared=bool(group) and rng.random() < 0.7, post=True, pre=rng.random() < 0.7,
                 gate=rng.choice(["none", "silu", "sigmoid"]), residual=rng.random() < 0.7,
                 strided=rng.random() < 0.4, dtype=rng.choice(["bf16"] * 3 + ["f32"]))
        if c["pre"] and rng.random() < 0.25:  # the norm before a block alone
            c.update(post=False, gate="none", group=0, shared=False)
    return c


def draw(rng):
    """Every call over its own range, a drawn case at most as large as the call's largest listed
    case (by bytes and by what its inputs hold)."""
    op = rng.choice(["rotary", "append", "logits", "logits", "norm", "norm_bwd"])
    c = _drawn(rng, op)
    size = "tokens" if op.startswith("norm") else "requests"
    most = [max(f(x) for x in listed() if x["op"] == op) for f in (_bytes, _held)]

    def large():
        return any(f(c) > m for f, m in zip((_bytes, _held), most))

    while c[size] > 1 and large():
        c[size] = c[size] * 4 // 5
    for k in ("nodes", "len_hi"):
        while k in c and c[k] > 1 and large():
            c[k] = c[k] * 4 // 5
            for j in ("nodes_lo", "len_lo", "block"):
                if j in c:
                    c[j] = min(c[j], c[k])
    return c


def _bytes(c):
    return work(c)["bytes"]


def _held(c):
    """Bytes of the inputs that grow with the batch, used or not."""
    e = DTYPES[c["dtype"]].itemsize
    if c["op"] == "append":
        return c["requests"] * (c["prefix_hi"] + c["len_hi"]) * c["kv_heads"] * c["head_dim"] * 2 * e
    if c["op"] == "logits":
        return c["requests"] * c["nodes"] * c["vocab"] * e
    if c["op"] == "rotary":
        return c["requests"] * c["len_hi"] * c["q_heads"] * c["head_dim"] * e
    return c["tokens"] * c["width"] * e


def _lens(lo, hi, n):
    """n whole numbers spread evenly over [lo, hi]."""
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _tree(rng, nodes):
    """Parents of a drafted tree: chains mixed with up to four siblings, as drafters make them."""
    parent, kids = [-1], [0] * nodes
    for i in range(1, nodes):
        at = i - 1 if rng.random() < 0.4 else rng.randint(max(0, i - 6), i - 1)
        at = at if kids[at] < 4 else i - 1
        kids[at] += 1
        parent.append(at)
    return parent


def _sizes(c):
    """Per request: how many tokens or nodes, its prefix and its tree, from the case alone
    (another seed deals them to other requests)."""
    n = c["requests"]
    hi = c.get("len_hi", c.get("nodes"))
    rng = random.Random("%d/%d" % (n, hi))
    lens = _lens(c.get("len_lo", c.get("nodes_lo")), hi, n)
    prefix = _lens(c.get("prefix_lo", 0), c.get("prefix_hi", 0), n)
    history = _lens(c.get("history", 0) // 2, c.get("history", 0), n)
    rng.shuffle(lens)
    return [dict(len=lens[r], prefix=prefix[r], history=history[r],
                 parent=_tree(rng, lens[r]) if c.get("tree") or c["op"] == "logits" else [])
            for r in range(n)]


def work(case):
    """What one pass cannot do without: every input that the result depends on read once, every
    output written once."""
    c, e = case, DTYPES[case["dtype"]].itemsize
    if c["op"] in ("rotary", "append"):
        n = sum(x["len"] for x in _sizes(c))
        rows = n * (c["q_heads"] + c["kv_heads"])
        b = 2 * rows * c["head_dim"] * e + 4 * c["requests"]
        if c["op"] == "append":  # values in and out; the keys' dense copy
            b += (3 if c["dense_k"] else 2) * n * c["kv_heads"] * c["head_dim"] * e
        return {"bytes": b, "flops": 3 * rows * c["rotary_dim"]}
    if c["op"] == "logits":
        rows = sum(x["len"] for x in _sizes(c))
        b = 2 * rows * c["vocab"] * e + (rows * -(-c["vocab"] // 32) * 4 if c["masked"] else 0)
        b += sum(x["history"] for x in _sizes(c)) * 4 + c["requests"] * c["bias"] * 8
        return {"bytes": b, "flops": 0}
    size = c["tokens"] * c["width"]
    gate, res, pre = c["gate"] != "none", c["residual"], c["pre"]
    y = res or not pre  # a norm alone has no other output
    weights = 4 * ((c["group"] if c["shared"] else c["width"]) * c["post"] + c["width"] * pre)
    if c["op"] == "norm":
        return {"bytes": size * e * (1 + gate + res + y + pre) + weights, "flops": 10 * size}
    return {"bytes": size * e * (1 + gate + res + y + pre + 1 + gate + res) + 2 * weights,
            "flops": 25 * size}


# ------------------------------------------------------------------ inputs


def _freqs(c):
    """Radians a position, in fp64."""
    rd = c["rotary_dim"]
    s = dict(factor=4.0, original_len=4096.0, low_turns=1.0, high_turns=32.0)
    base = BASE * s["factor"] ** (rd / (rd - 2)) if c["scaling"] == "base" else BASE
    f = torch.tensor([base ** (-2.0 * j / rd) for j in range(rd // 2)], dtype=torch.float64)
    if c["scaling"] == "linear":
        f = f / s["factor"]
    if c["scaling"] == "by_parts":
        turns = s["original_len"] * f / (2 * math.pi)
        keep = ((turns - s["low_turns"]) / (s["high_turns"] - s["low_turns"])).clamp(0, 1)
        f = keep * f + (1 - keep) * f / s["factor"]
    return f, s


def _amplitude(c):
    return 0.1 * math.log(4.0) + 1.0 if c["scaling"] == "by_parts" else 1.0


def prepare(case, seed):
    c = case
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    s = dict(case=c, dev_status=torch.zeros(1, dtype=torch.int32, device=dev))
    dt = DTYPES[c["dtype"]]

    def normal(*shape, dtype=dt):
        return torch.randn(shape, generator=g, device=dev).to(dtype)

    def whole(rows):
        return torch.tensor(rows, dtype=torch.int32, device=dev)

    def below(n, *shape):
        return torch.randint(0, n, shape, generator=g, device=dev, dtype=torch.int32)

    if c["op"].startswith("norm"):
        T, W = c["tokens"], c["width"]

        def rows(there=True):  # a slice of a fused projection where strided
            if not there:
                return None
            return normal(T, W + 64)[:, 64:] if c["strided"] else normal(T, W)

        s["x"], s["gate"] = rows(), rows(c["gate"] != "none")
        s["residual"] = normal(T, W) if c["residual"] else None
        wide = c["group"] if c["shared"] else W
        s["post_weight"] = 1 + 0.1 * normal(wide, dtype=torch.float32) if c["post"] else None
        s["pre_weight"] = 1 + 0.1 * normal(W, dtype=torch.float32) if c["pre"] else None
        s["has_y"] = c["residual"] or not c["pre"]
        if c["op"] == "norm":
            s["y"] = torch.empty(T, W, dtype=dt, device=dev) if s["has_y"] else None
            s["h"] = torch.empty(T, W, dtype=dt, device=dev) if c["pre"] else None
        else:
            s["dy"] = normal(T, W) if s["has_y"] else None
            s["dh"] = normal(T, W) if c["pre"] else None
            s["dx"] = torch.empty_strided(s["x"].shape, s["x"].stride(), dtype=dt, device=dev)
            s["dgate"] = (None if s["gate"] is None else torch.empty_strided(
                s["gate"].shape, s["gate"].stride(), dtype=dt, device=dev))
            s["dresidual"] = torch.empty(T, W, dtype=dt, device=dev) if c["residual"] else None
            for k in ("post_weight", "pre_weight"):
                s["d" + k] = None if s[k] is None else torch.empty_like(s[k])
    else:
        s["sizes"] = sizes = _sizes(c)
        random.Random(seed).shuffle(sizes)
        R = c["requests"]
        s["token_len"] = whole([x["len"] for x in sizes])
        s["prefix_len"] = whole([x["prefix"] for x in sizes])
    if c["op"] in ("rotary", "append"):
        Hq, Hkv, D = c["q_heads"], c["kv_heads"], c["head_dim"]
        if c["block"]:  # [R, B] rows, some of them unused
            rows, starts = R * c["block"], [r * c["block"] for r in range(R)]
        else:  # one request behind the other, and a few rows behind the last
            starts = [0]
            for x in sizes:
                starts.append(starts[-1] + x["len"])
            rows = starts[-1] + 3
            s["token_start"] = whole(starts)
        s["rows"] = rows
        if c["fused"]:
            qkv = normal(rows, (Hq + 2 * Hkv) * D)
            q, k, v = qkv.split([Hq * D, Hkv * D, Hkv * D], dim=1)
            s["q"], s["k"], s["v"] = (x.unflatten(1, (-1, D)) for x in (q, k, v))
        else:
            s["q"], s["k"], s["v"] = normal(rows, Hq, D), normal(rows, Hkv, D), normal(rows, Hkv, D)
        s["q_out"] = torch.zeros(rows, Hq, D, dtype=dt, device=dev)
        dense_k = c["op"] == "rotary" or c["dense_k"]
        s["k_out"] = torch.zeros(rows, Hkv, D, dtype=dt, device=dev) if dense_k else None
        s["freqs"] = _freqs(c)[0].to(dev)
        s["parent"] = (whole([x["parent"] + [-1] * (c["block"] - x["len"]) for x in sizes])
                       if c.get("tree") else None)
        if c["op"] == "append":
            page = c["page"]
            used = [-(-(x["prefix"] + x["len"]) // page) for x in sizes]
            pages = sum(used) + 3
            ids = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
            table = torch.full((R, max(1, max(used))), -1, dtype=torch.int32, device=dev)
            first = 0
            for r, n in enumerate(used):
                table[r, :n] = ids[first:first + n]
                first += n
            s["page_table"] = table
            s["k_pool"], s["v_pool"] = normal(pages, Hkv, page, D), normal(pages, Hkv, page, D)
    elif c["op"] == "logits":
        N, V, H = c["nodes"], c["vocab"], c["history"]
        s["logits"] = normal(R, N, V, dtype=torch.float32).mul_(3.0).to(dt)
        s["out"] = torch.zeros_like(s["logits"])
        s["parent"] = whole([x["parent"] + [-1] * (N - x["len"]) for x in sizes])
        # text repeats itself: low numbers are common
        common = (torch.rand(R, max(H, 1), generator=g, device=dev) ** 4 * V).to(torch.int32)
        s["history"] = torch.where(torch.rand(R, max(H, 1), generator=g, device=dev) < 0.3,
                                   below(V, R, max(H, 1)), common.clamp(max=V - 1))
        s["history_len"] = whole([x["history"] for x in sizes])
        s["output_start"] = whole([x["history"] * 3 // 4 for x in sizes])
        s["token"] = below(V, R, N)
        if H:
            s["token"][:, ::3] = s["history"][:, :1]
        s["repetition"] = 1 + torch.rand(R, generator=g, device=dev)
        s["presence"] = torch.rand(R, generator=g, device=dev)
        s["frequency"] = 0.2 * torch.rand(R, generator=g, device=dev)
        if c["bias"]:
            s["bias_token"] = below(V, R, c["bias"])
            s["bias_value"] = 2 * normal(R, c["bias"], dtype=torch.float32)
            s["bias_len"] = whole([c["bias"] - r % 2 for r in range(R)])
        if c["masked"]:  # a bit per token, its lowest bit first; some of the rows rule out nearly all
            bits = torch.zeros(R, N, -(-V // 32) * 32, dtype=torch.bool, device=dev)
            bits[:, :, :V] = torch.rand(R, N, V, generator=g, device=dev) >= c["masked"]
            weigh = torch.arange(32, device=dev, dtype=torch.int64)
            words = (bits.unflatten(2, (-1, 32)).long() << weigh).sum(-1)
            s["mask"] = torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32)
    if own:
        _handle(s)
    return s


def _handle(s):
    """The descriptors, the table and the workspace that a user's program keeps beside its buffers."""
    from paper_2606_01774_gb300 import flare

    c = s["case"]
    dt = flare.FLARE_DT_BF16 if c["dtype"] == "bf16" else flare.FLARE_DT_F32
    if c["op"].startswith("norm"):
        act = dict(none=flare.FLARE_ACT_NONE, silu=flare.FLARE_ACT_SILU,
                   sigmoid=flare.FLARE_ACT_SIGMOID)[c["gate"]]
        step = s["x"].stride(0)
        s["desc"] = flare.block_norm_desc(
            c["tokens"], c["width"], dt, group=c["group"], shared_weight=int(c["shared"]),
            post_norm=int(c["post"]), pre_norm=int(c["pre"]), gate_act=act, eps=EPS,
            residual_scale=0.5, x_stride=step, gate_stride=step)
        if c["op"] == "norm_bwd":
            need = flare.flare_block_norm_bwd_workspace_size(s["desc"])
            s["workspace"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    elif c["op"] == "logits":
        s["desc"] = flare.tree_logits_desc(c["requests"], c["nodes"], c["vocab"], dt,
                                           max_history=s["history"].shape[1], max_bias=c["bias"])
    else:
        rd, (_, how) = c["rotary_dim"], _freqs(c)
        kind = dict(plain=flare.FLARE_ROTARY_PLAIN, linear=flare.FLARE_ROTARY_LINEAR,
                    base=flare.FLARE_ROTARY_BASE, by_parts=flare.FLARE_ROTARY_BY_PARTS)
        s["table"] = torch.empty(rd // 2, dtype=torch.int64, device="cuda")
        flare.check(flare.flare_rotary_table(
            flare.rotary_freq_desc(rd, BASE, kind[c["scaling"]], **how), s["table"]))
        pool = {}
        if c["op"] == "append":
            pool = dict(page_size=c["page"], num_pages=s["k_pool"].shape[0],
                        max_pages_per_req=s["page_table"].shape[1])
        s["desc"] = flare.rotary_desc(
            c["requests"], c["block"], s["rows"], c["q_heads"], c["kv_heads"], c["head_dim"], rd, dt,
            layout=(flare.FLARE_ROTARY_HALF if c["layout"] == "half"
                    else flare.FLARE_ROTARY_INTERLEAVED),
            inverse=int(c.get("inverse", False)), amplitude=_amplitude(c),
            q_stride=s["q"].stride(0), k_stride=s["k"].stride(0), v_stride=s["v"].stride(0), **pool)


def run(state):
    return (_own if own else _plain)[state["case"]["op"]](state)


# ------------------------------------------------------------------ the library's calls


def _own_rotary(s):
    from paper_2606_01774_gb300 import flare

    packed = "token_start" in s
    flare.check(flare.flare_rotary(
        s["desc"], s["q"], s["k"], s["table"], None, s["prefix_len"],
        None if packed else s["token_len"], s["parent"], s.get("token_start"), s["q_out"],
        s["k_out"], s["dev_status"]))
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_append(s):
    from paper_2606_01774_gb300 import flare

    packed = "token_start" in s
    flare.check(flare.flare_rotary_append_kv(
        s["desc"], s["q"], s["k"], s["v"], s["table"], None, s["prefix_len"],
        None if packed else s["token_len"], s.get("token_start"), s["page_table"], s["q_out"],
        s["k_out"], s["k_pool"], s["v_pool"], s["dev_status"]))
    return {"q": s["q_out"], "k": s["k_out"], "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _own_logits(s):
    from paper_2606_01774_gb300 import flare

    flare.check(flare.flare_tree_logits(
        s["desc"], s["logits"], s["history"], s["history_len"], s["output_start"], s["token"],
        s["parent"], s["token_len"], s["repetition"], s["presence"], s["frequency"],
        s.get("bias_token"), s.get("bias_value"), s.get("bias_len"), s.get("mask"), s["out"],
        s["dev_status"]))
    return {"out": s["out"]}


def _own_norm(s):
    from paper_2606_01774_gb300 import flare

    flare.check(flare.flare_block_norm(
        s["desc"], s["x"], s["gate"], s["residual"], s["post_weight"], s["pre_weight"], s["y"],
        s["h"]))
    return {"y": s["y"], "h": s["h"]}


GRADS = ("dx", "dgate", "dresidual", "dpost_weight", "dpre_weight")


def _own_norm_bwd(s):
    from paper_2606_01774_gb300 import flare

    flare.check(flare.flare_block_norm_bwd(
        s["desc"], s["x"], s["gate"], s["residual"], s["post_weight"], s["pre_weight"], s["dy"],
        s["dh"], *(s[k] for k in GRADS), s["workspace"], s["workspace"].numel()))
    return {k: s[k] for k in GRADS}


_own = dict(rotary=_own_rotary, append=_own_append, logits=_own_logits, norm=_own_norm,
            norm_bwd=_own_norm_bwd)


# ------------------------------------------------------------------ the plain forms


def _sees(parent, node_len):
    """[R, N, N]: whether node j is node i or one of its ancestors, by doubling the reach."""
    N = parent.shape[1]
    here = torch.arange(N, device=parent.device)
    reach = ((parent[:, :, None] == here) | (here[:, None] == here)).float()
    for _ in range(6):  # 64 nodes
        reach = (torch.matmul(reach, reach) > 0).float()
    return (reach > 0) & (here < node_len[:, None])[:, :, None]


def _rows(s):
    """Which rows are tokens, their requests, and their places in them."""
    c = s["case"]
    row = torch.arange(s["rows"], device=s["q"].device)
    if c["block"]:
        r, t = row // c["block"], row % c["block"]
        return t < s["token_len"][r], r, t
    start = s["token_start"].long()
    r = (torch.searchsorted(start, row, right=True) - 1).clamp(max=c["requests"] - 1)
    return row < start[-1], r, row - start[r]


def _turned(s, x, pos):
    """x [rows, heads, D] at positions `pos`, in fp32."""
    c = s["case"]
    rd = c["rotary_dim"]
    angle = pos.double()[:, None, None] * s["freqs"]
    cos, sin = (torch.cos(angle) * _amplitude(c)).float(), (torch.sin(angle) * _amplitude(c)).float()
    sin = -sin if c.get("inverse") else sin
    x = x.float()
    if c["layout"] == "half":
        a, b = x[..., :rd // 2], x[..., rd // 2:rd]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:rd:2], x[..., 1:rd:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([y, x[..., rd:]], -1)


def _plain_rotary(s):
    live, r, t = _rows(s)
    if s["parent"] is not None:
        t = (_sees(s["parent"], s["token_len"]).sum(-1) - 1).reshape(-1)
    pos = s["prefix_len"][r] + t
    out = {}
    for k in ("q", "k"):
        y = _turned(s, s[k], pos).to(s[k].dtype)
        out[k] = torch.where(live[:, None, None], y, s[k + "_out"])
    return out


def _plain_append(s):
    page = s["case"]["page"]
    live, r, t = _rows(s)
    pos = s["prefix_len"][r] + t
    q = torch.where(live[:, None, None], _turned(s, s["q"], pos).to(s["q"].dtype), s["q_out"])
    k = _turned(s, s["k"], pos).to(s["k"].dtype)
    at = torch.where(live, pos, torch.zeros_like(pos)).long()
    where = s["page_table"][r, at // page].long()[live]
    s["k_pool"][where, :, at[live] % page] = k[live]
    s["v_pool"][where, :, at[live] % page] = s["v"][live]
    k = None if s["k_out"] is None else torch.where(live[:, None, None], k, s["k_out"])
    return {"q": q, "k": k, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _plain_logits(s):
    c = s["case"]
    R, N, V = c["requests"], c["nodes"], c["vocab"]
    dev = s["logits"].device
    at = torch.arange(s["history"].shape[1], device=dev)
    there = at < s["history_len"][:, None]
    said = there & (at >= s["output_start"][:, None])
    tok = s["history"].long()
    zero = torch.zeros(R, V, dtype=torch.int32, device=dev)
    total = zero.scatter_add(1, tok, there.int())
    said = zero.scatter_add(1, tok, said.int())
    path = _sees(s["parent"], s["token_len"]).int()
    here = torch.zeros(R, N, V, dtype=torch.int32, device=dev)
    here.scatter_add_(2, s["token"].long()[:, None, :].expand(R, N, N), path)
    count = said[:, None] + here
    seen = (total[:, None] + here) > 0
    x = s["logits"].float()
    rep, pres, freq = (s[k][:, None, None] for k in ("repetition", "presence", "frequency"))
    x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    x = x - freq * count - pres * (count > 0)
    if c["bias"]:
        use = torch.arange(c["bias"], device=dev) < s["bias_len"][:, None]
        bias = torch.zeros(R, V, device=dev).scatter_add(
            1, s["bias_token"].long(), torch.where(use, s["bias_value"], 0.0))
        x = x + bias[:, None]
    if c["masked"]:
        t = torch.arange(V, device=dev)
        x = torch.where((s["mask"][:, :, t // 32] >> (t % 32)) & 1 > 0, x, NEG)
    live = torch.arange(N, device=dev) < s["token_len"][:, None]
    return {"out": torch.where(live[:, :, None], x.to(s["logits"].dtype), s["out"])}


def _act(kind, z):
    """A gate's activation and its derivative."""
    if kind == "none":
        return torch.ones_like(z), torch.zeros_like(z)
    a = 1 / (1 + torch.exp(-z))
    return (a, a * (1 - a)) if kind == "sigmoid" else (z * a, a * (1 + z * (1 - a)))


def _stages(s):
    """The block's norm by groups, its gate, and the new residual stream, in fp32."""
    c = s["case"]
    G = c["group"] or c["width"]
    x = s["x"].float().unflatten(1, (-1, G))
    if c["post"]:
        rs = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        w = s["post_weight"].view(1, -1, G)
    else:
        rs, w = torch.ones_like(x[..., :1]), torch.ones_like(x[:1])
    n = x * rs * w
    z = s["x"].float() if s["gate"] is None else s["gate"].float()
    a, da = _act(c["gate"], z)
    y = 0.5 * n.flatten(1) * a
    return x, rs, w, n, a, da, y if s["residual"] is None else y + s["residual"].float()


def _plain_norm(s):
    y = _stages(s)[-1]
    dt, out = s["x"].dtype, {}
    out["y"] = y.to(dt) if s["has_y"] else None
    r = torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS)
    out["h"] = (y * r * s["pre_weight"]).to(dt) if s["case"]["pre"] else None
    return out


def _plain_norm_bwd(s):
    c, dt = s["case"], s["x"].dtype
    x, rs, w, n, a, da, y = _stages(s)
    g = torch.zeros_like(y) if s["dy"] is None else s["dy"].float()
    out = dict.fromkeys(GRADS)
    if c["pre"]:
        r = torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS)
        dh = s["dh"].float()
        m = dh * s["pre_weight"]
        g = g + r * (m - y * r * r * (y * m).mean(-1, keepdim=True))
        out["dpre_weight"] = (dh * y * r).sum(0)
    if c["residual"]:
        out["dresidual"] = g.to(dt)
    du = 0.5 * g
    if c["gate"] != "none":
        out["dgate"] = (du * n.flatten(1) * da).to(dt)
    dn = (du * a).view_as(x)
    if c["post"]:
        by = (dn * x * rs).sum(0)
        out["dpost_weight"] = by.sum(0) if c["shared"] else by.flatten()
        m = dn * w
        dn = rs * (m - x * rs * rs * (x * m).mean(-1, keepdim=True))
    out["dx"] = dn.flatten(1).to(dt)
    return out


_plain = dict(rotary=_plain_rotary, append=_plain_append, logits=_plain_logits, norm=_plain_norm,
              norm_bwd=_plain_norm_bwd)


# ------------------------------------------------------------------ the definitions in fp64


def exact(case, seed):
    s = prepare(case, seed)
    return dict(rotary=_exact_rotary, append=_exact_append, logits=_exact_logits,
                norm=_exact_norm, norm_bwd=_exact_norm_bwd)[case["op"]](s)


def _depths(parent):
    d = []
    for at in parent:
        d.append(0 if at < 0 else d[at] + 1)
    return d


def _spans(s):
    """Per request: its first row and its tokens' positions."""
    c, first = s["case"], 0
    for r, x in enumerate(s["sizes"]):
        first = r * c["block"] if c["block"] else first
        steps = _depths(x["parent"]) if c.get("tree") else range(x["len"])
        yield r, first, x["len"], torch.tensor([x["prefix"] + t for t in steps], dtype=torch.int64)
        first += x["len"]


def _exact_turned(s, x, pos):
    """As a product of complex numbers."""
    c = s["case"]
    rd = c["rotary_dim"]
    turn = torch.outer(pos.double(), s["freqs"].cpu()) * (-1 if c.get("inverse") else 1)
    turn = torch.polar(torch.full_like(turn, _amplitude(c)), turn).to(x.device)[:, None]
    y = x.double().clone()
    if c["layout"] == "half":
        z = torch.complex(y[..., :rd // 2], y[..., rd // 2:rd].contiguous()) * turn
        y[..., :rd // 2], y[..., rd // 2:rd] = z.real, z.imag
    else:
        z = torch.view_as_complex(y[..., :rd].unflatten(-1, (-1, 2)).contiguous()) * turn
        y[..., :rd] = torch.view_as_real(z).flatten(-2)
    return y


def _exact_rotary(s):
    out = {k: s[k + "_out"].double() for k in ("q", "k")}
    for _, first, n, pos in _spans(s):
        for k in out:
            out[k][first:first + n] = _exact_turned(s, s[k][first:first + n], pos)
    return out


def _exact_append(s):
    page = s["case"]["page"]
    out = {k: s[k].double() for k in ("k_pool", "v_pool")}
    out["q"] = s["q_out"].double()
    out["k"] = None if s["k_out"] is None else s["k_out"].double()
    for r, first, n, pos in _spans(s):
        rows = slice(first, first + n)
        out["q"][rows] = _exact_turned(s, s["q"][rows], pos)
        k = _exact_turned(s, s["k"][rows], pos)
        if out["k"] is not None:
            out["k"][rows] = k
        pages = s["page_table"][r].cpu().long()[pos // page].to(k.device)
        out["k_pool"][pages, :, (pos % page).to(k.device)] = k
        out["v_pool"][pages, :, (pos % page).to(k.device)] = s["v"][rows].double()
    return out


def _exact_logits(s):
    """Every node's context written out, and its tokens counted."""
    c = s["case"]
    V, dev = c["vocab"], s["logits"].device
    out = s["out"].double()
    for r, x in enumerate(s["sizes"]):
        n, paths = x["history"], []
        old = torch.bincount(s["history"][r, :n].long(), minlength=V)
        said = torch.bincount(s["history"][r, n * 3 // 4:n].long(), minlength=V)
        rep, pres, freq = (float(s[k][r]) for k in ("repetition", "presence", "frequency"))
        extra = torch.zeros(V, dtype=torch.float64, device=dev)
        if c["bias"]:
            m = c["bias"] - r % 2
            extra.index_put_((s["bias_token"][r, :m].long(),), s["bias_value"][r, :m].double(),
                             accumulate=True)
        for i, at in enumerate(x["parent"]):
            paths.append((paths[at] if at >= 0 else []) + [i])
            mine = torch.bincount(s["token"][r, paths[i]].long(), minlength=V)
            y = s["logits"][r, i].double()
            hit = (old + mine) > 0
            y[hit] = torch.where(y[hit] > 0, y[hit] / rep, y[hit] * rep)
            count = (said + mine).double()
            y = y - freq * count - pres * (count > 0).double() + extra
            if c["masked"]:
                words = s["mask"][r, i].long()[:, None] & (1 << torch.arange(32, device=dev))
                y[(words == 0).flatten()[:V]] = NEG
            out[r, i] = y
    return {"out": out}


def _exact_forward(s, x, gate, residual, post_weight, pre_weight):
    c = s["case"]
    n = x
    if c["post"]:
        parts = x.split(c["group"] or c["width"], dim=1)
        n = torch.cat([p / (p.pow(2).mean(1, keepdim=True) + EPS).sqrt() for p in parts], 1)
        n = n * (post_weight.repeat(len(parts)) if c["shared"] else post_weight)
    if c["gate"] != "none":
        n = n * torch.sigmoid(gate) * (gate if c["gate"] == "silu" else 1.0)
    y = n / 2 if residual is None else residual + n / 2
    h = y / (y.pow(2).mean(1, keepdim=True) + EPS).sqrt() * pre_weight if c["pre"] else None
    return y, h


INPUTS = ("x", "gate", "residual", "post_weight", "pre_weight")


def _exact_norm(s):
    y, h = _exact_forward(s, *(None if s[k] is None else s[k].double() for k in INPUTS))
    return {"y": y if s["has_y"] else None, "h": h}


def _exact_norm_bwd(s):
    """By automatic differentiation of the definition."""
    ins = [None if s[k] is None else s[k].detach().double().requires_grad_() for k in INPUTS]
    y, h = _exact_forward(s, *ins)
    total = 0.0
    for out, grad in ((y, s["dy"]), (h, s["dh"])):
        if grad is not None:
            total = total + (out * grad.double()).sum()
    total.backward()
    return {"d" + k: None if x is None else x.grad for k, x in zip(INPUTS, ins)}
