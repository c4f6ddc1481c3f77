"""Seeded inputs for the rotary, logits and norm calls, the calls on them, and their comparison.

Whatever a call must not use is poisoned: unused rows (NaN), unused positions, tokens and table
entries (far out of range); whatever it must not write holds a mark that is looked for after."""
from __future__ import annotations

import random
from types import SimpleNamespace

import numpy as np
import torch

from oracle import steps as ref
from paper_2606_01774_gb300 import flare
from tree_helpers import DTYPES, FAR, make_tree

HALF_STEP = {t: torch.finfo(DTYPES[t][0]).eps / 2 for t in DTYPES}
LAYOUTS = {"half": flare.FLARE_ROTARY_HALF, "pairs": flare.FLARE_ROTARY_INTERLEAVED}
SCALINGS = {"plain": flare.FLARE_ROTARY_PLAIN, "linear": flare.FLARE_ROTARY_LINEAR,
            "base": flare.FLARE_ROTARY_BASE, "by_parts": flare.FLARE_ROTARY_BY_PARTS}
ACTS = {"none": flare.FLARE_ACT_NONE, "silu": flare.FLARE_ACT_SILU,
        "sigmoid": flare.FLARE_ACT_SIGMOID}
MARK = 7.0


def word():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def bits(x):
    return x.contiguous().view({2: torch.int16, 4: torch.int32}[x.element_size()])


def whole(rows):
    return torch.tensor(rows, dtype=torch.int32, device="cuda")


def close(got, want, size, dtype, rel):
    """Every element within its type's half step of the definition, and `rel` of what enters it."""
    got, off = got.double().cpu().numpy(), rel * size
    assert np.array_equal(np.isnan(got), np.isnan(want))
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf])
    fine = ~inf & ~np.isnan(want)
    off = np.broadcast_to(off, want.shape)[fine]
    half = HALF_STEP[dtype]
    bad = np.abs(got[fine] - want[fine]) > half * np.abs(want[fine]) + (1 + half) * off + 1e-37
    assert not bad.any(), (got[fine][bad][:4], want[fine][bad][:4], off[bad][:4])


# ------------------------------------------------------------------ rotary


def make_table(rotary_dim, base=1e4, scaling="plain", **how):
    table = torch.empty(rotary_dim // 2, dtype=torch.int64, device="cuda")
    flare.check(flare.flare_rotary_table(
        flare.rotary_freq_desc(rotary_dim, base, SCALINGS[scaling], **how), table))
    return table


def rotary_inputs(seed, lens, B, Hq, Hkv, D, rd, dtype="bf16", layout="half", fused=True,
                  prefix=None, tree=False, inverse=False, amplitude=1.0, page=0, spare=3,
                  position=None, base=1e4):
    """B = 0: packed rows, `spare` of them behind the last request."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = random.Random(seed)
    dt, code = DTYPES[dtype]
    R = len(lens)
    s = SimpleNamespace(R=R, B=B, lens=lens, Hq=Hq, Hkv=Hkv, D=D, rd=rd, dtype=dtype, code=code,
                        layout=layout, inverse=inverse, amplitude=amplitude, page=page)
    if B:
        s.rows, starts = R * B, [r * B for r in range(R)]
        s.token_len, s.token_start = whole(lens), None
    else:
        starts = [sum(lens[:r]) for r in range(R + 1)]
        s.rows = starts[-1] + spare
        s.token_len, s.token_start = None, whole(starts)
    s.prefix = prefix if prefix is not None else [rng.randrange(5000) for _ in lens]
    s.prefix_len = whole(s.prefix)
    s.live = torch.zeros(s.rows, dtype=torch.bool)
    s.owner, step = np.full(s.rows, -1), np.zeros(s.rows, np.int64)
    s.at = np.zeros(s.rows, np.int64)
    trees = []
    for r, n in enumerate(lens):
        at = slice(starts[r], starts[r] + n)
        s.live[at] = True
        s.owner[at] = r
        s.at[at] = s.prefix[r] + np.arange(n)
        parent = make_tree(rng, n) if tree else []
        trees.append(parent + [FAR] * (B - n))
        depth = []
        for p in parent:
            depth.append(0 if p < 0 else depth[p] + 1)
        step[at] = s.prefix[r] + np.array(depth if tree else range(n))
    s.parent = whole(trees) if tree else None
    s.pos, s.position = step, None
    if position is not None:
        s.position = torch.full((s.rows,), FAR, dtype=torch.int32, device="cuda")
        s.pos = np.array([position(i) for i in range(s.rows)])
        s.position[s.live.cuda()] = whole(s.pos.tolist())[s.live.cuda()]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(dt)

    if fused:
        wide = (Hq + 2 * Hkv) * D
        s.raw = normal(s.rows, wide)
        s.raw[~s.live.cuda()] = float("nan")
        q, k, v = s.raw.split([Hq * D, Hkv * D, Hkv * D], 1)
        s.q, s.k, s.v = (x.unflatten(1, (-1, D)) for x in (q, k, v))
    else:
        s.q, s.k, s.v = normal(s.rows, Hq, D), normal(s.rows, Hkv, D), normal(s.rows, Hkv, D)
        for x in (s.q, s.k, s.v):
            x[~s.live.cuda()] = float("nan")
    s.table = make_table(rd, base)
    pool = {}
    if page:
        used = [-(-(p + n) // page) for p, n in zip(s.prefix, lens)]
        pages = sum(used) + 2
        ids = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        s.page_table = torch.full((R, max([1] + used)), -1, dtype=torch.int32, device="cuda")
        at = 0
        for r, n in enumerate(used):
            s.page_table[r, :n] = ids[at:at + n]
            at += n
        s.k_pool, s.v_pool = normal(pages, Hkv, page, D), normal(pages, Hkv, page, D)
        pool = dict(page_size=page, num_pages=pages, max_pages_per_req=s.page_table.shape[1])
    s.desc = flare.rotary_desc(R, B, s.rows, Hq, Hkv, D, rd, code, LAYOUTS[layout], int(inverse),
                               amplitude, s.q.stride(0), s.k.stride(0), s.v.stride(0), **pool)
    return s


def marked(*shape, dtype):
    return torch.full(shape, MARK, dtype=DTYPES[dtype][0], device="cuda")


def run_rotary(s, q=True, k=True, expect=0, in_place=False, stream=None):
    if in_place:
        qo, ko = s.q, s.k
    else:
        qo = marked(s.rows, s.Hq, s.D, dtype=s.dtype) if q else None
        ko = marked(s.rows, s.Hkv, s.D, dtype=s.dtype) if k else None
    st = word()
    flare.check(flare.flare_rotary(s.desc, s.q if q else None, s.k if k else None, s.table,
                                   s.position, s.prefix_len, s.token_len, s.parent, s.token_start,
                                   qo, ko, st, stream))
    _, got = flare.flare_read_status(st, stream)
    assert got == expect, hex(got)
    return qo, ko


def run_append(s, q=True, dense_k=True, expect=0, pools=None, stream=None):
    qo = marked(s.rows, s.Hq, s.D, dtype=s.dtype) if q else None
    ko = marked(s.rows, s.Hkv, s.D, dtype=s.dtype) if dense_k else None
    k_pool, v_pool = (s.k_pool.clone(), s.v_pool.clone()) if pools is None else pools
    st = word()
    flare.check(flare.flare_rotary_append_kv(
        s.desc, s.q if q else None, s.k, s.v, s.table, s.position, s.prefix_len, s.token_len,
        s.token_start, s.page_table, qo, ko, k_pool, v_pool, st, stream))
    _, got = flare.flare_read_status(st, stream)
    assert got == expect, hex(got)
    return qo, ko, k_pool, v_pool


# cos and sin are each within an ulp and the angle's rounding (2^-23 in all), times the amplitude,
# times the elements, and summed: three more roundings of 2^-24
ROTARY_REL = 2.0 ** -21


def check_rotated(s, x, out, live=None):
    """`out` against the definition in the live rows, the mark in all others."""
    live = s.live if live is None else live
    idx = live.nonzero()[:, 0]
    angle = ref.angles(s.table.cpu().tolist(), s.pos[idx.numpy()])
    want, size = ref.rotate(x[idx.cuda()].cpu(), angle, s.layout, s.inverse, s.amplitude)
    size[..., s.rd:] = 0  # passed on bit for bit
    close(out[idx.cuda()], want, size, s.dtype, ROTARY_REL)
    if (~live).any():
        assert bool((out[~live.cuda()] == MARK).all())


# ------------------------------------------------------------------ logits


def logits_inputs(seed, R, N, V, dtype="bf16", nodes=None, history=100, bias=5, masked=0.5,
                  tree=True, offset=0, penalties=True):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = random.Random(seed)
    dt, code = DTYPES[dtype]
    s = SimpleNamespace(R=R, N=N, V=V, dtype=dtype)
    s.nodes = [rng.randint(0, N) for _ in range(R)] if nodes is None else nodes
    raw = torch.empty(R * N * V + offset, dtype=dt, device="cuda")
    s.logits = raw[offset:].view(R, N, V)
    s.logits.copy_(4 * torch.randn(R, N, V, generator=g, device="cuda"))
    dead = torch.arange(N, device="cuda") >= whole(s.nodes)[:, None]
    s.logits[dead] = float("nan")
    s.node_len = whole(s.nodes)
    few = max(1, V // 7)  # tokens that repeat

    def some(n):
        return [rng.randrange(few) if rng.random() < 0.7 else rng.randrange(V) for _ in range(n)]

    s.history = s.history_len = s.output_start = None
    s.text = s.start = None
    if history:
        s.text = [some(rng.choice([0, 1, history, history - 1, history // 2])) for _ in range(R)]
        s.start = [rng.randint(0, len(t)) for t in s.text]
        s.history = whole([t + [FAR] * (history - len(t)) for t in s.text])
        s.history_len, s.output_start = whole([len(t) for t in s.text]), whole(s.start)
    s.token = s.parent = None
    if tree:
        s.token = whole([some(n) + [FAR] * (N - n) for n in s.nodes])
        s.parent = whole([make_tree(rng, n) + [FAR] * (N - n) for n in s.nodes])
    s.repetition = s.presence = s.frequency = None
    if penalties:
        s.repetition = 0.5 + 2 * torch.rand(R, generator=g, device="cuda")
        s.presence = torch.randn(R, generator=g, device="cuda")
        s.frequency = torch.randn(R, generator=g, device="cuda") * 0.3
    s.bias_token = s.bias_value = s.bias_len = s.bias = None
    if bias:
        s.bias = [[(t, rng.gauss(0, 2)) for t in some(rng.choice([0, 1, bias, bias // 2]))]
                  for _ in range(R)]
        s.bias = [[(t, float(np.float32(b))) for t, b in line] for line in s.bias]
        s.bias_token = whole([[t for t, _ in x] + [FAR] * (bias - len(x)) for x in s.bias])
        s.bias_value = torch.tensor([[b for _, b in x] + [float("nan")] * (bias - len(x))
                                     for x in s.bias], device="cuda")
        s.bias_len = whole([len(x) for x in s.bias])
    s.allowed = s.mask = None
    if masked is not None:
        s.allowed = torch.rand(R, N, V, generator=g, device="cuda") >= masked
        s.mask = pack(s.allowed)
    s.desc = flare.tree_logits_desc(R, N, V, code, history, bias)
    return s


def pack(allowed):
    """[..., V] truth values as words of 32 bits, the first token's bit lowest; bits past V set."""
    V = allowed.shape[-1]
    b = torch.ones(*allowed.shape[:-1], -(-V // 32) * 32, dtype=torch.int64, device=allowed.device)
    b[..., :V] = allowed.long()
    w = (b.unflatten(-1, (-1, 32)) << torch.arange(32, device=allowed.device)).sum(-1)
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32).contiguous()


def run_logits(s, out=None, expect=0, in_place=False, stream=None):
    if in_place:
        out = s.logits
    elif out is None:
        out = torch.full_like(s.logits, MARK)
    st = word()
    flare.check(flare.flare_tree_logits(
        s.desc, s.logits, s.history, s.history_len, s.output_start, s.token, s.parent, s.node_len,
        s.repetition, s.presence, s.frequency, s.bias_token, s.bias_value, s.bias_len, s.mask, out,
        st, stream))
    _, got = flare.flare_read_status(st, stream)
    assert got == expect, hex(got)
    return out


# the reciprocal of the penalty, its product, the count's product, the sums: each 2^-24 of what
# enters, and one more for every bias of a token (up to six here)
LOGITS_REL = 12 * 2.0 ** -24


def check_logits(s, out):
    cpu = lambda x: None if x is None else x.cpu()  # noqa: E731
    want, size = ref.tree_logits(s.logits.cpu(), s.nodes, cpu(s.token), cpu(s.parent), s.text,
                                 s.start, cpu(s.repetition), cpu(s.presence), cpu(s.frequency),
                                 s.bias, None if s.allowed is None else s.allowed.cpu().numpy())
    for r, n in enumerate(s.nodes):
        close(out[r, :n], want[r, :n], size[r, :n], s.dtype, LOGITS_REL)


# ------------------------------------------------------------------ norms


def norm_inputs(seed, T, W, dtype="bf16", group=0, shared=False, post=True, pre=True, gate="none",
                gated=None, residual=True, weights=True, x_pad=0, gate_pad=0, eps=1e-6, alpha=1.0,
                dy=True, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, code = DTYPES[dtype]
    s = SimpleNamespace(T=T, W=W, dtype=dtype, x_pad=x_pad, gate_pad=gate_pad)
    s.how = dict(group=group, shared=shared, post=post, pre=pre, act=gate, eps=eps, alpha=alpha)

    def normal(*shape, dt=dt):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(dt)

    def rows(pad):
        return normal(T, W + pad)[:, pad:] if pad else normal(T, W)

    s.x = rows(x_pad)
    has_gate = gate != "none" if gated is None else gated
    s.gate = rows(gate_pad) if has_gate else None
    s.residual = normal(T, W) if residual else None
    s.post_weight = normal(group if shared else W, dt=torch.float32) if post and weights else None
    s.pre_weight = normal(W, dt=torch.float32) if pre and weights else None
    s.dy = normal(T, W) if dy or not pre else None
    s.dh = normal(T, W) if pre else None
    s.desc = flare.block_norm_desc(T, W, code, group, int(shared), int(post), int(pre), ACTS[gate],
                                   eps, alpha, W + x_pad if x_pad else 0,
                                   W + gate_pad if gate_pad else 0)
    return s


def like_rows(x, pad):
    """Marked rows as x lies, and the marked memory around them."""
    if x is None:
        return None, None
    raw = torch.full((x.shape[0], x.shape[1] + pad), MARK, dtype=x.dtype, device="cuda")
    return (raw[:, pad:] if pad else raw), raw


def run_norm(s, y=True, stream=None):
    y = torch.full((s.T, s.W), MARK, dtype=s.x.dtype, device="cuda") if y else None
    h = torch.full((s.T, s.W), MARK, dtype=s.x.dtype, device="cuda") if s.how["pre"] else None
    flare.check(flare.flare_block_norm(s.desc, s.x, s.gate, s.residual, s.post_weight,
                                       s.pre_weight, y, h, stream))
    return y, h


def run_norm_bwd(s, weights=True, dresidual=True, stream=None):
    need = flare.flare_block_norm_bwd_workspace_size(s.desc)
    ws = torch.full((max(need, 1),), 0xFF, dtype=torch.uint8, device="cuda")
    dx, raw = like_rows(s.x, s.x_pad)
    dgate, raw_gate = like_rows(s.gate, s.gate_pad)
    new = dict(dx=dx, dgate=dgate)
    new["dresidual"] = (torch.full_like(s.residual, MARK)
                        if s.residual is not None and dresidual else None)
    for name, there, wide in (
            ("dpost_weight", s.how["post"],
             s.how["group"] if s.how["shared"] and s.how["group"] else s.W),
            ("dpre_weight", s.how["pre"], s.W)):
        new[name] = torch.full((wide,), MARK, device="cuda") if there and weights else None
    flare.check(flare.flare_block_norm_bwd(
        s.desc, s.x, s.gate, s.residual, s.post_weight, s.pre_weight, s.dy, s.dh, dx, dgate,
        new["dresidual"], new["dpost_weight"], new["dpre_weight"], ws, need, stream))
    for pad, mem in ((s.x_pad, raw), (s.gate_pad, raw_gate)):
        if mem is not None and pad:
            assert bool((mem[:, :pad] == MARK).all())
    return new


# A sum of squares: a thread's terms one after another (64 at most), the threads' by halving (10):
# 75 roundings of 2^-24 of positive terms, half of that in the root, and a few more of its own and
# of the products: 2^-18.  h has two such norms.  A gradient passes four such sums.
Y_REL, H_REL, GRAD_REL = 2.0 ** -18, 2.0 ** -17, 2.0 ** -16


def ins(s):
    return [None if x is None else x.double().cpu().numpy()
            for x in (s.x, s.gate, s.residual, s.post_weight, s.pre_weight)]


def check_norm(s, y, h):
    wy, wh, sy, sh = ref.block_norm(*ins(s), **s.how)
    if y is not None:
        close(y, wy, sy, s.dtype, Y_REL)
    if h is not None:
        close(h, wh, sh, s.dtype, H_REL)


def check_norm_bwd(s, got):
    down = lambda x: None if x is None else x.double().cpu().numpy()  # noqa: E731
    want, size = ref.block_norm_bwd(*ins(s), down(s.dy), down(s.dh), **s.how)
    for name, x in got.items():
        if x is not None:
            close(x, want[name], size[name], "f32" if "weight" in name else s.dtype, GRAD_REL)
