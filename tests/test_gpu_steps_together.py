"""The rotary, logits and norm calls together with the attention and verification calls they stand
between: a decoder, a cache filled and attended to, masked verification; and all of them on
streams and from graphs.

Tolerances as in test_gpu_tree.py (the attention's) and steps_helpers.py."""
import importlib.util
import threading
from pathlib import Path

import numpy as np
import pytest
import torch

from oracle import steps as ref, tree as ref_tree
from paper_2606_01774_gb300 import flare
from steps_helpers import (bits, logits_inputs, norm_inputs, rotary_inputs, run_append, run_logits,
                           run_norm, run_norm_bwd, run_rotary, whole, word)
from test_gpu_tree import SOFTMAX_REL, rel

pytestmark = pytest.mark.gpu

_at = Path(__file__).resolve().parents[1] / "examples" / "tree_decode.py"
_spec = importlib.util.spec_from_file_location("tree_decode", _at)
tree_decode = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(tree_decode)


def prompt(R, n, seed=3):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randint(0, 512, (R, n), dtype=torch.int32, device="cuda", generator=g)


@pytest.mark.parametrize("layers,length", [("llsl", 21), ("ss", 1), ("sl", 40)])
def test_trees_with_stages_decode_what_single_tokens_decode(layers, length):
    """Every node's penalties are those that its tokens would have one by one."""
    R, rounds = 5, 12
    tokens = prompt(R, length)
    make = lambda: tree_decode.HybridDecoder(R, layers=layers, stages=True)  # noqa: E731
    trees, rate = make().decode(tokens, rounds)
    one, _ = make().decode(tokens, 3 * rounds, plain=True)
    assert rate > 1.1  # the drafter is accepted now and then, or nothing was tested
    for a, b in zip(trees, one):
        assert a == b[:len(a)]
    free, _ = tree_decode.HybridDecoder(R, layers=layers, stages=True, repetition=1.0).decode(
        tokens, 3 * rounds, plain=True)
    assert free != one  # and the penalty does something


def test_bf16_rounds_with_stages_stay_sound():
    new, rate = tree_decode.HybridDecoder(4, dtype="bf16", stages=True).decode(prompt(4, 9), 10)
    assert all(0 <= t < 512 for line in new for t in line) and rate >= 1.0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_prompts_appended_and_attended_to(layout, dtype):
    """Ragged prompts enter the cache by one call; a new token turns, is appended and attends."""
    lens, Hq, Hkv, D, rd, page = [70, 1, 33], 4, 2, 64, 32, 16
    s = rotary_inputs(1, lens, 0, Hq, Hkv, D, rd, dtype, layout, prefix=[0] * 3, page=page)
    table = torch.cat([s.page_table, torch.full((3, 1), -1, dtype=torch.int32, device="cuda")], 1)
    spare = [p for p in range(s.k_pool.shape[0]) if p not in set(s.page_table.flatten().tolist())]
    table[0, 5 if 70 % page == 0 else 4] = int(s.page_table[0, 4])
    s.page_table = table.contiguous()
    s.desc.max_pages_per_req = table.shape[1]
    assert len(spare) == 2
    _, _, k_pool, v_pool = run_append(s, q=False, dense_k=False)
    n = rotary_inputs(2, [1, 1, 1], 1, Hq, Hkv, D, rd, dtype, layout, prefix=lens, page=page)
    n.page_table, n.desc.num_pages, n.desc.max_pages_per_req = (s.page_table, k_pool.shape[0],
                                                                table.shape[1])
    n.table = s.table
    q, k, k_pool, v_pool = run_append(n, pools=(k_pool, v_pool))
    d = flare.softmax_desc(3, 1, Hq, Hkv, D, page, k_pool.shape[0], table.shape[1], s.code,
                           D ** -0.5)
    parent, one = whole([[-1]] * 3), whole([1] * 3)
    ws = torch.empty(flare.flare_tree_softmax_workspace_size(d), dtype=torch.uint8, device="cuda")
    out, st = torch.empty(3, 1, Hq, D, dtype=q.dtype, device="cuda"), word()
    flare.check(flare.flare_tree_softmax_attn(
        d, q.view(3, 1, Hq, D), k.view(3, 1, Hkv, D), n.v.contiguous().view(3, 1, Hkv, D), k_pool,
        v_pool, s.page_table, n.prefix_len, parent, one, out, None, ws, ws.numel(), st))
    assert int(st) == 0
    # the definition: every key turned to its place, one softmax over all of them
    turns = s.table.cpu().tolist()
    at = 0
    for r, m in enumerate(lens):
        rows = slice(at, at + m)
        at += m
        angle = ref.angles(turns, range(m + 1))
        keys = torch.cat([s.k[rows], n.k[r:r + 1]]).double().cpu().numpy()
        keys = ref.rotate(keys, angle, layout)[0]
        if dtype == "bf16":  # the cache holds rounded keys
            keys = torch.from_numpy(keys).bfloat16().double().numpy()
        values = torch.cat([s.v[rows], n.v[r:r + 1]]).double().cpu().numpy()
        query = ref.rotate(n.q[r:r + 1].cpu(), angle[m:], layout)[0][0]
        if dtype == "bf16":
            query = torch.from_numpy(query).bfloat16().double().numpy()
        for h in range(Hq):
            x = keys[:, h // 2] @ query[h] * D ** -0.5
            p = np.exp(x - x.max())
            want = (p / p.sum()) @ values[:, h // 2]
            # the roundings of keys and queries are the definition's but for ties: one more bf16 step
            assert rel(out[r, 0, h], want) <= 2 * SOFTMAX_REL[dtype]


@pytest.mark.parametrize("greedy", [True, False])
def test_verification_of_masked_logits(greedy):
    """What a mask rules out is neither accepted nor drawn, whatever the target thought of it."""
    R, N, V = 4, 6, 3001
    s = logits_inputs(4, R, N, V, "f32", [6, 1, 4, 6], history=30, masked=0.6)
    s.allowed[:, :, 5] = True
    from steps_helpers import pack
    s.mask = pack(s.allowed)
    s.logits.masked_fill_(~s.allowed, 30.0)  # the likeliest tokens are ruled out
    out = run_logits(s)
    d = flare.tree_verify_desc(R, N, V, flare.FLARE_DT_F32,
                               flare.FLARE_VERIFY_GREEDY if greedy else flare.FLARE_VERIFY_SAMPLE)
    ws = torch.empty(flare.flare_tree_verify_workspace_size(d), dtype=torch.uint8, device="cuda")
    path, st = torch.zeros(R, N, dtype=torch.int32, device="cuda"), word()
    path_len, nxt = (torch.zeros(R, dtype=torch.int32, device="cuda") for _ in range(2))
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    uniform = torch.rand(R, N, generator=g, device="cuda")
    noise = torch.empty(R, V, device="cuda").exponential_(generator=g).clamp_(min=1e-12)
    flare.check(flare.flare_tree_verify(
        d, out, None, s.token, s.parent, s.node_len, None if greedy else uniform,
        None if greedy else noise, path, path_len, nxt, torch.empty(R, N, device="cuda"), ws,
        ws.numel(), st))
    assert int(st) == 0
    want = ref_tree.tree_verify(out.cpu(), None, s.token.cpu(), s.parent.cpu(), s.node_len.cpu(),
                                None if greedy else uniform.cpu(), None if greedy else noise.cpu(),
                                greedy=greedy)
    assert np.array_equal(path.cpu().numpy(), want["path"])
    assert np.array_equal(nxt.cpu().numpy(), want["next_token"])
    for r in range(R):
        line = path[r, :int(path_len[r])].tolist()
        for a, b in zip(line, line[1:]):
            assert bool(s.allowed[r, a, int(s.token[r, b])])
        assert bool(s.allowed[r, line[-1], int(nxt[r])])


def everything():
    """Calls of every kind with their outputs, as functions of a stream."""
    rot = rotary_inputs(7, [300, 0, 45], 0, 8, 2, 128, 96, "bf16")
    tree = rotary_inputs(8, [9, 16, 1], 16, 4, 2, 64, 64, "f32", "pairs", tree=True, inverse=True)
    app = rotary_inputs(9, [33, 1, 64], 64, 6, 3, 64, 32, "bf16", prefix=[10, 0, 200], page=32)
    log = [logits_inputs(10, 3, 9, 5000, "bf16", [9, 4, 1]),
           logits_inputs(11, 2, 1, 1111, "f32", [1, 1], history=5000)]
    norm = [norm_inputs(12, 500, 1024, gate="silu", group=128, shared=True, x_pad=64),
            norm_inputs(13, 37, 6000, "f32", gate="sigmoid")]

    def f(stream):
        out = list(run_rotary(rot, stream=stream)) + list(run_rotary(tree, stream=stream))
        out += list(run_append(app, stream=stream))
        for s in log:
            out.append(run_logits(s, stream=stream))
        for s in norm:
            out += list(run_norm(s, stream=stream))
            out += list(run_norm_bwd(s, stream=stream).values())
        return [x for x in out if x is not None]
    return f


def test_on_other_streams_and_repeated_bit_for_bit():
    calls = everything()
    first = calls(None)
    torch.cuda.synchronize()
    for _ in range(10):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = calls(None)  # the current stream
        given = calls(None)
        torch.cuda.synchronize()
        for a, b, c in zip(first, again, given):
            assert torch.equal(bits(a), bits(b)) and torch.equal(bits(a), bits(c))


def test_stream_argument():
    s = norm_inputs(14, 64, 2048)
    want = run_norm(s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, h = torch.empty_like(s.x), torch.empty_like(s.x)
    side.wait_stream(torch.cuda.current_stream())
    flare.check(flare.flare_block_norm(s.desc, s.x, s.gate, s.residual, s.post_weight, s.pre_weight,
                                       y, h, side))
    side.synchronize()
    assert torch.equal(bits(y), bits(want[0])) and torch.equal(bits(h), bits(want[1]))


def test_two_threads_at_once():
    """Calls of the same kernels at different sizes from two host threads, each on its own stream."""
    def work(i):
        log = logits_inputs(30 + i, 3, 2, (90000, 700)[i], "bf16", [2, 1, 2])
        norm = norm_inputs(32 + i, 300, (7168, 512)[i], gate="silu")
        return lambda: ([run_logits(log)] + list(run_norm(norm)) + list(run_norm_bwd(norm).values()))

    calls = [work(0), work(1)]
    want = [f() for f in calls]
    torch.cuda.synchronize()
    wrong = []

    def run(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(30):
                    got = calls[i]()
                    torch.cuda.current_stream().synchronize()
                    # a request's unused rows are marked in both
                    wrong.extend(not torch.equal(bits(a), bits(b)) for a, b in zip(got, want[i]))
        except Exception as e:  # noqa: BLE001
            wrong.append(e)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not any(wrong), [x for x in wrong if x][:3]


def test_from_graphs_that_share_a_workspace():
    """Two graphs of a backward pass over one workspace, replayed in turn, and the other calls."""
    s = [norm_inputs(15 + i, 700, 2048, gate="silu") for i in range(2)]
    need = flare.flare_block_norm_bwd_workspace_size(s[0].desc)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    rot = rotary_inputs(17, [100, 3], 0, 4, 2, 64, 64, "bf16", prefix=[0, 60], page=16)
    log = logits_inputs(18, 2, 5, 4000, "bf16", [5, 3])
    st = word()

    def outputs(x):
        return ([torch.zeros_like(t) for t in (x.x, x.gate, x.residual)] +
                [torch.zeros_like(x.post_weight), torch.zeros_like(x.pre_weight)])

    def calls(x, got, qo, ko, pools, lo):
        flare.check(flare.flare_block_norm_bwd(x.desc, x.x, x.gate, x.residual, x.post_weight,
                                               x.pre_weight, x.dy, x.dh, *got, ws, need))
        flare.check(flare.flare_rotary_append_kv(
            rot.desc, rot.q, rot.k, rot.v, rot.table, None, rot.prefix_len, None, rot.token_start,
            rot.page_table, qo, ko, *pools, st))
        flare.check(flare.flare_tree_logits(
            log.desc, log.logits, log.history, log.history_len, log.output_start, log.token,
            log.parent, log.node_len, log.repetition, log.presence, log.frequency, log.bias_token,
            log.bias_value, log.bias_len, log.mask, lo, st))

    sets = []
    for x in s:
        sets.append((x, outputs(x), torch.zeros(rot.rows, 4, 64, dtype=torch.bfloat16, device="cuda"),
                     torch.zeros(rot.rows, 2, 64, dtype=torch.bfloat16, device="cuda"),
                     (rot.k_pool.clone(), rot.v_pool.clone()), torch.zeros_like(log.logits)))
    flat = lambda c: [*c[1], c[2], c[3], *c[4], c[5]]  # noqa: E731
    for c in sets:
        calls(*c)
    want = [[t.clone() for t in flat(c)] for c in sets]
    graphs = []
    for c in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls(*c)
        graphs.append(graph)
    for _ in range(3):
        for c in sets:
            for t in (*c[1], c[2], c[3], c[5]):
                t.zero_()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for c, w in zip(sets, want):
            for a, b in zip(flat(c), w):
                assert torch.equal(bits(a), bits(b))
    assert int(st) == 0
