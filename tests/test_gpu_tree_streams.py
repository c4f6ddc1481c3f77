"""Tree calls repeated bit for bit, beside other calls on a second stream, and from graphs; and the
tensor-core linear kernel's own error.

Tolerance of that error, before any run: rounding to bf16 leaves at most 2^-7 / sqrt 12 of an
output in the root mean square (all mantissas at one); states, deltas and tables as two bf16 parts
add some 2^-16 each, 2^-14 in all.  A state rounded once would add 2^-7 / sqrt 12 again."""
import pytest
import torch

from oracle import tree as ref
from paper_2606_01774_gb300 import flare
from test_gpu_tree import rel
from tree_helpers import (linear_inputs, random_paths, run_linear, run_softmax, run_verify,
                          softmax_inputs, verify_inputs)

pytestmark = pytest.mark.gpu

LINEAR_TC_REL = 2.0 ** -7 / 12 ** 0.5 + 2.0 ** -14


def bits(x):
    return x.contiguous().view({2: torch.int16, 4: torch.int32}[x.element_size()])


@pytest.mark.parametrize("N,Hk,Hv,nodes", [(8, 4, 4, [8, 7, 1, 5]), (16, 2, 8, [16, 15, 9]),
                                           (30, 2, 4, [30, 17]), (64, 2, 4, [64, 63, 40])])
@pytest.mark.parametrize("shape", ["chain", "mixed"])
def test_linear_on_tensor_cores_rounds_its_output_alone(N, Hk, Hv, nodes, shape):
    s = linear_inputs(100 + N, len(nodes), N, Hk, Hv, 128, 128, "bf16", nodes, shape)
    out = run_linear(s)
    want = ref.tree_linear(*(x.cpu() for x in (s.q, s.k, s.v, s.log_decay, s.beta, s.state_pool,
                                               s.slot, s.parent, s.node_len)))
    live = torch.arange(N, device="cuda") < s.node_len[:, None]
    assert rel(out[live], want[live.cpu().numpy()]) <= LINEAR_TC_REL


@pytest.mark.parametrize("N,dtype,d", [(16, "bf16", 128), (32, "bf16", 128), (64, "bf16", 128),
                                       (16, "bf16", 64), (40, "f32", 128)])
def test_linear_repeats_bit_for_bit(N, dtype, d):
    """More items than the GPU holds at once, of every length."""
    R = 48
    s = linear_inputs(101, R, N, 16, 32, d, d, dtype, [(r * 7) % (N + 1) for r in range(R)])
    out = run_linear(s)
    for _ in range(60):
        assert torch.equal(bits(run_linear(s)), bits(out))


@pytest.mark.parametrize("R,N,Hq,Hkv,D,page,longest", [(60, 5, 8, 2, 64, 16, 700),
                                                       (24, 20, 8, 2, 128, 32, 500),
                                                       (20, 9, 4, 1, 256, 64, 900)])
def test_fp32_softmax_repeats_bit_for_bit(R, N, Hq, Hkv, D, page, longest):
    prefix = [longest * r // R for r in range(R)]
    s = softmax_inputs(102, R, N, Hq, Hkv, D, page, prefix, "f32", [1 + r % N for r in range(R)])
    out, lse = run_softmax(s)
    for _ in range(60):
        again, lse2 = run_softmax(s)
        assert torch.equal(bits(again), bits(out)) and torch.equal(bits(lse2), bits(lse))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("drafts", ["sampled", "top"])
@pytest.mark.parametrize("R", [1, 8, 64])
def test_verification_repeats_bit_for_bit(R, drafts, dtype):
    """Clusters of every size, several passes over a row each."""
    s = verify_inputs(103, R, 9, 32000, dtype, drafts, nodes=[9] * R, shape="star", close=4.0)
    first = run_verify(s)
    for _ in range(60):
        again = run_verify(s)
        for k in first:
            assert torch.equal(bits(again[k]), bits(first[k])), k


def test_commit_repeats_bit_for_bit():
    R = 48
    s = linear_inputs(104, R, 16, 16, 32, 128, 128, "bf16", [16] * R)
    path, n = random_paths(1, R, 16, [r % 17 for r in range(R)])
    st = torch.zeros(1, dtype=torch.int32, device="cuda")

    def commit():
        flare.check(flare.flare_tree_commit_state(s.desc, s.k, s.v, s.log_decay, s.beta,
                                                  s.state_pool, s.slot, s.dst_slot, path, n, st))
        return s.state_pool[s.dst_slot.long()]

    first = commit()
    for _ in range(30):
        s.state_pool[s.dst_slot.long()] = 0
        assert torch.equal(bits(commit()), bits(first))
    assert int(st) == 0


def test_two_streams_at_once():
    """Calls on two streams, each with its own workspace, as each alone."""
    soft = [softmax_inputs(105 + i, 24, 16, 16, 2, 128, 64, [(i * 300 + 170 * r) % 2100
                                                            for r in range(24)], "bf16",
                           [1 + (r + i) % 16 for r in range(24)]) for i in range(2)]
    lin = [linear_inputs(107 + i, 12, 16, 4, 16, 128, 128, "bf16",
                         [(r + i) % 17 for r in range(12)]) for i in range(2)]
    ver = [verify_inputs(109 + i, 12, 8, 9001, "bf16", "sampled", nodes=[8] * 12, close=2.0)
           for i in range(2)]

    def buffers(i):
        b = dict(st=torch.zeros(1, dtype=torch.int32, device="cuda"))
        for k, need in (("sw", flare.flare_tree_softmax_workspace_size(soft[i].desc)),
                        ("vw", flare.flare_tree_verify_workspace_size(ver[i].desc))):
            b[k] = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
        b["out"], b["lse"] = torch.zeros_like(soft[i].q), torch.zeros(soft[i].q.shape[:3],
                                                                      device="cuda")
        b["lin"] = torch.zeros_like(lin[i].v)
        v = ver[i]
        b["path"] = torch.zeros(v.R, v.N, dtype=torch.int32, device="cuda")
        b["len"], b["next"] = (torch.zeros(v.R, dtype=torch.int32, device="cuda") for _ in range(2))
        b["logp"] = torch.zeros(v.R, v.N, device="cuda")
        return b

    def calls(i, b, stream):
        s, x, v = soft[i], lin[i], ver[i]
        flare.check(flare.flare_tree_softmax_attn(
            s.desc, s.q, s.k_blk, s.v_blk, s.k_pool, s.v_pool, s.page_table, s.prefix_len,
            s.parent, s.node_len, b["out"], b["lse"], b["sw"], b["sw"].numel(), b["st"], stream))
        flare.check(flare.flare_tree_linear_attn(
            x.desc, x.q, x.k, x.v, x.log_decay, x.beta, x.state_pool, x.slot, x.parent, x.node_len,
            b["lin"], b["st"], stream))
        flare.check(flare.flare_tree_verify(
            v.desc, v.logits, v.draft_probs, v.token, v.parent, v.node_len, v.uniform, v.noise,
            b["path"], b["len"], b["next"], b["logp"], b["vw"], b["vw"].numel(), b["st"], stream))

    alone = [buffers(i) for i in range(2)]
    for i in range(2):
        calls(i, alone[i], torch.cuda.current_stream())
    torch.cuda.synchronize()
    both, streams = [buffers(i) for i in range(2)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            calls(i, both[i], streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert int(alone[i]["st"]) == 0 and int(both[i]["st"]) == 0
        for k in ("out", "lse", "lin", "path", "len", "next", "logp"):
            assert torch.equal(bits(both[i][k]), bits(alone[i][k])), k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_linear_commit_and_append_from_a_graph(dtype):
    s = linear_inputs(111, 4, 12, 2, 4, 128, 128, dtype, [12] * 4)
    a = softmax_inputs(112, 4, 12, 2, 2, 64, 16, [30, 0, 16, 47], dtype, [12] * 4, room=12)
    path, n = random_paths(2, 4, 12, [12, 0, 5, 1])
    pools = [a.k_pool.clone(), a.v_pool.clone()]
    out, st = torch.zeros_like(s.v), torch.zeros(1, dtype=torch.int32, device="cuda")

    def calls(k_pool, v_pool):
        flare.check(flare.flare_tree_linear_attn(s.desc, s.q, s.k, s.v, s.log_decay, s.beta,
                                                 s.state_pool, s.slot, s.parent, s.node_len, out,
                                                 st))
        flare.check(flare.flare_tree_commit_state(s.desc, s.k, s.v, s.log_decay, s.beta,
                                                  s.state_pool, s.slot, s.dst_slot, path, n, st))
        flare.check(flare.flare_tree_append_kv(a.desc, [a.k_blk], [a.v_blk], [k_pool], [v_pool],
                                               a.page_table, a.prefix_len, path, n, st))

    calls(*pools)
    want = [x.clone() for x in (out, s.state_pool[s.dst_slot.long()], *pools)]
    k_pool, v_pool = a.k_pool.clone(), a.v_pool.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(k_pool, v_pool)
    out.zero_()
    s.state_pool[s.dst_slot.long()] = 0
    graph.replay()
    torch.cuda.synchronize()
    got = (out, s.state_pool[s.dst_slot.long()], k_pool, v_pool)
    assert int(st) == 0
    for x, y in zip(got, want):
        assert torch.equal(bits(x), bits(y))
