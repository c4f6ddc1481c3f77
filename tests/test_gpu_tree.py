"""The tree-drafted decoding calls on the GPU against their fp64 definitions.

Tolerances, from the arithmetic and before any run:
  softmax  fp32: the score error of a D-long fp32 dot product, ~ sqrt(D) 2^-24
           of |q||k| s ~ sqrt(D), enters the probabilities relatively: 1e-5.
           bf16: rounding the output (2^-9 at most, 2^-9 / sqrt 3 in the mean)
           and the probabilities (the same, averaged over the keys): 2 x 2^-9.
           lse: fp32 sums of exponentials in both: 5e-5 absolute.
  linear   fp32: 1e-5.  bf16: the output, the state operand, the deltas and
           the decayed products rounded to bf16, 2^-9 / sqrt 3 each,
           independent: 5e-3.
  commit   fp32 recurrence: 1e-5.
  verify   decisions equal wherever the fp64 margin exceeds 1e-4; node_logp
           5e-5 absolute (fp32 logits up to ~20 and an fp32 log-sum-exp).
All relative ones are Frobenius norms per tensor.
"""
import numpy as np
import pytest
import torch

from oracle import tree as ref
from paper_2606_01774_gb300 import flare
from tree_helpers import (linear_inputs, random_paths, run_linear, run_softmax, run_verify,
                          softmax_inputs, verify_inputs)

pytestmark = pytest.mark.gpu

SOFTMAX_REL = {"f32": 1e-5, "bf16": 2 * 2.0 ** -9}
LINEAR_REL = {"f32": 1e-5, "bf16": 5e-3}
LSE_ABS = 5e-5
STATE_REL = 1e-5
LOGP_ABS = 5e-5


def rel(a, b):
    a = a.double().cpu().numpy()
    assert np.isfinite(a).all()
    n = np.linalg.norm(b)
    return np.linalg.norm(a - b) / n if n else np.abs(a).max()


def check_softmax(s, **kw):
    out, lse = run_softmax(s, **kw)
    want, want_lse = ref.tree_softmax(*(x.cpu() for x in (s.q, s.k_blk, s.v_blk, s.k_pool, s.v_pool,
                                                          s.page_table, s.prefix_len, s.parent,
                                                          s.node_len)))
    dead = np.arange(s.N) >= s.node_len.cpu().numpy()[:, None]
    assert (out.float().cpu().numpy()[dead] == 0).all()
    assert (lse.cpu().numpy()[dead] == -np.inf).all()
    live = ~dead
    if live.any():
        assert rel(out[torch.from_numpy(live).cuda()], want[live]) <= SOFTMAX_REL[s.dtype]
        assert np.abs(lse.double().cpu().numpy()[live] - want_lse[live]).max() <= LSE_ABS
    return out, lse


SOFTMAX_SHAPES = [
    # N, Hq, Hkv, D, page, prefix lengths
    (1, 4, 1, 128, 16, [0, 1, 63, 64, 65, 700]),
    (16, 16, 2, 256, 64, [5, 513, 0, 64]),
    (64, 8, 4, 128, 32, [130, 0, 1]),
    (64, 16, 2, 256, 64, [190, 1027]),  # four row tiles of 128
    (13, 6, 2, 64, 128, [127, 128, 129, 1, 0]),
    (33, 7, 1, 64, 16, [77, 15, 16, 17]),  # a group that does not divide a row tile
    (5, 40, 1, 128, 64, [200, 333]),
    (7, 3, 3, 256, 128, [1000, 2, 0]),
    (64, 12, 4, 128, 16, [70, 129]),   # three heads a group, two row tiles of whole nodes
    (61, 10, 2, 64, 64, [300, 31]),    # five
    (50, 7, 1, 256, 32, [100]),        # seven, three row tiles
    (3, 150, 1, 64, 16, [70, 0]),      # more heads than a row tile has rows
    (5, 260, 2, 128, 64, [65, 300]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,Hq,Hkv,D,page,prefix", SOFTMAX_SHAPES)
def test_softmax_matches_the_definition(N, Hq, Hkv, D, page, prefix, dtype):
    R = len(prefix)
    nodes = [N] + [max(1, N * (r + 1) // (R + 1)) for r in range(1, R)]
    check_softmax(softmax_inputs(11 + N, R, N, Hq, Hkv, D, page, prefix, dtype, nodes))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", ["chain", "star", "mixed"])
def test_softmax_tree_shapes_and_resting_requests(shape, dtype):
    nodes = [64, 0, 63, 33, 0, 32, 31, 2]
    prefix = [40, 50, 0, 64, 0, 129, 3, 0]
    check_softmax(softmax_inputs(3, 8, 64, 4, 2, 64, 16, prefix, dtype, nodes, shape))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_softmax_one_long_prefix_is_shared_by_the_whole_gpu(dtype):
    check_softmax(softmax_inputs(5, 1, 3, 4, 2, 128, 64, [20011], dtype, [3]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_softmax_many_short_requests(dtype):
    """More requests than one CTA has threads for, most of them tiny."""
    R = 700
    prefix = [(r * 37) % 50 if r % 100 else 900 for r in range(R)]
    nodes = [r % 4 for r in range(R)]
    check_softmax(softmax_inputs(6, R, 3, 2, 1, 64, 16, prefix, dtype, nodes))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_softmax_without_any_cache(dtype):
    s = softmax_inputs(8, 3, 9, 4, 2, 128, 16, [0, 0, 0], dtype, [9, 4, 1])
    s.desc.max_pages_per_req = 0
    s.desc.num_pages = 0
    need = flare.flare_tree_softmax_workspace_size(s.desc)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    out, st = torch.empty_like(s.q), torch.zeros(1, dtype=torch.int32, device="cuda")
    flare.check(flare.flare_tree_softmax_attn(s.desc, s.q, s.k_blk, s.v_blk, None, None, None,
                                              s.prefix_len, s.parent, s.node_len, out, None, ws,
                                              need, st))
    assert flare.flare_read_status(st) == (0, 0)
    want, _ = ref.tree_softmax(*(x.cpu() for x in (s.q, s.k_blk, s.v_blk, s.k_pool, s.v_pool,
                                                   s.page_table, s.prefix_len, s.parent,
                                                   s.node_len)))
    assert rel(out, want) <= SOFTMAX_REL[dtype]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_softmax_tensors_on_16_byte_boundaries(dtype):
    """Every tensor 16 bytes off a 32-byte boundary."""
    s = softmax_inputs(12, 3, 20, 8, 2, 128, 32, [500, 33, 0], dtype, [20, 7, 1])
    for k in ("q", "k_blk", "v_blk", "k_pool", "v_pool"):
        x = getattr(s, k)
        pad = 16 // x.element_size()
        y = torch.empty(x.numel() + pad, dtype=x.dtype, device="cuda")[pad:].view(x.shape)
        y.copy_(x)
        setattr(s, k, y)
    out = torch.empty(s.q.numel() + 16 // s.q.element_size(), dtype=s.q.dtype, device="cuda")
    out = out[16 // s.q.element_size():].view(s.q.shape)
    assert out.data_ptr() % 32 == 16
    check_softmax(s, out=out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefix", [[9000, 3000, 6100], [2500] * 40, [64 * 150 - 1] * 2])
def test_softmax_items_in_a_few_pieces(prefix, dtype):
    """Items that two to four spans share, and more."""
    R = len(prefix)
    check_softmax(softmax_inputs(13, R, 17, 8, 2, 64, 64, prefix, dtype, [17 - r % 5 for r in range(R)]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_softmax_skips_bad_requests_and_no_other(dtype):
    prefix = [300, 100, 64, 65, 0, 129, 500]
    s = softmax_inputs(9, 7, 20, 4, 2, 128, 16, prefix, dtype, [20, 3, 20, 7, 5, 20, 1])
    good = check_softmax(s)
    s.page_table[0, 3] = s.k_pool.shape[0]  # a page past the pool
    s.parent[2, 5] = 5                      # its own parent
    s.prefix_len[5] = s.cols * 16 + 1       # past the table
    s.node_len[6] = 21                      # more nodes than the descriptor has
    out, lse = torch.full_like(s.q, 7.0), torch.full(s.q.shape[:3], 7.0, device="cuda")
    run_softmax(s, flare.FLARE_DEV_BAD_PAGE | flare.FLARE_DEV_BAD_TREE |
                flare.FLARE_DEV_BAD_PREFIX_LEN, out, lse)
    for r in (0, 2, 5, 6):
        assert (out[r] == 7).all() and (lse[r] == 7).all()
    for r in (1, 3, 4):  # the batch is cut elsewhere now: equal to rounding, not to the bit
        assert torch.allclose(out[r].float(), good[0][r].float(), atol=2e-2, rtol=2e-2)
        assert torch.allclose(lse[r], good[1][r], atol=LSE_ABS)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_softmax_is_the_same_bits_again_on_another_stream_and_from_a_graph(dtype):
    s = softmax_inputs(10, 5, 16, 16, 2, 128, 64, [4000, 0, 777, 64, 1500], dtype, [16, 1, 9, 0, 16])
    first = run_softmax(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run_softmax(s, stream=side)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    need = flare.flare_tree_softmax_workspace_size(s.desc)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros_like(s.q), torch.zeros(s.q.shape[:3], device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        flare.check(flare.flare_tree_softmax_attn(
            s.desc, s.q, s.k_blk, s.v_blk, s.k_pool, s.v_pool, s.page_table, s.prefix_len,
            s.parent, s.node_len, out, lse, ws, need, st))
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    assert int(st) == 0


# ------------------------------------------------------------------ linear layers


def check_linear(s):
    out = run_linear(s)
    want = ref.tree_linear(*(x.cpu() for x in (s.q, s.k, s.v, s.log_decay, s.beta, s.state_pool,
                                               s.slot, s.parent, s.node_len)))
    dead = torch.arange(s.N, device="cuda") >= s.node_len[:, None]
    assert (out[dead] == 0).all()
    if (~dead).any():
        live = ~dead
        assert rel(out[live], want[live.cpu().numpy()]) <= LINEAR_REL[s.dtype]
    return out


LINEAR_SHAPES = [
    # N, Hk, Hv, dk, dv, nodes
    (1, 2, 4, 128, 128, [1, 1, 0]),
    (8, 4, 4, 128, 128, [8, 7, 1, 5]),
    (16, 2, 4, 128, 128, [16, 15, 2]),
    (17, 2, 2, 128, 128, [17, 16, 3]),
    (32, 1, 2, 128, 128, [32, 31, 0]),
    (33, 2, 4, 128, 128, [33, 1]),
    (64, 2, 4, 128, 128, [64, 63, 33, 32, 7]),
    (64, 2, 2, 64, 64, [64, 17]),
    (21, 1, 3, 64, 128, [21, 20]),
    (21, 3, 3, 128, 64, [21, 4]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,Hk,Hv,dk,dv,nodes", LINEAR_SHAPES)
def test_linear_matches_the_recurrence(N, Hk, Hv, dk, dv, nodes, dtype):
    check_linear(linear_inputs(20 + N, len(nodes), N, Hk, Hv, dk, dv, dtype, nodes))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [16, 30, 64])
@pytest.mark.parametrize("shape", ["chain", "star"])
def test_linear_chains_and_stars(shape, N, dtype):
    check_linear(linear_inputs(4, 3, N, 2, 2, 128, 128, dtype, [N, N - 1, 2], shape))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [16, 30, 64])
@pytest.mark.parametrize("decay", [0.0, -3.0, -40.0])
def test_linear_decay_extremes(decay, N, dtype):
    """No decay, and decays whose differences across branches overflow exp()."""
    check_linear(linear_inputs(5, 2, N, 1, 2, 128, 128, dtype, [N, N // 2], "mixed", decay))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [16, 64])
def test_linear_more_items_than_the_gpu_holds(N, dtype):
    R, Hv = 40, 16
    s = linear_inputs(6, R, N, 16, Hv, 128, 128, dtype, [N if r % 3 else r % N for r in range(R)])
    out = run_linear(s)
    pick = [0, 1, 20, 38, 39]
    want = ref.tree_linear(*(x.cpu() for x in (s.q, s.k, s.v, s.log_decay, s.beta, s.state_pool,
                                               s.slot, s.parent, s.node_len)), requests=pick)
    for a, r in enumerate(pick):
        n = int(s.node_len[r])
        if n:
            assert rel(out[r, :n], want[a, :n]) <= LINEAR_REL[dtype]
    assert torch.equal(out, run_linear(s))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [12, 64])
def test_linear_skips_bad_requests_and_leaves_the_pool(N, dtype):
    s = linear_inputs(7, 4, N, 2, 4, 128, 128, dtype, [N, N, N, 5])
    good = check_linear(s)
    before = s.state_pool.clone()
    s.slot[0] = s.state_pool.shape[0]
    s.parent[1, 3] = 3
    s.node_len[2] = -1
    out = run_linear(s, flare.FLARE_DEV_BAD_SLOT | flare.FLARE_DEV_BAD_TREE)
    assert (out[:3] == 7).all()
    assert torch.equal(out[3], good[3])
    same = (s.state_pool == before) | (s.state_pool.isnan() & before.isnan())
    assert bool(same.all())


def test_linear_chain_agrees_with_the_commit():
    """A chain's last node reads the state that committing the whole chain writes."""
    s = linear_inputs(12, 2, 12, 2, 2, 64, 64, "f32", [12, 12], "chain")
    out = run_linear(s)
    path, n = random_paths(0, 2, 12, [12, 12])
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    flare.check(flare.flare_tree_commit_state(s.desc, s.k, s.v, s.log_decay, s.beta, s.state_pool,
                                              s.slot, s.dst_slot, path, n, st))
    S = s.state_pool[s.dst_slot.long()].double()
    y = torch.einsum("rhkv,rhk->rhv", S, s.q[:, 11].double()) * s.desc.scale
    assert int(st) == 0 and rel(out[:, 11], y.cpu().numpy()) <= 2e-5


# ------------------------------------------------------------------ commit


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("N,Hk,Hv,dk,dv", [(1, 2, 4, 128, 128), (16, 2, 4, 128, 128),
                                           (64, 1, 2, 128, 128), (40, 2, 2, 64, 64),
                                           (9, 1, 3, 64, 128), (9, 1, 1, 128, 64)])
def test_commit_state_follows_the_path(N, Hk, Hv, dk, dv, in_place, dtype):
    lens = [N, 0, 1, N // 2, max(0, N - 1)]
    s = linear_inputs(30 + N, 5, N, Hk, Hv, dk, dv, dtype, [N] * 5)
    path, n = random_paths(N, 5, N, lens)
    dst = s.slot if in_place else s.dst_slot
    before = s.state_pool.clone()
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    flare.check(flare.flare_tree_commit_state(s.desc, s.k, s.v, s.log_decay, s.beta, s.state_pool,
                                              s.slot, dst, path, n, st))
    assert int(st) == 0
    want = ref.tree_commit(*(x.cpu() for x in (s.k, s.v, s.log_decay, s.beta, before, s.slot, path,
                                               n)))
    for r in range(5):
        got = s.state_pool[int(dst[r])]
        assert rel(got, want[r]) <= STATE_REL
        if lens[r] == 0:
            assert torch.equal(got, before[int(s.slot[r])])
    rest = torch.ones(before.shape[0], dtype=torch.bool)
    rest[dst.long().cpu()] = False
    a, b = s.state_pool[rest.cuda()], before[rest.cuda()]
    assert bool(((a == b) | (a.isnan() & b.isnan())).all())


def test_commit_state_forks_one_source():
    s = linear_inputs(31, 3, 8, 2, 2, 128, 128, "bf16", [8, 8, 8])
    s.slot[:] = s.slot[0].clone()
    path, n = random_paths(2, 3, 8, [5, 0, 8])
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    before = s.state_pool.clone()
    flare.check(flare.flare_tree_commit_state(s.desc, s.k, s.v, s.log_decay, s.beta, s.state_pool,
                                              s.slot, s.dst_slot, path, n, st))
    want = ref.tree_commit(*(x.cpu() for x in (s.k, s.v, s.log_decay, s.beta, before, s.slot, path,
                                               n)))
    assert int(st) == 0 and rel(s.state_pool[s.dst_slot.long()], want) <= STATE_REL
    assert torch.equal(s.state_pool[int(s.slot[0])], before[int(s.slot[0])])


def test_commit_state_skips_bad_requests():
    s = linear_inputs(32, 5, 8, 2, 2, 128, 128, "bf16", [8] * 5)
    path, n = random_paths(3, 5, 8, [8, 3, 4, 5, 6])
    s.slot[0] = -1
    s.dst_slot[1] = s.state_pool.shape[0]
    path[2, 3] = 8
    n[3] = 9
    before = s.state_pool.clone()
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    flare.check(flare.flare_tree_commit_state(s.desc, s.k, s.v, s.log_decay, s.beta, s.state_pool,
                                              s.slot, s.dst_slot, path, n, st))
    assert int(st) == (flare.FLARE_DEV_BAD_SLOT | flare.FLARE_DEV_BAD_TREE |
                       flare.FLARE_DEV_BAD_ACCEPT_LEN)
    moved = (s.state_pool != before) & ~(s.state_pool.isnan() & before.isnan())
    assert [i for i in range(before.shape[0]) if bool(moved[i].any())] == [int(s.dst_slot[4])]


# ------------------------------------------------------------------ append


def _append(s, layers, path, n):
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    kb, vb, kp, vp = ([x[i] for x in layers] for i in range(4))
    flare.check(flare.flare_tree_append_kv(s.desc, kb, vb, kp, vp, s.page_table, s.prefix_len, path,
                                           n, st))
    return int(st)


@pytest.mark.parametrize("dtype,num_layers", [("bf16", 1), ("f32", 3), ("bf16", 64)])
@pytest.mark.parametrize("N,Hkv,D,page,prefix", [(16, 2, 256, 64, [0, 63, 64, 500]),
                                                 (64, 3, 64, 16, [15, 1, 0, 33]),
                                                 (1, 1, 128, 128, [127, 128, 0, 3])])
def test_append_places_the_path_bit_for_bit(N, Hkv, D, page, prefix, dtype, num_layers):
    s = softmax_inputs(40, 4, N, Hkv, Hkv, D, page, prefix, dtype, [N] * 4, room=N)
    path, n = random_paths(N, 4, N, [N, 0, (N + 1) // 2, 1])
    layers = []
    for i in range(num_layers):
        layers.append([s.k_blk + i, s.v_blk - i, s.k_pool.clone(), s.v_pool.clone()])
    want = [[ref.tree_append(b.cpu(), q.cpu(), s.page_table.cpu(), s.prefix_len.cpu(), path.cpu(),
                             n.cpu()) for b, q in ((x[0], x[2]), (x[1], x[3]))] for x in layers]
    assert _append(s, layers, path, n) == 0
    view = torch.int16 if dtype == "bf16" else torch.int32
    for x, w in zip(layers, want):
        assert torch.equal(x[2].cpu().view(view), w[0].view(view))
        assert torch.equal(x[3].cpu().view(view), w[1].view(view))


def test_append_skips_bad_requests():
    s = softmax_inputs(41, 5, 8, 2, 2, 64, 16, [20, 30, 40, 50, 60], "bf16", [8] * 5, room=8)
    path, n = random_paths(1, 5, 8, [8, 8, 8, 8, 8])
    s.page_table[0, 27 // 16] = s.k_pool.shape[0]
    path[1, 2] = -1
    n[2] = 9
    s.prefix_len[3] = s.cols * 16 - 7
    layers = [[s.k_blk, s.v_blk, s.k_pool.clone(), s.v_pool.clone()]]
    got = _append(s, layers, path, n)
    assert got == (flare.FLARE_DEV_BAD_PAGE | flare.FLARE_DEV_BAD_TREE |
                   flare.FLARE_DEV_BAD_ACCEPT_LEN | flare.FLARE_DEV_BAD_PREFIX_LEN)
    n2 = n.clone()
    n2[:4] = 0
    want = ref.tree_append(s.k_blk.cpu(), s.k_pool.cpu(), s.page_table.cpu(), s.prefix_len.cpu(),
                           path.cpu(), n2.cpu())
    assert torch.equal(layers[0][2].cpu().view(torch.int16), want.view(torch.int16))


# ------------------------------------------------------------------ verification


def check_verify(s, near_allowed=0.05):
    got = run_verify(s)
    cpu = {k: (None if v is None else v.cpu()) for k, v in
           dict(l=s.logits, d=s.draft_probs, t=s.token, p=s.parent, n=s.node_len, u=s.uniform,
                e=s.noise).items()}
    want = ref.tree_verify(cpu["l"], cpu["d"], cpu["t"], cpu["p"], cpu["n"], cpu["u"], cpu["e"],
                           s.greedy, s.inv_temp)
    sure = want["margin"] > 1e-4
    assert (~sure).mean() <= near_allowed
    for k in ("path", "path_len", "next_token"):
        assert np.array_equal(got[k].cpu().numpy()[sure], want[k][sure]), k
    assert np.abs(got["node_logp"].double().cpu().numpy() - want["node_logp"]).max() <= LOGP_ABS
    return got, want


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("drafts,greedy", [("sampled", False), ("top", False), ("top", True)])
@pytest.mark.parametrize("R,N,V,shape", [(40, 16, 1000, "mixed"), (24, 9, 4999, "star"),
                                         (24, 12, 777, "chain"), (5, 64, 2049, "mixed"),
                                         (12, 1, 3001, "mixed"), (64, 7, 5, "mixed"),
                                         (3, 6, 70001, "mixed")])
def test_verify_matches_the_definition(R, N, V, shape, drafts, greedy, dtype):
    nodes = [max(1, N - r % 4) for r in range(R)]
    nodes[-1] = 0
    check_verify(verify_inputs(50 + N, R, N, V, dtype, drafts, greedy, nodes=nodes, shape=shape))


def test_verify_vocabulary_of_one():
    s = verify_inputs(51, 3, 4, 1, "f32", "sampled", nodes=[4, 1, 0], shape="chain")
    got = run_verify(s)
    assert got["path_len"].tolist() == [4, 1, 0] and got["next_token"].tolist() == [0, 0, -1]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [1, 3])
def test_verify_rows_off_every_alignment(offset, dtype):
    check_verify(verify_inputs(52, 9, 6, 1003, dtype, "sampled", offset=offset, nodes=[6] * 9))


@pytest.mark.parametrize("close", [0.0, 0.05, 4.0])
def test_verify_near_and_far_drafters(close):
    """A drafter equal to the target is always accepted; far ones are rejected down to residuals
    of several siblings."""
    s = verify_inputs(53, 48, 10, 600, "f32", "sampled", inv_temp=1.0, nodes=[10] * 48,
                      shape="chain" if close == 0 else "star", close=close)
    got, want = check_verify(s, 1.0 if close == 0 else 0.05)
    if close == 0:
        assert got["path_len"].tolist() == [10] * 48
    if close == 4.0:
        assert (want["path_len"] == 1).sum() >= 4


def test_verify_equal_logits_take_the_lowest_index():
    s = verify_inputs(54, 4, 5, 300, "bf16", "top", greedy=True, nodes=[5] * 4, shape="chain")
    s.logits.fill_(0.5)
    s.logits[:, :, 100:] = 1.5
    s.token[:, 1:] = 100
    s.token[2, 3] = 101
    got = run_verify(s)
    assert got["path_len"].tolist() == [5, 5, 3, 5]
    assert got["next_token"].tolist() == [100] * 4


def test_verify_tokens_ruled_out_are_never_drawn():
    """-inf logits, and the type's lowest finite value, beside ordinary ones."""
    s = verify_inputs(55, 30, 5, 400, "bf16", "sampled", nodes=[5, 1, 3] * 10)
    s.logits[:, :, ::2] = float("-inf")
    s.logits[:, :, 1::4] = torch.finfo(torch.bfloat16).min
    for r in range(30):
        s.logits[r, int(s.node_len[r]):] = float("nan")
    got = run_verify(s)
    assert bool((got["next_token"] % 4 == 3).all())
    x = s.logits.float() * s.inv_temp
    logp = torch.log_softmax(x, -1)
    for r in range(30):
        for i in range(1, int(s.node_len[r])):
            want = float(logp[r, int(s.parent[r, i]), int(s.token[r, i])])
            have = float(got["node_logp"][r, i])
            assert have == want if want == float("-inf") else abs(have - want) <= max(
                LOGP_ABS, 1e-6 * abs(want))


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("greedy", [False, True])
def test_verify_flags_bad_rows_and_no_other_request(value, greedy):
    s = verify_inputs(56, 6, 4, 2000, "f32", "top" if greedy else "sampled", greedy, nodes=[4] * 6,
                      shape="chain")
    good = run_verify(s)
    s.logits[1, 2, 1234] = value   # a row with a child
    s.logits[4, 0] = float("-inf")  # no token left
    got = run_verify(s, flare.FLARE_DEV_BAD_LOGITS)
    for k in got:
        assert (got[k][[1, 4]] == 99).all(), k
        assert torch.equal(got[k][[0, 2, 3, 5]], good[k][[0, 2, 3, 5]]), k


def test_verify_skips_bad_trees_and_tokens():
    s = verify_inputs(57, 5, 6, 500, "bf16", "sampled", nodes=[6] * 5)
    good = run_verify(s)
    s.node_len[0] = 7
    s.parent[1, 4] = 4
    s.token[2, 3] = 500
    s.token[3, 5] = -1
    got = run_verify(s, flare.FLARE_DEV_BAD_TREE)
    for k in got:
        assert (got[k][:4] == 99).all() and torch.equal(got[k][4], good[k][4])


def test_verify_follows_the_target_distribution():
    """Accepted first tokens of many identical requests follow the target, whatever the drafter:
    frequencies within five standard errors."""
    R, V = 20000, 8
    g = torch.Generator(device="cuda")
    g.manual_seed(60)
    target = torch.tensor([0.02, 0.28, 0.05, 0.2, 0.1, 0.15, 0.17, 0.03], device="cuda")
    draft = torch.tensor([0.4, 0.05, 0.1, 0.05, 0.1, 0.1, 0.1, 0.1], device="cuda")
    s = verify_inputs(61, R, 4, V, "f32", "sampled", inv_temp=1.0, nodes=[4] * R, shape="star")
    s.logits[:] = torch.log(target)
    s.draft_probs[:] = draft
    s.token[:, 1:] = torch.multinomial(draft.expand(R, V), 3, replacement=True, generator=g).int()
    got = run_verify(s)
    took = got["path_len"] == 2
    first = torch.where(took, s.token.gather(1, got["path"][:, 1:2].long().clamp(min=0))[:, 0],
                        got["next_token"])
    freq = torch.bincount(first.long(), minlength=V).double() / R
    err = 5 * torch.sqrt(target.double() * (1 - target.double()) / R)
    assert bool(((freq - target.double()).abs() <= err).all()), freq


def test_verify_is_the_same_bits_from_a_graph():
    s = verify_inputs(62, 4, 12, 30001, "bf16", "sampled", nodes=[12] * 4)
    first = run_verify(s)
    need = flare.flare_tree_verify_workspace_size(s.desc)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out = {k: torch.zeros_like(v) for k, v in first.items()}
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        flare.check(flare.flare_tree_verify(s.desc, s.logits, s.draft_probs, s.token, s.parent,
                                            s.node_len, s.uniform, s.noise, out["path"],
                                            out["path_len"], out["next_token"], out["node_logp"],
                                            ws, need, st))
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for k in out:
        assert torch.equal(out[k], first[k]), k
