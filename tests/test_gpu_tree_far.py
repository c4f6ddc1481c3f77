"""The tree calls where offsets pass 32 bits: long caches, many state slots, large vocabularies.

Tolerances as in test_gpu_tree.py, for the same arithmetic."""
import math

import numpy as np
import pytest
import torch

from oracle import tree as ref
from paper_2606_01774_gb300 import flare
from test_gpu_tree import LOGP_ABS, LINEAR_REL, LSE_ABS, SOFTMAX_REL, STATE_REL, rel
from tree_helpers import DTYPES, linear_inputs, random_paths, run_softmax, run_verify, softmax_inputs

pytestmark = pytest.mark.gpu


def need_memory(gib):
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB of device memory")


def far_cache(s, pages):
    """s with its cache's pages moved to the far end of pools of `pages` pages; the small pools
    and table for the reference."""
    small = s.k_pool, s.v_pool, s.page_table.clone()
    n = s.k_pool.shape[0]
    far = []
    for pool in small[:2]:
        x = torch.empty((pages,) + tuple(pool.shape[1:]), dtype=pool.dtype, device="cuda")
        x[pages - n:] = pool
        far.append(x)
    s.k_pool, s.v_pool = far
    assert s.k_pool[:pages - n].numel() > 1 << 31
    s.page_table[s.page_table >= 0] += pages - n
    s.desc.num_pages = pages
    return small


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_softmax_and_append_in_the_far_pages_of_a_cache(dtype):
    need_memory(40)
    s = softmax_inputs(50, 2, 9, 16, 2, 256, 64, [300, 65], dtype, [9, 4], room=9)
    k_small, v_small, table = far_cache(s, 66000)
    out, lse = run_softmax(s)
    want, want_lse = ref.tree_softmax(*(x.cpu() for x in (s.q, s.k_blk, s.v_blk, k_small, v_small,
                                                          table, s.prefix_len, s.parent,
                                                          s.node_len)))
    for r, n in enumerate((9, 4)):
        assert rel(out[r, :n], want[r, :n]) <= SOFTMAX_REL[dtype]
        assert np.abs(lse[r, :n].double().cpu().numpy() - want_lse[r, :n]).max() <= LSE_ABS
    path, count = random_paths(4, 2, 9, [5, 3])
    path[1, :3] = torch.tensor([0, 2, 3])
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    flare.check(flare.flare_tree_append_kv(s.desc, [s.k_blk], [s.v_blk], [s.k_pool], [s.v_pool],
                                           s.page_table, s.prefix_len, path, count, st))
    assert int(st) == 0
    for blk, pool, small in ((s.k_blk, s.k_pool, k_small), (s.v_blk, s.v_pool, v_small)):
        want = ref.tree_append(blk.cpu(), small.cpu(), table.cpu(), s.prefix_len.cpu(), path.cpu(),
                               count.cpu())
        got = pool[pool.shape[0] - small.shape[0]:].cpu()
        same = (got == want) | (got.isnan() & want.isnan())
        assert bool(same.all())


@pytest.mark.parametrize("dtype,dk,dv", [("bf16", 128, 128), ("f32", 128, 128), ("bf16", 128, 64)])
def test_linear_and_commit_in_the_far_slots_of_a_pool(dtype, dk, dv):
    need_memory(20)
    s = linear_inputs(51, 2, 9, 2, 32, dk, dv, dtype, [9, 9])
    n = s.state_pool.shape[0]
    slots = (1 << 31) // (32 * dk * dv) + n + 1
    pool = torch.empty(slots, 32, dk, dv, device="cuda")
    pool[slots - n:] = s.state_pool
    s.desc.num_state_slots = slots
    slot, dst = s.slot + (slots - n), s.dst_slot + (slots - n)
    out = torch.full_like(s.v, 7.0)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    flare.check(flare.flare_tree_linear_attn(s.desc, s.q, s.k, s.v, s.log_decay, s.beta, pool, slot,
                                             s.parent, s.node_len, out, st))
    want = ref.tree_linear(*(x.cpu() for x in (s.q, s.k, s.v, s.log_decay, s.beta, s.state_pool,
                                               s.slot, s.parent, s.node_len)))
    assert int(st) == 0 and rel(out, want) <= LINEAR_REL[dtype]
    path, count = random_paths(5, 2, 9, [4, 9])
    flare.check(flare.flare_tree_commit_state(s.desc, s.k, s.v, s.log_decay, s.beta, pool, slot, dst,
                                              path, count, st))
    want = ref.tree_commit(*(x.cpu() for x in (s.k, s.v, s.log_decay, s.beta, s.state_pool, s.slot,
                                               path, count)))
    assert int(st) == 0 and rel(pool[dst.long()], want) <= STATE_REL


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_verify_in_the_far_rows_of_the_logits(dtype):
    """Three requests of 64 rows over 2^24 tokens; the last one's rows lie past 2^31 elements."""
    need_memory(60)
    R, N, V = 3, 64, 1 << 24
    dt, code = DTYPES[dtype]
    g = torch.Generator(device="cuda")
    g.manual_seed(52)
    s = type("S", (), {})()
    s.R, s.N, s.V, s.greedy = R, N, V, False
    i32 = dict(dtype=torch.int32, device="cuda")
    s.parent = torch.full((R, N), -1, **i32)
    s.parent[2, :3] = torch.tensor([-1, 0, 0], **i32)
    s.node_len = torch.tensor([0, 0, 3], **i32)
    s.logits = torch.empty(R, N, V, dtype=dt, device="cuda")
    s.draft_probs = torch.empty(R, N, V, device="cuda")
    s.logits[2, :3] = torch.randn(3, V, generator=g, device="cuda").to(dt)
    s.draft_probs[2, 0] = torch.softmax(torch.randn(V, generator=g, device="cuda"), 0)
    s.token = torch.full((R, N), -5, **i32)
    s.token[2, 1], s.token[2, 2] = 17, V - 3
    s.logits[2, 0, 17] = -4.0           # the first sibling is rejected at u = 0.9
    s.logits[2, 0, V - 3] = 6.0         # the second one accepted
    s.uniform = torch.full((R, N), 0.9, device="cuda")
    s.noise = torch.empty(R, V, device="cuda").exponential_(generator=g).clamp_(min=1e-12)
    s.desc = flare.tree_verify_desc(R, N, V, code)
    got = run_verify(s)
    want = ref.tree_verify(s.logits[2:, :3].cpu(), s.draft_probs[2:, :3].cpu(),
                           s.token[2:, :3].cpu(), s.parent[2:, :3].cpu(), s.node_len[2:].cpu(),
                           s.uniform[2:, :3].cpu(), s.noise[2:].cpu())
    assert want["path"][0].tolist() == [0, 2, -1]
    assert got["path"][2, :3].tolist() == [0, 2, -1] and int(got["path_len"][2]) == 2
    if want["margin"][0] > 1e-4:
        assert int(got["next_token"][2]) == want["next_token"][0]
    logp = got["node_logp"][2, :3].double().cpu().numpy()
    assert np.abs(logp - want["node_logp"][0]).max() <= LOGP_ABS
    assert math.isfinite(logp[1]) and got["next_token"][:2].tolist() == [-1, -1]
