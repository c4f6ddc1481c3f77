"""Softmax calls whose pieces, tiles and warps race one another: the same bits every time, and
the definition's values (tolerances as in test_gpu_tree.py); and unused rows beside a NaN."""
import numpy as np
import pytest
import torch

from oracle import tree as ref
from test_gpu_tree import SOFTMAX_REL, rel
from tree_helpers import linear_inputs, run_linear, run_softmax, softmax_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R,N,Hq,Hkv,D,page,longest", [
    (104, 1, 64, 8, 256, 32, 737),   # many items a CTA, every second tile a partial one
    (180, 5, 8, 4, 256, 16, 694),
    (104, 1, 32, 4, 128, 32, 737),
    (60, 61, 24, 8, 128, 64, 1239),  # row tiles with rows to spare
    (90, 20, 8, 2, 64, 16, 500),
])
def test_softmax_repeats_bit_for_bit(R, N, Hq, Hkv, D, page, longest):
    prefix = [(longest * (3 * r + 7)) // (3 * R + 4) - 13 * (r % 5) for r in range(R)]
    prefix = [max(0, p) for p in prefix]
    s = softmax_inputs(70 + N, R, N, Hq, Hkv, D, page, prefix, "bf16",
                       [max(1, N - r % 7) for r in range(R)])
    out, lse = run_softmax(s)
    for _ in range(120):
        again, lse2 = run_softmax(s)
        assert torch.equal(again.view(torch.int16), out.view(torch.int16))
        assert torch.equal(lse2.view(torch.int32), lse.view(torch.int32))
    sample = list(range(0, R, 13))
    want, _ = ref.tree_softmax(*(x.cpu() for x in (s.q, s.k_blk, s.v_blk, s.k_pool, s.v_pool,
                                                   s.page_table, s.prefix_len, s.parent,
                                                   s.node_len)), requests=sample)
    live = np.arange(N) < s.node_len.cpu().numpy()[sample][:, None]
    got = out[torch.tensor(sample, device="cuda")][torch.from_numpy(live).cuda()]
    assert rel(got, want[live]) <= SOFTMAX_REL["bf16"]


@pytest.mark.parametrize("dtype,dk", [("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("N,n", [(12, 5), (16, 15), (30, 17), (40, 33)])
def test_linear_unused_rows_are_zero_beside_a_nan(N, n, dtype, dk):
    """A NaN in the last used node stays out of the rows after it."""
    s = linear_inputs(80, 2, N, 2, 4, dk, dk, dtype, [n, N])
    s.v[0, n - 1] = float("nan")
    out = run_linear(s)
    assert bool((out[0, n:] == 0).all())
    assert bool(torch.isfinite(out[1]).all())
