"""Log-gates so low that the gate is zero in fp32, as models that reset their state write them.

Tolerances, before any run: as in test_gpu_tree.py, and in fp32 the rounding of a path's summed
log-gates, whose differences are the exponents: a gate of zero counts as at most e^-104, K of them
on a path sum to 104 K, and a sum of that size is off by 2^-24 of itself at each addition; over
both sums of a difference and a few additions 2^-22 * 104 K at most, a third of it in the mean."""
import pytest
import torch

from oracle import tree as ref
from test_gpu_tree import LINEAR_REL, rel
from tree_helpers import linear_inputs, run_linear

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,dk,dv", [("bf16", 128, 128), ("f32", 128, 128), ("bf16", 64, 64),
                                         ("f32", 64, 128)])
@pytest.mark.parametrize("N", [12, 30, 64])
@pytest.mark.parametrize("gate", [-200.0, -1e5, -1e9, float(torch.finfo(torch.float32).min)])
def test_linear_after_a_gate_of_zero(gate, N, dtype, dk, dv):
    s = linear_inputs(85, 4, N, 2, 4, dk, dv, dtype, [N, N, N - 1, N // 2], "mixed")
    resets = torch.zeros(4, N, dtype=torch.bool)
    resets[0, 0] = resets[1, [2, 5]] = resets[2, 3] = True
    resets[3, 1:5] = True
    s.log_decay[resets.cuda()] = gate
    s.log_decay[1, :, 1] = -0.25  # a head that resets nowhere
    out = run_linear(s)
    want = ref.tree_linear(*(x.cpu() for x in (s.q, s.k, s.v, s.log_decay, s.beta, s.state_pool,
                                               s.slot, s.parent, s.node_len)))
    for r in range(4):
        n = int(s.node_len[r])
        paths = ref.paths(s.parent[r].tolist(), n)
        K = max(sum(bool(resets[r, i]) for i in line) for line in paths)
        more = 2.0 ** -22 * 104 * K / 3
        assert rel(out[r, :n], want[r, :n]) <= LINEAR_REL[dtype] + more
