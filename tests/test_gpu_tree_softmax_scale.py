"""Tree softmax with a logit scale of zero: the mean over what a node sees.

Tolerances as in test_gpu_tree.py (uniform probabilities round no worse than others)."""
import numpy as np
import pytest
import torch

from oracle import tree as ref
from test_gpu_tree import LSE_ABS, SOFTMAX_REL, rel
from tree_helpers import run_softmax, softmax_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-44, 1e-30])
@pytest.mark.parametrize("N,Hq,Hkv,D,page,prefix", [
    (9, 4, 2, 64, 16, [0, 70, 64, 130]),
    (40, 8, 1, 128, 32, [33, 0, 200, 1]),   # more than one row tile
    (5, 6, 2, 256, 64, [0, 65, 3000, 7]),
])
def test_scale_of_zero_is_the_mean_of_the_visible_values(N, Hq, Hkv, D, page, prefix, scale, dtype):
    s = softmax_inputs(95, len(prefix), N, Hq, Hkv, D, page, prefix, dtype,
                       [N, max(1, N // 2), 1, N])
    s.desc.scale = scale
    out, lse = run_softmax(s)
    want, want_lse = ref.tree_softmax(*(x.cpu() for x in (s.q, s.k_blk, s.v_blk, s.k_pool, s.v_pool,
                                                          s.page_table, s.prefix_len, s.parent,
                                                          s.node_len)), scale=0.0)
    live = np.arange(N) < s.node_len.cpu().numpy()[:, None]
    assert rel(out[torch.from_numpy(live).cuda()], want[live]) <= SOFTMAX_REL[dtype]
    assert np.abs(lse.double().cpu().numpy()[live] - want_lse[live]).max() <= LSE_ABS
