"""One weight for all groups where there is one group, the whole row: shared_weight = 1 with group = 0
or group = width, rows of one CTA and of a cluster.

Tolerances: steps_helpers.Y_REL, H_REL and GRAD_REL, and half a step of the output's type."""
import pytest
import torch

from steps_helpers import bits, check_norm, check_norm_bwd, norm_inputs, run_norm, run_norm_bwd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gate,pre", [("none", True), ("silu", True), ("sigmoid", False)])
@pytest.mark.parametrize("group", ["none", "width"])
@pytest.mark.parametrize("T,W", [(700, 256), (5, 4104), (300, 6016), (9, 8192), (3, 8200),
                                 (170, 16384)])
def test_shared_weight_over_whole_rows(T, W, group, gate, pre, dtype):
    s = norm_inputs(40 + W, T, W, dtype, group=0 if group == "none" else W, gate=gate, pre=pre)
    want_y, want_h = run_norm(s)
    want = run_norm_bwd(s)
    s.desc.shared_weight, s.how["shared"] = 1, True
    y, h = run_norm(s)
    check_norm(s, y, h)
    got = run_norm_bwd(s)
    check_norm_bwd(s, got)
    # G = W entries either way: the same weight, the same call
    assert torch.equal(bits(y), bits(want_y)) and (h is None or torch.equal(bits(h), bits(want_h)))
    for name, x in got.items():
        assert x is None or torch.equal(bits(x), bits(want[name])), name
