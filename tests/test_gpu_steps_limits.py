"""Block norms at the largest number of rows that a descriptor can name, and what their gradients take of
a workspace."""
import pytest
import torch

from paper_2606_01774_gb300 import flare
from steps_helpers import GRAD_REL, bits, norm_inputs, run_norm, run_norm_bwd

pytestmark = pytest.mark.gpu


def test_as_many_rows_as_an_int_counts():
    """2^31 - 1 rows of 8, zeros but for the last five, in place."""
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 120 GiB of device memory")
    T, W = 2 ** 31 - 1, 8
    s = norm_inputs(90, 5, W, residual=False, pre=False)
    want, grad = run_norm(s)[0], run_norm_bwd(s)
    d = flare.block_norm_desc(T, W, flare.FLARE_DT_BF16, pre_norm=0)
    x, dy = (torch.zeros(T, W, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x[-5:] = s.x
    dy[-5:] = s.dy
    dw = torch.empty(W, device="cuda")
    ws = torch.empty(flare.flare_block_norm_bwd_workspace_size(d), dtype=torch.uint8, device="cuda")
    flare.check(flare.flare_block_norm_bwd(d, x, None, None, s.post_weight, None, dy, None, dy, None,
                                           None, dw, None, ws, ws.numel()))
    flare.check(flare.flare_block_norm(d, x, None, None, s.post_weight, None, x, None))
    for got, w in ((x, want), (dy, grad["dx"])):
        assert torch.equal(bits(got[-5:]), bits(w))
        assert float(got[:-5].amax()) == 0 and float(got[:-5].amin()) == 0
    # five terms by other teams than before: each sum is off by GRAD_REL of their size at most
    n = s.x.double()
    size = (s.dy.double() * n / (n.square().mean(1, keepdim=True) + 1e-6).sqrt()).abs().sum(0)
    off = (dw.double() - grad["dpost_weight"].double()).abs()
    assert bool((off <= 2 * GRAD_REL * size).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,W,how", [
    (1, 128, {}), (189, 128, {}), (189, 512, dict(gate="silu")), (1924, 128, dict(pre=False)),
    (444, 1024, {}), (2000, 2048, dict(gate="silu", group=128, shared=True, pre=False)),
    (700, 4104, {}), (90, 6400, dict(gate="silu", group=128, shared=True)), (300, 16384, {})])
def test_a_workspace_of_more_rows(T, W, how, dtype):
    """Calls stay within what their own number of rows needs, and take a workspace of more rows."""
    s = norm_inputs(91 + W, T, W, dtype, **how)
    want = run_norm_bwd(s)
    need = flare.flare_block_norm_bwd_workspace_size(s.desc)
    s.desc.num_tokens = 1 << 20
    more = flare.flare_block_norm_bwd_workspace_size(s.desc)
    s.desc.num_tokens = T
    assert more >= need
    ws = torch.full((more + 4096,), 0x55, dtype=torch.uint8, device="cuda")
    new = {k: None if x is None else torch.empty_like(x) for k, x in want.items()}
    flare.check(flare.flare_block_norm_bwd(s.desc, s.x, s.gate, s.residual, s.post_weight,
                                           s.pre_weight, s.dy, s.dh, *new.values(), ws, more))
    for k, x in new.items():
        assert x is None or torch.equal(bits(x), bits(want[k])), k
    assert bool((ws[need:] == 0x55).all())
