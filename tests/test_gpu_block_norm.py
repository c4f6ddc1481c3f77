"""Block norms, gates and residuals and their gradients, against their fp64 definition.

Tolerances: steps_helpers.Y_REL, H_REL and GRAD_REL, and half a step of the output's type."""
import pytest
import torch

from paper_2606_01774_gb300 import flare
from steps_helpers import (bits, check_norm, check_norm_bwd, norm_inputs, run_norm, run_norm_bwd)

pytestmark = pytest.mark.gpu

CASES = [
    dict(T=1, W=2048), dict(T=64, W=4096, gate="sigmoid", x_pad=64, gate_pad=128),
    dict(T=3, W=8), dict(T=5, W=264, gate="silu"), dict(T=200, W=512, residual=False),
    dict(T=33, W=2048, group=128, shared=True, gate="silu", residual=False, pre=False, x_pad=8),
    dict(T=9, W=768, group=256, gate="sigmoid"), dict(T=17, W=64, group=64, shared=True),
    dict(T=11, W=1088, group=64, shared=True, gate="silu", alpha=-0.5),
    dict(T=7, W=16384, gate="silu"), dict(T=6, W=8200), dict(T=4, W=2056, gate="none", gated=True),
    dict(T=1200, W=640, post=False, residual=True, alpha=0.25),
    dict(T=10, W=1000, post=False, residual=False, weights=False),
    dict(T=10, W=1000, pre=False, weights=False), dict(T=3, W=5000, eps=0.5, scale=30.0),
    dict(T=2000, W=128, group=128, residual=False, gate="silu", shared=True),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_matches_the_definition(case, dtype):
    s = norm_inputs(1 + case["W"], dtype=dtype, **case)
    y, h = run_norm(s)
    check_norm(s, y, h)
    if s.how["pre"]:
        assert torch.equal(bits(run_norm(s, y=False)[1]), bits(h))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_gradients_match_the_definition(case, dtype):
    s = norm_inputs(2 + case["W"], dtype=dtype, **case)
    got = run_norm_bwd(s)
    check_norm_bwd(s, got)
    again = run_norm_bwd(s)
    for name, x in got.items():  # a fixed order of sums
        assert x is None or torch.equal(bits(x), bits(again[name])), name
    bare = run_norm_bwd(s, weights=False, dresidual=False)
    assert torch.equal(bits(bare["dx"]), bits(got["dx"]))


MORE = [
    dict(T=700, W=6400, group=128, gate="silu", shared=True), dict(T=500, W=7424, gate="sigmoid"),
    dict(T=1500, W=4096), dict(T=400, W=6144), dict(T=5000, W=2048, gate="silu"),
    dict(T=333, W=5632, group=256, post=True, residual=False),
    dict(T=2500, W=1360, gate="silu", residual=False), dict(T=3001, W=512, group=64, pre=False),
    dict(T=160, W=16384), dict(T=310, W=9000, gate="silu", pre=False, residual=False),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", MORE, ids=str)
def test_several_rows_to_every_team(case, dtype):
    s = norm_inputs(30 + case["W"], dtype=dtype, **case)
    check_norm(s, *run_norm(s))
    check_norm_bwd(s, run_norm_bwd(s))


def test_gradients_in_their_inputs_place():
    """dx, dgate and dresidual over x, gate and residual, slices of one projection; over dy and dh."""
    s = norm_inputs(20, 900, 1024, gate="silu", group=128)
    want = run_norm_bwd(s)
    both = torch.cat([s.x, s.gate], 1)
    x, gate = both.split(1024, 1)
    d = s.desc
    d.x_stride = d.gate_stride = 2048
    ws = torch.empty(flare.flare_block_norm_bwd_workspace_size(d), dtype=torch.uint8, device="cuda")
    res = s.residual.clone()
    w = [torch.empty_like(s.post_weight), torch.empty_like(s.pre_weight)]
    flare.check(flare.flare_block_norm_bwd(d, x, gate, res, s.post_weight, s.pre_weight, s.dy, s.dh,
                                           x, gate, res, *w, ws, ws.numel()))
    for a, b in ((x, "dx"), (gate, "dgate"), (res, "dresidual"), (w[0], "dpost_weight"),
                 (w[1], "dpre_weight")):
        assert torch.equal(bits(a), bits(want[b])), b
    d.x_stride = d.gate_stride = 0
    dy, dh = s.dy.clone(), s.dh.clone()
    dgate = torch.empty_like(s.gate)
    flare.check(flare.flare_block_norm_bwd(d, s.x, s.gate, s.residual, s.post_weight, s.pre_weight,
                                           dy, dh, dh, dgate, dy, None, None, None, 0))
    assert torch.equal(bits(dh), bits(want["dx"])) and torch.equal(bits(dy), bits(want["dresidual"]))


def test_no_gradient_at_y():
    s = norm_inputs(3, 20, 512, gate="silu", dy=False)
    check_norm_bwd(s, run_norm_bwd(s))


def test_gradients_against_differences():
    """Central differences of the kernel's own forward in fp32: the loss is linear in dy, dh, the
    step 2^-6, so each difference is off by its third derivative (step^2, some 2^-12 of the slope)
    and by fp32 sums of 3 x 256 products near one over the step (3 x 256 x 2^-24 x 2^6 at most)."""
    s = norm_inputs(4, 3, 256, "f32", gate="silu", group=64, shared=True, eps=1e-2)
    grad = run_norm_bwd(s)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)

    def loss():
        y, h = run_norm(s)
        return (y.double() * s.dy.double()).sum() + (h.double() * s.dh.double()).sum()

    step = 2.0 ** -6
    for name in ("x", "gate", "residual", "post_weight", "pre_weight"):
        t = getattr(s, name)
        d = torch.randn(t.shape, generator=g, device="cuda")
        d /= d.norm()
        keep = t.clone()
        t.copy_(keep + step * d)
        up = loss()
        t.copy_(keep - step * d)
        down = loss()
        t.copy_(keep)
        slope = (grad["d" + name].double() * d.double()).sum()
        size = grad["d" + name].double().norm()
        assert abs((up - down) / (2 * step) - slope) < 2.0 ** -10 * size + 768 * 2.0 ** -18, name


def test_in_place():
    s = norm_inputs(6, 40, 1024, gate="sigmoid")
    y, h = run_norm(s)
    res, x = s.residual.clone(), s.x.clone()
    flare.check(flare.flare_block_norm(s.desc, x, s.gate, res, s.post_weight, s.pre_weight, res, x))
    assert torch.equal(bits(res), bits(y)) and torch.equal(bits(x), bits(h))
    grad = run_norm_bwd(s)
    need = flare.flare_block_norm_bwd_workspace_size(s.desc)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    dy, dx, dg = s.dy.clone(), torch.empty_like(s.x), torch.empty_like(s.gate)
    w = [torch.empty_like(s.post_weight), torch.empty_like(s.pre_weight)]
    flare.check(flare.flare_block_norm_bwd(s.desc, s.x, s.gate, s.residual, s.post_weight,
                                           s.pre_weight, dy, s.dh, dx, dg, dy, *w, ws, need))
    for a, b in ((dy, "dresidual"), (dx, "dx"), (dg, "dgate"), (w[0], "dpost_weight")):
        assert torch.equal(bits(a), bits(grad[b])), b


def test_far_gates_and_zero_rows():
    """Gates far out neither overflow nor make NaN; a row of zeros gives zeros."""
    s = norm_inputs(7, 6, 512, "f32", gate="silu", eps=1e-5)
    s.gate[0], s.gate[1] = 200.0, -200.0
    s.gate[2], s.gate[3] = 3e38, -3e38
    s.x[4] = 0
    s.residual[4] = 0
    s.gate[2].fill_(1e4)
    y, h = run_norm(s)
    assert bool(torch.isfinite(y).all() and torch.isfinite(h).all())
    assert bool((y[4] == 0).all() and (h[4] == 0).all())
    got = run_norm_bwd(s)
    for name, x in got.items():
        assert bool(torch.isfinite(x).all()), name
    keep = [0, 1, 3, 4, 5]
    assert bool((got["dgate"][[1, 3]] == 0).all())
    sig = norm_inputs(8, 4, 64, "f32", gate="sigmoid", residual=False, pre=False)
    sig.gate[0], sig.gate[1] = float("inf"), float("-inf")
    y, _ = run_norm(sig)
    assert bool(torch.isfinite(y[keep[:2]]).all()) and bool((y[1] == 0).all())
    sig.gate[0] = float("nan")
    assert bool(run_norm(sig)[0][0].isnan().all())


def test_no_rows():
    s = norm_inputs(9, 0, 256)
    run_norm(s)
    got = run_norm_bwd(s)
    assert bool((got["dpost_weight"] == 0).all() and (got["dpre_weight"] == 0).all())


def test_rows_beyond_32_bits():
    if torch.cuda.mem_get_info()[0] < 50 << 30:
        pytest.skip("needs 50 GiB of device memory")
    T, W = 270_000, 8192
    assert T * W > 1 << 31
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.zeros(T, W, dtype=torch.bfloat16, device="cuda")
    s = norm_inputs(10, 5, W, residual=False)
    x[-5:] = s.x
    d = flare.block_norm_desc(T, W, flare.FLARE_DT_BF16)
    y, h = torch.empty_like(x), torch.empty_like(x)
    flare.check(flare.flare_block_norm(d, x, None, None, s.post_weight, s.pre_weight, y, h))
    want = run_norm(s)
    assert torch.equal(bits(y[-5:]), bits(want[0])) and torch.equal(bits(h[-5:]), bits(want[1]))
    grad = run_norm_bwd(s)
    dy, dh = y, h  # their memory again
    dy.zero_()
    dh.zero_()
    dy[-5:], dh[-5:] = s.dy, s.dh
    dx = torch.empty_like(x)
    ws = torch.empty(flare.flare_block_norm_bwd_workspace_size(d), dtype=torch.uint8, device="cuda")
    flare.check(flare.flare_block_norm_bwd(d, x, None, None, s.post_weight, s.pre_weight, dy, dh,
                                           dx, None, None, None, None, ws, ws.numel()))
    assert torch.equal(bits(dx[-5:]), bits(grad["dx"])) and int((dx[:-5] != 0).sum()) == 0
