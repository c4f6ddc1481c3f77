"""Verification at the limits of its inputs, against the fp64 definition: maxima one ulp apart,
logits at the type's lowest value, low temperatures, and drafts that hold nearly all of a row.

Tolerances, from the arithmetic and before any run.  A log-probability is a difference of logits
(exact or rounded once), a product with the inverse temperature (rounded once) and an fp32
log-sum (5e-5 absolute is ten times what 2^17 terms summed pairwise and in chunks can lose):
5e-5 + 2^-22 |logp|.  Decisions are compared where the fp64 margin exceeds 1e-4, unless a test
says otherwise."""
import numpy as np
import pytest
import torch

from oracle import tree as ref
from paper_2606_01774_gb300 import flare
from tree_helpers import DTYPES, run_verify, verify_inputs

pytestmark = pytest.mark.gpu

F32_MAX = float(torch.finfo(torch.float32).max)


def check_verify(s, margin=1e-4, allowed=0.05):
    """Against the definition; log-probabilities past fp32's range are -inf."""
    got = run_verify(s)
    cpu = [None if x is None else x.cpu() for x in (s.logits, s.draft_probs, s.token, s.parent,
                                                    s.node_len, s.uniform, s.noise)]
    want = ref.tree_verify(*cpu, s.greedy, s.inv_temp)
    sure = want["margin"] > margin
    assert (~sure).mean() <= allowed
    for k in ("path", "path_len", "next_token"):
        assert np.array_equal(got[k].cpu().numpy()[sure], want[k][sure]), k
    have, logp = got["node_logp"].double().cpu().numpy(), want["node_logp"]
    out = logp < -F32_MAX * (1 - 2.0 ** -22)
    assert (have[out] <= -F32_MAX * (1 - 2.0 ** -20)).all()
    err = np.abs(have[~out] - logp[~out])
    assert (err <= 5e-5 + 2.0 ** -22 * np.abs(logp[~out])).all(), err.max()
    return got, want


def _colliding(x):
    """fp32 a, b = the next float after a, from x up, whose products with log2 e round alike."""
    a, c = np.float32(x), np.float32(1.4426950408889634)
    while a * c != np.nextafter(a, np.float32(np.inf)) * c:
        a = np.nextafter(a, np.float32(np.inf))
    return float(a), float(np.nextafter(a, np.float32(np.inf)))


@pytest.mark.parametrize("low,high", [(5, 900), (5, 9000), (4097, 19999), (0, 3), (2047, 2048)])
@pytest.mark.parametrize("x", [1.4, 3.0, 12.7])
def test_greedy_tells_maxima_one_ulp_apart(x, low, high):
    """The greater of two neighbouring floats wins at the higher index, in another thread or chunk,
    on a row with a child and on one without; the lower index among equals."""
    a, b = _colliding(x)
    s = verify_inputs(90, 3, 2, 20000, "f32", "top", greedy=True, nodes=[2, 1, 2])
    s.logits.clamp_(max=1.0)
    s.logits[:, :, low], s.logits[:, :, high] = a, b
    s.logits[2, :, low] = b
    s.token[0, 1], s.token[2, 1] = high, low
    got, _ = check_verify(s)
    assert got["path_len"].tolist() == [2, 1, 2]
    assert got["next_token"].tolist() == [high, high, low]


LOWEST_RUNS = {"head": [(0, 3001)], "tail": [(5003, 9001)], "chunks": [(2048, 8192)],
               "all but a few": [(0, 4000), (4003, 8990)], "every second 64": [
                   (a, a + 64) for a in range(0, 9001, 128)]}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("drafts,greedy", [("sampled", False), ("top", False), ("top", True)])
@pytest.mark.parametrize("inv_temp", [0.5, 1.0, 3.0])
@pytest.mark.parametrize("run", sorted(LOWEST_RUNS))
def test_runs_of_the_lowest_finite_logit(run, inv_temp, drafts, greedy, dtype):
    """Tokens ruled out by the type's lowest value in long runs, as masks leave them."""
    s = verify_inputs(91, 12, 6, 9001, dtype, drafts, greedy, inv_temp, nodes=[6 - r % 3 for r in
                                                                              range(12)])
    for a, b in LOWEST_RUNS[run]:
        s.logits[:, :, a:b] = torch.finfo(DTYPES[dtype][0]).min
    check_verify(s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("drafts,greedy", [("sampled", False), ("top", False), ("top", True)])
def test_rows_of_nothing_but_the_lowest_finite_logit(drafts, greedy, dtype):
    """Every token alike: the first when greedy, else the uniform distribution."""
    s = verify_inputs(92, 16, 3, 3001, dtype, drafts, greedy, nodes=[3] * 16, shape="star")
    s.logits[:, 0] = torch.finfo(DTYPES[dtype][0]).min
    s.token[:, 1:] = s.token[:, 1:].clamp(min=1)
    if s.draft_probs is not None:
        s.uniform.fill_(0.999)  # rejected mostly: the residual of a uniform row decides
    got, _ = check_verify(s)
    if greedy:
        assert got["next_token"].tolist() == [0] * 16


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inv_temp", [2.0 ** -20, 100.0, 1e4, 2.9e38])
@pytest.mark.parametrize("drafts", ["sampled", "top"])
def test_temperatures_far_from_one_on_rows_with_children(drafts, inv_temp, dtype):
    """Logits near 40 under inverse temperatures whose product with them has no digits left for
    their differences."""
    s = verify_inputs(93, 20, 5, 2500, dtype, drafts, False, 1.0, nodes=[5] * 20, shape="star")
    s.logits += 40.0
    s.inv_temp = s.desc.inv_temperature = float(np.float32(inv_temp))
    s.token[:, 1] = s.logits[:, 0].argmax(-1).int()
    got, want = check_verify(s, allowed=1.0)
    assert np.array_equal(got["path"].cpu().numpy()[want["margin"] > 1e-4],
                          want["path"][want["margin"] > 1e-4])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inv_temp", [1.0, 1e4, 1e7, 2.9e38])
def test_next_token_among_equal_logits_at_low_temperatures(inv_temp, dtype):
    """Twenty tokens share the greatest logit: the noise alone chooses among them, on a row without
    children, however low the temperature."""
    s = verify_inputs(94, 64, 2, 5003, dtype, "top", False, inv_temp, nodes=[1 + r % 2 for r in
                                                                           range(64)])
    s.inv_temp = s.desc.inv_temperature = float(np.float32(inv_temp))
    s.logits.clamp_(max=10.0)
    s.logits[:, :, 7::251] = 41.5
    got, _ = check_verify(s)
    assert bool((got["next_token"] % 251 == 7).all())
    assert len(set(got["next_token"].tolist())) > 10


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", ["lowest", "greatest"])
@pytest.mark.parametrize("inv_temp", [0.5, 1.0, 2.0])
def test_next_token_from_rows_at_the_ends_of_the_range(inv_temp, value, dtype):
    """A row without children that holds one finite value throughout is a uniform distribution."""
    s = verify_inputs(95, 32, 1, 4001, dtype, "top", False, inv_temp, nodes=[1] * 32)
    info = torch.finfo(DTYPES[dtype][0])
    s.logits.fill_(info.min if value == "lowest" else info.max)
    s.logits[:, :, 1::2] = float("-inf")
    got, _ = check_verify(s)
    assert bool((got["next_token"] % 2 == 0).all())


@pytest.mark.parametrize("rest", [1e-5, 2e-6, 1e-6, 6e-7, 4e-7])
@pytest.mark.parametrize("siblings", [2, 3])
def test_fixed_drafts_that_hold_nearly_all_of_the_mass(siblings, rest):
    """The first sibling holds all but `rest` of the row and is rejected by the greatest uniform
    below one; the second is accepted with its share of the rest, to 5 % here.  (With three, the
    second in turn holds all but `rest` of that.)  1 - p from fp32's p knows the rest to 1e-7.
    Every decision's fp64 margin exceeds 2.4e-7, twice what an fp32 p near one is off by."""
    R, V = 64, 1000
    s = verify_inputs(96, R, 1 + siblings, V, "f32", "top", False, 1.0, nodes=[1 + siblings] * R,
                      shape="star")
    s.logits[:] = -1e4
    x = torch.full((R, V), -1e4, dtype=torch.float64)
    spread = torch.rand(R, V - 10, dtype=torch.float64, generator=torch.Generator().manual_seed(1))
    tail = rest * (1 if siblings == 2 else 1e-3)
    share = 0.5 * tail  # the last sibling's half of the tail, the rest spread over the row
    x[:, 10:] = torch.log(share * spread / spread.sum(1, keepdim=True))
    x[:, 0] = np.log1p(-rest)
    if siblings == 3:
        x[:, 1] = np.log(rest - tail)
    x[:, siblings - 1] = np.log(share)
    s.logits[:, 0] = (x + 80.0 - 0.37 * torch.arange(R, dtype=torch.float64)[:, None]).float().cuda()
    s.token[:, 1:] = torch.arange(siblings, dtype=torch.int32)
    s.uniform[:, 1:siblings] = 1.0 - 2.0 ** -24
    s.uniform[0::2, siblings] = 0.475
    s.uniform[1::2, siblings] = 0.525
    got, want = check_verify(s, margin=0.0 if siblings == 3 else 2.4e-7, allowed=0.0)
    if siblings == 2:
        assert got["path_len"].tolist() == [2, 1] * (R // 2)
