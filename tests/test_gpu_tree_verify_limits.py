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
