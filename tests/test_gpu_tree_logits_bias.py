"""Bias lists of the logits call whose bits its lanes set for each other: many to a word, one to a word,
lists that end within a round of the warp, chunks with few of them and with all.

In fp32 without penalties a biased token is the rounded sum of its logit and its bias, which a
reference in fp32 gives bit for bit; the other tokens stay as they are."""
import random

import pytest
import torch

from steps_helpers import bits, logits_inputs, run_logits, whole
from tree_helpers import FAR

pytestmark = pytest.mark.gpu

LENS = [0, 1, 2, 31, 32, 33, 63, 64, 65, 97, 300]


def tokens(kind, n, V, rng):
    """n different tokens."""
    if kind == "side_by_side":
        first = rng.randrange(V - n + 1)
        return list(range(first, first + n))
    if kind == "a_word_each":
        step = min(32, V // max(n, 1))
        first = rng.randrange(V - step * n + 1)
        return [first + step * i for i in range(n)][::-1]
    if kind == "ends":  # the first and last tokens in turn
        return [i // 2 if i % 2 == 0 else V - 1 - i // 2 for i in range(n)]
    return rng.sample(range(V), n)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kind", ["side_by_side", "a_word_each", "ends", "anywhere"])
@pytest.mark.parametrize("N,V", [(1, 301), (1, 40000), (2, 5001), (5, 3000)])
def test_every_bias_meets_its_token(N, V, kind, in_place):
    R, rng = len(LENS), random.Random(V + N)
    s = logits_inputs(80, R, N, V, "f32", [N] * R, history=0, bias=0, masked=None, tree=False,
                      penalties=False)
    lists = [tokens(kind, n, V, rng) for n in LENS]
    s.desc.max_bias = max(LENS)
    s.bias_len = whole(LENS)
    s.bias_token = whole([x + [FAR] * (max(LENS) - len(x)) for x in lists])
    g = torch.Generator(device="cuda")
    g.manual_seed(V)
    s.bias_value = torch.randn(R, max(LENS), generator=g, device="cuda")
    want = s.logits.clone()
    for r, x in enumerate(lists):
        if x:
            want[r][:, x] += s.bias_value[r, :len(x)]
    first = s.logits.clone()
    for _ in range(10):
        s.logits.copy_(first)
        assert torch.equal(bits(run_logits(s, in_place=in_place)), bits(want))
