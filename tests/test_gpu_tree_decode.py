"""The tree calls as examples/tree_decode.py uses them: drafted trees decode the tokens that one
token a round decodes."""
import importlib.util
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu

_at = Path(__file__).resolve().parents[1] / "examples" / "tree_decode.py"
_spec = importlib.util.spec_from_file_location("tree_decode", _at)
tree_decode = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(tree_decode)


def prompt(R, n, seed=3):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randint(0, 512, (R, n), dtype=torch.int32, device="cuda", generator=g)


@pytest.mark.parametrize("layers,length", [("llsl", 21), ("ss", 1), ("l", 40)])
def test_trees_decode_what_single_tokens_decode(layers, length):
    R, rounds = 5, 12
    tokens = prompt(R, length)
    trees, rate = tree_decode.HybridDecoder(R, layers=layers).decode(tokens, rounds)
    one, _ = tree_decode.HybridDecoder(R, layers=layers).decode(tokens, 3 * rounds, plain=True)
    assert rate > 1.2  # the drafter is accepted now and then, or nothing was tested
    for a, b in zip(trees, one):
        assert a == b[:len(a)]


def test_bf16_rounds_stay_sound():
    new, rate = tree_decode.HybridDecoder(4, dtype="bf16").decode(prompt(4, 9), 10)
    assert all(0 <= t < 512 for line in new for t in line) and rate >= 1.0
