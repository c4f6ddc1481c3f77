"""Penalties, biases and masks on a tree's logits, against their fp64 definition.

Tolerances: steps_helpers.LOGITS_REL and half a step of the logits' type."""
import pytest
import torch

from paper_2606_01774_gb300 import flare
from steps_helpers import (MARK, bits, check_logits, logits_inputs, pack, run_logits, whole)
from tree_helpers import FAR

pytestmark = pytest.mark.gpu


def check_all(s):
    """Out of place against the definition, unused rows marked; in place the same bits."""
    out = run_logits(s)
    check_logits(s, out)
    dead = torch.arange(s.N, device="cuda") >= whole(s.nodes)[:, None]
    assert bool((out[dead] == MARK).all())
    given = s.logits.clone()
    run_logits(s, in_place=True)
    assert torch.equal(bits(s.logits[~dead]), bits(out[~dead]))
    assert bool(s.logits[dead].isnan().all())
    s.logits.copy_(given)
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,N,V,nodes", [
    (1, 1, 1, None), (1, 1, 7, [1]), (3, 4, 33, [4, 0, 2]), (2, 5, 1000, [5, 3]),
    (1, 1, 50257, [1]), (2, 13, 4099, [13, 6]), (40, 2, 515, None), (1, 64, 9001, [64]),
    (5, 16, 8192, [16, 1, 9, 0, 16])])
def test_matches_the_definition(R, N, V, nodes, dtype):
    check_all(logits_inputs(R + N + V, R, N, V, dtype, nodes))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("without", ["history", "tree", "penalties", "bias", "mask", "all"])
def test_each_part_may_be_missing(without, dtype):
    kw = dict(history=0) if without == "history" else dict(bias=0) if without == "bias" else \
        dict(masked=None) if without == "mask" else dict(tree=False) if without == "tree" else \
        dict(penalties=False) if without == "penalties" else \
        dict(history=0, bias=0, masked=None, tree=False, penalties=False)
    s = logits_inputs(50, 4, 6, 2500, dtype, [6, 2, 0, 5], **kw)
    out = check_all(s)
    if without == "all":
        assert torch.equal(bits(out[0]), bits(s.logits[0]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,N,V,nodes", [
    (64, 1, 128000, None), (3, 2, 50264, [2, 1, 2]), (3, 2, 1004, [2, 2, 0]),
    (60, 3, 120004, [3, 0, 1, 2] + [0] * 56), (5, 7, 30004, None), (150, 1, 66000, None)])
def test_few_rows_and_large_chunks(R, N, V, nodes, dtype):
    check_all(logits_inputs(R + N + V, R, N, V, dtype, nodes))


@pytest.mark.parametrize("H", [32766, 32767, 32768, 70000])
@pytest.mark.parametrize("x", [6, 7])
def test_counts_up_to_their_last_bit(H, x):
    """A token all through a history that is as long as counts of 16 bits allow, and longer, over a
    vocabulary that makes them worth while; the next token in the prompt alone."""
    R, V = 150, 66000
    s = logits_inputs(70, R, 1, V, "f32", [1] * R, history=1, bias=0, masked=None)
    s.text = [[x ^ 1, x ^ 1] + [x] * (H - 2)] + [[x]] * (R - 1)
    s.start = [2] + [0] * (R - 1)
    s.history = torch.full((R, H), FAR, dtype=torch.int32, device="cuda")
    s.history[:, 0] = x
    s.history[0] = whole(s.text[0])
    s.history_len, s.output_start = whole([H] + [1] * (R - 1)), whole(s.start)
    s.desc.max_history = H
    check_all(s)


def test_no_node_lengths_no_starts():
    s = logits_inputs(51, 3, 2, 700, "f32", [2, 2, 2], tree=False)
    s.node_len = s.output_start = None
    s.start = [0, 0, 0]
    check_all(s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_off_every_grid(dtype):
    """Logits that start between 16-byte boundaries, and outputs on another grid than theirs."""
    for offset in (1, 3, 7):
        s = logits_inputs(52 + offset, 2, 3, 1001, dtype, [3, 2], offset=offset)
        out = check_all(s)
        raw = torch.full((2 * 3 * 1001 + 8,), MARK, dtype=s.logits.dtype, device="cuda")
        other = raw[5:5 + 2 * 3 * 1001].view(2, 3, 1001)
        run_logits(s, other)
        assert torch.equal(bits(other), bits(out))
        assert bool((raw[:5] == MARK).all() and (raw[-3:] == MARK).all())


def test_long_histories_and_many_biases():
    s = logits_inputs(60, 3, 4, 6000, "f32", [4, 4, 1], history=20000, bias=300)
    check_all(s)


def test_everything_repeats():
    """One token throughout: in the prompt, the output, every node and every bias."""
    s = logits_inputs(61, 1, 8, 300, "f32", [8], history=64, bias=6, masked=0.0)
    s.text, s.start = [[299] * 64], [10]
    s.history, s.history_len, s.output_start = whole(s.text), whole([64]), whole([10])
    s.token = whole([[299] * 8])
    s.bias = [[(299, 0.5 + i) for i in range(6)]]
    s.bias_token, s.bias_len = whole([[299] * 6]), whole([6])
    s.bias_value = torch.tensor([[0.5 + i for i in range(6)]], device="cuda")
    check_all(s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_a_token_and_what_masks_hide(dtype):
    s = logits_inputs(62, 2, 3, 900, dtype, [3, 3], masked=0.5)
    s.allowed[0, 1] = False
    s.allowed[1, 2] = False
    s.allowed[1, 2, 899] = True
    s.mask = pack(s.allowed)
    hidden = ~s.allowed
    low = torch.finfo(s.logits.dtype).min
    for value in (float("nan"), float("inf"), float("-inf"), low):
        s.logits.masked_fill_(hidden, value)
        out = check_all(s)
        assert bool((out[hidden] == float("-inf")).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ends_of_the_range_where_nothing_is_hidden(dtype):
    """-inf stays, +inf stays, a NaN stays; the type's ends may pass over into infinities."""
    s = logits_inputs(63, 1, 2, 640, dtype, [2], masked=None)
    top = torch.finfo(s.logits.dtype).max
    for i, v in enumerate((float("nan"), float("inf"), float("-inf"), 0.0, -0.0, 1e-30)):
        s.logits[:, :, i::8] = v
    check_all(s)
    s.logits[:, :, ::3] = top
    s.logits[:, :, 1::3] = -top
    s.repetition = whole([1]).float()
    s.presence = s.frequency = None
    s.bias = s.bias_token = s.bias_value = s.bias_len = None
    out = run_logits(s)
    # by value: -0 + 0 is 0
    assert bool(((out == s.logits) | (out.isnan() & s.logits.isnan())).all())


def test_bans_by_bias():
    s = logits_inputs(64, 1, 2, 256, "bf16", [2], bias=4)
    s.bias = [[(3, float("-inf")), (9, 1.0), (3, 2.0)]]
    s.bias_token, s.bias_len = whole([[3, 9, 3, FAR]]), whole([3])
    s.bias_value = torch.tensor([[float("-inf"), 1.0, 2.0, float("nan")]], device="cuda")
    assert bool((check_all(s)[:, :, 3] == float("-inf")).all())


def test_a_bad_request_is_skipped():
    s = logits_inputs(65, 3, 4, 5000, "f32", [4, 4, 2], history=40, bias=6)
    good = run_logits(s)

    def check(expect, r, name, change):
        old = getattr(s, name)
        new = old.clone()
        new[r] = change(new[r])
        setattr(s, name, new)
        out = run_logits(s, expect=expect)
        setattr(s, name, old)
        assert bool((out[r] == MARK).all())
        rest = [i for i in range(3) if i != r]
        assert torch.equal(bits(out[rest]), bits(good[rest]))

    def put(i, v):
        def f(row):
            row = row.clone()
            row[i] = v
            return row
        return f

    n = max(range(3), key=lambda r: len(s.text[r]))
    assert len(s.text[n]) > 0
    hist, pen, tree = (flare.FLARE_DEV_BAD_HISTORY, flare.FLARE_DEV_BAD_PENALTY,
                       flare.FLARE_DEV_BAD_TREE)
    for v in (-1, 5000, FAR):
        check(hist, n, "history", put(len(s.text[n]) - 1, v))
    for name in ("history_len", "output_start"):
        check(hist, 1, name, lambda x: x * 0 + 41)
        check(hist, 1, name, lambda x: x * 0 - 1)
    for v in (-1, 7):
        check(hist, 2, "bias_len", lambda x: x * 0 + v)
    s.bias_len[0], s.bias_token[0, :2], s.bias_value[0, :2] = 2, 1, 0.5
    good = run_logits(s)
    check(hist, 0, "bias_token", put(1, 5000))
    for v in (0.0, -1.0, float("inf"), float("nan"), 1e-40):
        check(pen, 1, "repetition", lambda x: x * 0 + v if v == v else x * v)
    for name in ("presence", "frequency"):
        for v in (float("inf"), float("nan")):
            check(pen, 2, name, lambda x: torch.full_like(x, v))
    check(tree, 0, "node_len", lambda x: x * 0 + 5)
    check(tree, 0, "node_len", lambda x: x * 0 - 1)
    check(tree, 2, "token", put(1, 5000))
    check(tree, 2, "token", put(0, -1))
    check(tree, 1, "parent", put(2, 2))
    check(tree, 1, "parent", put(0, 0))


def test_rows_beyond_32_bits():
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 30 GiB of device memory")
    R, N, V = 9, 64, 4_000_037
    x = torch.zeros(R, N, V, dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 1 << 31
    s = logits_inputs(66, R, N, 8, "bf16", [N] * R, history=3, bias=2, masked=None, tree=False)
    s.logits, s.V = x, V
    s.desc.vocab_size = V
    s.history = whole([[V - 1, V - 1, 5]] * R)
    s.history_len, s.output_start = whole([3] * R), whole([0] * R)
    s.bias_token, s.bias_len = whole([[V - 2, 0]] * R), whole([2] * R)
    s.bias_value = torch.ones(R, 2, device="cuda")
    s.presence, s.frequency = torch.ones(R, device="cuda"), torch.ones(R, device="cuda")
    run_logits(s, in_place=True)
    assert bool((x[-1, -1, -2:] == torch.tensor([1.0, -3.0], device="cuda")).all())
    assert bool((x[:, :, 0] == 1).all() and (x[:, :, 5] == -2).all())
    assert int((x != 0).sum()) == 4 * R * N
