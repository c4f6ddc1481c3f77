"""Rotary positions and the append with the rotation on the way, against their fp64 definition.

Tolerances: steps_helpers.ROTARY_REL, and half a step of the output's type; what is not rotated is
passed on bit for bit."""
import numpy as np
import pytest
import torch

from oracle import steps as ref
from paper_2606_01774_gb300 import flare
from steps_helpers import (MARK, bits, check_rotated, make_table, rotary_inputs, run_append,
                           run_rotary, whole)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rd", [16, 48, 64, 256])
@pytest.mark.parametrize("scaling,how", [
    ("plain", {}), ("linear", dict(factor=4.0)), ("base", dict(factor=8.0)),
    ("by_parts", dict(factor=32.0, original_len=8192.0, low_turns=1.0, high_turns=4.0)),
    ("by_parts", dict(factor=0.5, original_len=100.0, low_turns=0.0, high_turns=32.0))])
def test_table(rd, scaling, how):
    """Within 2^-52 turns: fp64 powers and quotients, a few roundings of at most 0.16 turns."""
    table = make_table(rd, 5e5, scaling, **how).cpu().tolist()
    f = ref.rotary_freqs(rd, 5e5, scaling, **how) / (8 * np.arctan(np.longdouble(1)))
    for got, want in zip(table, f):
        got = np.longdouble(got % 2 ** 64) / np.longdouble(2) ** 64
        assert abs(got - (want - np.floor(want))) <= 2.0 ** -52


CASES = [
    # lens, B (0: packed), Hq, Hkv, D, rd
    ([1], 1, 16, 2, 256, 64),
    ([1] * 70, 1, 4, 1, 128, 128),
    ([5, 0, 16, 1], 16, 6, 2, 64, 48),
    ([64, 33], 64, 3, 3, 256, 256),
    ([300, 0, 1, 0, 17, 0], 0, 5, 1, 128, 96),
    ([0, 0, 1500], 0, 8, 4, 64, 16),
    ([257, 31], 0, 40, 8, 128, 64),
    ([2], 200, 1, 1, 64, 64),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("lens,B,Hq,Hkv,D,rd", CASES)
def test_rotation_matches_the_definition(lens, B, Hq, Hkv, D, rd, layout, dtype):
    s = rotary_inputs(len(lens) + rd, lens, B, Hq, Hkv, D, rd, dtype, layout, fused=B != 64,
                      amplitude=1.0 if rd != 96 else 1.3)
    q, k = run_rotary(s)
    check_rotated(s, s.q, q)
    check_rotated(s, s.k, k)
    # one at a time, and in place, the same bits
    assert torch.equal(bits(run_rotary(s, k=False)[0]), bits(q))
    assert torch.equal(bits(run_rotary(s, q=False)[1]), bits(k))
    before, live = s.v.clone(), s.live.cuda()
    run_rotary(s, in_place=True)
    assert torch.equal(bits(s.q[live]), bits(q[live])) and torch.equal(bits(s.k[live]), bits(k[live]))
    assert bool(s.q[~live].isnan().all()) and torch.equal(bits(s.v), bits(before))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_trees_turn_by_depth(layout, dtype):
    s = rotary_inputs(5, [64, 1, 0, 13, 40], 64, 4, 2, 128, 64, dtype, layout, tree=True)
    q, k = run_rotary(s)
    check_rotated(s, s.q, q)
    check_rotated(s, s.k, k)


def test_given_positions_near_and_far():
    far = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 9 + 7, 1 << 20, -12345]
    s = rotary_inputs(6, [40, 2], 0, 2, 1, 128, 128, "f32", position=lambda i: far[i % 8])
    q, _ = run_rotary(s)
    check_rotated(s, s.q, q)


def test_far_prefixes_keep_every_digit():
    """Position p and p + 2^20 differ by a fixed rotation; the definition holds at both."""
    for prefix in ([0, 7], [1 << 24, (1 << 31) - 9]):
        s = rotary_inputs(7, [9, 9], 0, 2, 1, 64, 64, "f32", prefix=prefix)
        q, _ = run_rotary(s)
        check_rotated(s, s.q, q)


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_inverse_is_the_gradient(layout):
    """The transposed map: <g, R x> = <R^-1 g, x>, and R^-1 R = 1 without an amplitude."""
    s = rotary_inputs(8, [200, 55], 0, 4, 2, 128, 96, "f32", layout, amplitude=0.7)
    q, _ = run_rotary(s)
    b = rotary_inputs(9, [200, 55], 0, 4, 2, 128, 96, "f32", layout, amplitude=0.7, inverse=True,
                      prefix=s.prefix)
    dq, _ = run_rotary(b)
    check_rotated(b, b.q, dq)
    live = s.live.cuda()
    lhs = (b.q[live].double() * q[live].double()).sum()
    rhs = (dq[live].double() * s.q[live].double()).sum()
    # both sums of 130560 products of numbers near one, each off by ROTARY_REL of them
    assert abs(lhs - rhs) < 130560 ** 0.5 * 2.0 ** -19
    # the derivative along a direction, exactly linear: R (x + d) - R x
    x0 = s.q.clone()
    s.q.add_(b.q)
    moved, _ = run_rotary(s)
    s.q.copy_(x0)
    change = (moved[live].double() - q[live].double() - 0).mul(b.q[live].double()).sum()
    rot_of_b = ((dq[live].double()) * b.q[live].double()).sum()  # <b, R^-1 b> = <b, R b>
    assert abs(change - rot_of_b) < 130560 ** 0.5 * 2.0 ** -18


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("lens,B,Hq,Hkv,D,rd,prefix", [
    ([1, 1, 1], 1, 16, 2, 256, 64, [0, 63, 1000]),
    ([7, 0, 16], 16, 4, 4, 64, 64, [15, 16, 1]),
    ([130, 0, 1, 517], 0, 6, 3, 128, 96, [0, 5, 31, 127]),
])
def test_append(lens, B, Hq, Hkv, D, rd, prefix, page, dtype):
    s = rotary_inputs(20 + page, lens, B, Hq, Hkv, D, rd, dtype, "half", prefix=prefix, page=page)
    q, k, k_pool, v_pool = run_append(s)
    check_rotated(s, s.q, q)
    check_rotated(s, s.k, k)
    plain = run_rotary(s)
    assert torch.equal(bits(plain[0]), bits(q)) and torch.equal(bits(plain[1]), bits(k))
    # the pools: the dense keys' bits, the values' bits, and nothing else changed
    want_k, want_v = s.k_pool.clone(), s.v_pool.clone()
    for i in s.live.nonzero()[:, 0].tolist():
        p = int(s.page_table[s.owner[i], s.at[i] // page])
        want_k[p, :, s.at[i] % page], want_v[p, :, s.at[i] % page] = k[i], s.v[i]
    assert torch.equal(bits(k_pool), bits(want_k)) and torch.equal(bits(v_pool), bits(want_v))
    _, none, k2, v2 = run_append(s, q=False, dense_k=False)
    assert none is None and torch.equal(bits(k2), bits(k_pool)) and torch.equal(bits(v2), bits(v_pool))


def test_append_with_positions_of_its_own():
    s = rotary_inputs(30, [20, 9], 0, 4, 2, 64, 32, "bf16", prefix=[30, 0], page=16,
                      position=lambda i: 3 * i - 7)
    q, k, k_pool, _ = run_append(s)
    check_rotated(s, s.q, q)
    check_rotated(s, s.k, k)
    assert torch.equal(bits(k_pool[int(s.page_table[0, 1]), :, 14]), bits(k[0]))


def test_a_bad_request_is_skipped():
    s = rotary_inputs(31, [3, 5, 2, 4], 8, 4, 2, 64, 64, "bf16", prefix=[3, 9, 40, 11], page=16)
    whole_call = run_append(s)

    def check(expect, skipped, **change):
        old = {n: getattr(s, n) for n in change}
        for n, v in change.items():
            setattr(s, n, v)
        got = run_append(s, expect=expect)
        for n, v in old.items():
            setattr(s, n, v)
        live = s.live.clone()
        for r in skipped:
            live[8 * r:8 * r + 8] = False
        check_rotated(s, s.q, got[0], live)
        check_rotated(s, s.k, got[1], live)
        for i, first in ((2, s.k_pool), (3, s.v_pool)):
            want = whole_call[i].clone()
            for r in skipped:
                pages = s.page_table[r][s.page_table[r] >= 0].long()
                want[pages] = first[pages]
            assert torch.equal(bits(got[i]), bits(want))

    lens = lambda *n: whole(list(n))  # noqa: E731
    check(flare.FLARE_DEV_BAD_ACCEPT_LEN, [1], token_len=lens(3, 9, 2, 4))
    check(flare.FLARE_DEV_BAD_ACCEPT_LEN, [0], token_len=lens(-1, 5, 2, 4))
    check(flare.FLARE_DEV_BAD_PREFIX_LEN, [2], prefix_len=lens(3, 9, -1, 11))
    cols = s.page_table.shape[1]
    check(flare.FLARE_DEV_BAD_PREFIX_LEN, [2], prefix_len=lens(3, 9, 16 * cols - 1, 11))
    table = s.page_table.clone()
    table[1, 0] = s.k_pool.shape[0]
    check(flare.FLARE_DEV_BAD_PAGE, [1], page_table=table)
    table = s.page_table.clone()
    table[3, 0] = -1
    check(flare.FLARE_DEV_BAD_PAGE, [3], page_table=table)


def test_the_tokens_of_a_bad_page_are_skipped_alone():
    s = rotary_inputs(32, [40], 0, 2, 1, 64, 64, "bf16", prefix=[10], page=16)
    s.page_table[0, 1] = 1 << 20
    q, k, _, _ = run_append(s, expect=flare.FLARE_DEV_BAD_PAGE)
    live = s.live & torch.tensor([i >= 40 or not 16 <= s.at[i] < 32 for i in range(s.rows)])
    check_rotated(s, s.q, q, live)
    check_rotated(s, s.k, k, live)


def test_a_wrong_tree_or_packing_is_flagged():
    s = rotary_inputs(33, [4, 5], 8, 2, 1, 64, 64, "bf16", tree=True)
    good = s.parent.clone()
    for r, i, p in ((0, 2, 2), (0, 3, 7), (1, 0, 0), (1, 4, -1)):
        s.parent = good.clone()
        s.parent[r, i] = p
        q, _ = run_rotary(s, expect=flare.FLARE_DEV_BAD_TREE)
        live = s.live.clone()
        live[8 * r:8 * r + 8] = False
        check_rotated(s, s.q, q, live)
    p = rotary_inputs(34, [4, 5, 6], 0, 2, 1, 64, 64, "bf16")
    good = p.token_start.clone()
    for at, value in ((0, -1), (1, 20), (3, p.rows + 1), (2, 3), (1, -2 ** 31), (3, 2 ** 31 - 1)):
        p.token_start = good.clone()
        p.token_start[at] = value
        run_rotary(p, expect=flare.FLARE_DEV_BAD_ACCEPT_LEN)


def test_rows_beyond_32_bits():
    """Keys at the far end of strided rows and of pools of more than 2^31 elements."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GiB of device memory")
    D, Hkv, page, rows = 256, 2, 64, 3
    wide = 1 << 30
    raw = torch.zeros(3 * wide, dtype=torch.bfloat16, device="cuda")
    s = rotary_inputs(35, [2, 1], 0, 2, Hkv, D, 64, "bf16", fused=False, prefix=[5, 70], page=page,
                      spare=0)
    view = raw.as_strided((rows, Hkv, D), (wide, D, 1))
    view.copy_(s.k)
    small, s.k = s.k, view
    pages, n = 70000, s.k_pool.shape[0]
    pools = [torch.zeros(pages, Hkv, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    assert pools[0].numel() > 1 << 31
    table = s.page_table.clone()
    s.page_table[table >= 0] += pages - n
    s.desc.k_stride, s.desc.num_pages = wide, pages
    _, k, k_pool, v_pool = run_append(s, pools=pools)
    check_rotated(s, small, k)
    for i in range(rows):
        p = int(s.page_table[s.owner[i], s.at[i] // page])
        assert torch.equal(bits(k_pool[p, :, s.at[i] % page]), bits(k[i]))
        assert torch.equal(bits(v_pool[p, :, s.at[i] % page]), bits(s.v[i]))
    assert int((k_pool[:pages - n] != 0).sum()) == 0


def test_nothing_to_do():
    s = rotary_inputs(36, [0, 0], 0, 2, 1, 64, 64, "bf16", page=16)
    q, k, k_pool, _ = run_append(s)
    assert bool((q == MARK).all()) and torch.equal(bits(k_pool), bits(s.k_pool))
    s.desc.num_requests = 0
    before = flare.flare_launch_count()
    run_append(s)
    assert flare.flare_launch_count() == before
