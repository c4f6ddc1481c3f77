"""CPU pins of oracle/steps.py: closed forms, invariances, worked examples and differences."""
import math

import numpy as np
import pytest

from oracle import steps


def rng(seed):
    return np.random.default_rng(seed)


def test_frequencies_closed_forms():
    f = steps.rotary_freqs(64, 1e4)
    assert float(f[0]) == 1.0
    assert np.allclose((f[1:] / f[:-1]).astype(float), 1e4 ** (-1 / 32), rtol=1e-15)
    assert np.array_equal(steps.rotary_freqs(64, 1e4, "linear", 4.0) * 4, f)
    # the rescaled base leaves the fastest pair and divides the slowest by the factor
    g = steps.rotary_freqs(64, 1e4, "base", 8.0)
    assert float(g[0]) == 1.0 and math.isclose(float(g[-1] * 8), float(f[-1]), rel_tol=1e-14)
    h = steps.rotary_freqs(64, 1e4, "by_parts", 8.0, original_len=4096, low_turns=1, high_turns=32)
    turns = (4096 * f / (2 * np.pi)).astype(float)
    ratio = (h / f).astype(float)
    assert np.allclose(ratio[turns >= 32], 1) and np.allclose(ratio[turns <= 1], 1 / 8)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and np.allclose(ratio[mid], 1 / 8 + 7 / 8 * (turns[mid] - 1) / 31, atol=1e-12)


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_rotation_keeps_products_of_equal_distances(layout):
    x, y = rng(0).standard_normal((2, 1, 3, 32))
    f = steps.rotary_freqs(16, 100.0).astype(float)

    def dot(m, n):
        a = steps.rotate(x, np.outer([m], f), layout)[0]
        b = steps.rotate(y, np.outer([n], f), layout)[0]
        return (a * b).sum(-1)

    assert np.allclose(dot(7, 3), dot(104, 100), atol=1e-12)
    assert not np.allclose(dot(7, 3), dot(7, 4), atol=1e-3)
    there = steps.rotate(x, np.outer([9], f), layout, amplitude=2.0)[0]
    assert np.allclose(steps.rotate(there, np.outer([9], f), layout, inverse=True,
                                    amplitude=0.5)[0], x, atol=1e-12)


def test_rotation_layouts_by_hand():
    x = np.arange(1.0, 33).reshape(1, 1, 32)
    quarter = np.full((1, 8), math.pi / 2)
    y = steps.rotate(x, quarter, "half")[0][0, 0]
    assert np.allclose(y[:8], -x[0, 0, 8:16]) and np.allclose(y[8:16], x[0, 0, :8])
    assert np.array_equal(y[16:], x[0, 0, 16:])
    z = steps.rotate(x, quarter, "pairs")[0][0, 0]
    assert np.allclose(z[0:16:2], -x[0, 0, 1:16:2]) and np.allclose(z[1:16:2], x[0, 0, 0:16:2])


def test_angles_are_reduced_exactly():
    third = 2 ** 64 // 3
    a = steps.angles([third, 2 ** 63], [3, 2 ** 31 - 1])
    assert abs(a[0, 0]) < 1e-18 * 10 and a[0, 1] == pytest.approx(-math.pi)
    assert a[1, 0] == pytest.approx(2 * math.pi / 3 * ((2 ** 31 - 1) % 3), abs=1e-8)


def test_logits_worked_example():
    x = np.array([[[2.0, -2.0, 1.0, 0.5, 4.0]] * 3])
    mask = np.ones((1, 3, 5), bool)
    mask[0, 2, 4] = False
    y, _ = steps.tree_logits(x, [3], token=[[0, 1, 1]], parent=[[-1, 0, 1]], history=[[2, 3, 3]],
                             output_start=[1], repetition=[2.0], presence=[0.25],
                             frequency=[0.5], bias=[[(4, 1.0), (4, 0.5)]], mask=mask)
    # node 0: prompt 2; output 3 3 0; nodes 1 and 2 add one token 1 each
    assert np.allclose(y[0, 0], [1 - .75, -2, .5, .25 - 1.25, 5.5])
    assert np.allclose(y[0, 1], [.25, -4 - .75, .5, -1, 5.5])
    assert np.allclose(y[0, 2, :4], [.25, -4 - 1.25, .5, -1]) and y[0, 2, 4] == -np.inf


@pytest.mark.parametrize("case", [
    dict(), dict(group=8, shared=True, act="silu", gate=1, pre=False),
    dict(group=8, act="sigmoid", gate=1, residual=1), dict(residual=1, alpha=0.3),
    dict(post=False, residual=1, gate=1), dict(post=False, residual=1, dy=0)])
def test_block_norm_gradients_against_differences(case):
    r = rng(3)
    T, W = 3, 24
    group, shared = case.get("group", 0), case.get("shared", False)
    kw = dict(group=group, shared=shared, post=case.get("post", True), pre=case.get("pre", True),
              act=case.get("act", "none"), alpha=case.get("alpha", 1.0), eps=1e-3)
    ins = dict(x=r.standard_normal((T, W)),
               gate=r.standard_normal((T, W)) if case.get("gate") else None,
               residual=r.standard_normal((T, W)) if case.get("residual") else None,
               post_weight=r.standard_normal(group if shared else W) if kw["post"] else None,
               pre_weight=r.standard_normal(W) if kw["pre"] else None)
    dy = r.standard_normal((T, W)) if case.get("dy", 1) else None
    dh = r.standard_normal((T, W)) if kw["pre"] else None
    grad, size = steps.block_norm_bwd(**ins, dy=dy, dh=dh, **kw)

    def loss(**change):
        y, h, _, _ = steps.block_norm(**{**ins, **change}, **kw)
        return (0 if dy is None else (y * dy).sum()) + (0 if dh is None else (h * dh).sum())

    for name, value in ins.items():
        if value is None:
            continue
        for _ in range(4):
            d = r.standard_normal(value.shape)
            step = 1e-5
            slope = (loss(**{name: value + step * d}) - loss(**{name: value - step * d})) / (2 * step)
            assert slope == pytest.approx((grad["d" + name] * d).sum(), rel=1e-6, abs=1e-7), name
        assert (size["d" + name] >= np.abs(grad["d" + name]) * (1 - 1e-12)).all()


def test_block_norm_closed_forms():
    x = np.full((2, 16), 3.0)
    y, h, _, _ = steps.block_norm(x, eps=1e-12)
    assert np.allclose(y, 1) and np.allclose(h, 1)
    y, h, _, _ = steps.block_norm(x, residual=-x, post=False, pre=False)
    assert np.array_equal(y, 0 * x) and h is None
    y = steps.block_norm(x, gate=np.zeros((2, 16)), pre=False, act="sigmoid", eps=1e-12)[0]
    assert np.allclose(y, 0.5)
