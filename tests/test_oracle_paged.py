"""Pins of the paged cache's oracle: attention against torch's in float64 on gathered
pages, rotary positions against hand-worked angles and their invariants, eviction
against a hand-worked case."""
import math

import numpy as np
import pytest

from oracle import paged as op

torch = pytest.importorskip("torch")


def _cache(seed, layers=2, pages=7, heads=2, page=32, hd=64):
    rng = np.random.default_rng(seed)
    return op.Paged(rng.normal(size=(layers, pages, heads, page, hd)), rng.normal(size=(layers, pages, heads, page, hd)),
                    rng.random((layers, pages, heads, page)), page)


@pytest.mark.parametrize("cap", [0.0, 2.0])
def test_attention_is_torch_s(cap):
    o, rng = _cache(0), np.random.default_rng(1)
    pages, length, n, group = [4, 1, 6], 50, 5, 3
    q, masks = rng.normal(size=(n, 2 * group, 64)), [{0}, {0, 1}, {2}, set(), {1, 4}]
    out, top, total = o.attention(1, pages, length, q, masks, 0.125, cap)
    flat = [(pages[s // 32], s % 32) for s in range(length + n)]
    k = torch.tensor(np.array([o.k[1, p, :, a] for p, a in flat])).repeat_interleave(group, dim=1)
    v = torch.tensor(np.array([o.v[1, p, :, a] for p, a in flat])).repeat_interleave(group, dim=1)
    see = torch.tensor([[j < length or j - length in m for j in range(length + n)] for m in masks])
    z = torch.einsum("ihd,jhd->hij", torch.tensor(q), k) * 0.125
    z = cap * torch.tanh(z / cap) if cap else z
    z = z.masked_fill(~see, -math.inf)
    want = torch.einsum("hij,jhd->ihd", torch.softmax(z, dim=-1), v)
    np.testing.assert_allclose(out, want, rtol=0, atol=1e-13)
    np.testing.assert_allclose(top + np.log(total), torch.logsumexp(z, dim=-1).T, rtol=0, atol=1e-13)
    # the masses that a call adds are the weights, and add up to the rows that count
    before = o.mass.copy()
    o.add_mass(1, pages, length, q, masks, 0.125, cap, 0b10101)
    assert abs((o.mass - before).sum() - 3 * 2 * group) < 1e-10 and (o.mass[0] == before[0]).all()


def test_a_row_that_sees_nothing():
    o = _cache(2)
    out, top, total = o.attention(0, [3], 0, np.ones((2, 2, 64)), [set(), {1}], 1.0)
    assert not out[0].any() and (top[0] == -np.inf).all() and not total[0].any()
    np.testing.assert_allclose(out[1], o.v[0, 3, :, 1])


def test_turned_by_hand():
    f = op.frequencies(4, base=100.0)
    np.testing.assert_allclose(f, [1.0, 0.1])
    x = [1.0, 2.0, 3.0, 4.0, 5.0, 6.0]
    c, s, c2, s2 = math.cos(3), math.sin(3), math.cos(0.3), math.sin(0.3)
    np.testing.assert_allclose(op.turned(x, 3, f, False), [c - 3 * s, 2 * c2 - 4 * s2, 3 * c + s, 4 * c2 + 2 * s2, 5, 6])
    np.testing.assert_allclose(op.turned(x, 3, f, True), [c - 2 * s, 2 * c + s, 3 * c2 - 4 * s2, 4 * c2 + 3 * s2, 5, 6])
    # scores depend on the distance alone
    rng = np.random.default_rng(0)
    q, k, f = rng.normal(size=64), rng.normal(size=64), op.frequencies(48)
    for il in (False, True):
        a = op.turned(q, 900, f, il) @ op.turned(k, 893, f, il)
        assert abs(a - op.turned(q, 7, f, il) @ op.turned(k, 0, f, il)) < 1e-11


def test_scaled_frequencies():
    plain = op.frequencies(128)
    np.testing.assert_allclose(op.frequencies(128, scaling=op.LINEAR, factor=4.0), plain / 4)
    for kind, low, high in ((op.TURNS, 1, 4), (op.LOG_TURNS, 1, 32)):
        f = op.frequencies(128, scaling=kind, factor=8.0, low=low, high=high, ctx=4096)
        turns = 4096 * plain / (2 * math.pi)
        np.testing.assert_allclose(f[turns >= high], plain[turns >= high])
        np.testing.assert_allclose(f[turns <= low], plain[turns <= low] / 8)
        between = (turns > low) & (turns < high)
        assert between.any() and ((f < plain) & (f > plain / 8))[between].all()
    f = op.frequencies(2, base=10.0, scaling=op.TURNS, factor=2.0, low=1.0, high=3.0, ctx=2 * math.pi * 2)
    np.testing.assert_allclose(f, [0.75])           # 2 turns are half way: (1 + 1/2) / 2


def test_commit_and_eviction_by_hand():
    o = _cache(3, layers=1, heads=1)
    pages = [2, 5]
    before = o.k.copy()
    assert o.commit(pages, 30, [0, 2, 5]) == 33
    np.testing.assert_array_equal(o.k[0, 2, 0, 30], before[0, 2, 0, 30])
    np.testing.assert_array_equal(o.k[0, 2, 0, 31], before[0, 5, 0, 0])
    np.testing.assert_array_equal(o.k[0, 5, 0, 0], before[0, 5, 0, 3])
    o = _cache(4, layers=1, heads=1)
    o.mass[0, 2, 0, :7] = [0.5, 2.0, np.nan, 0.5, 0.0, -0.0, 0.5]
    assert o.kept(0, 0, [2], 7, 4, 1) == [0, 1, 2, 6]
    assert o.kept(0, 0, [2], 7, 5, 1) == [0, 1, 2, 3, 6]
    assert o.kept(0, 0, [2], 7, 6, 1) == [0, 1, 2, 3, 4, 6]
    assert o.kept(0, 0, [2], 7, 3, 3) == [4, 5, 6]
    assert o.evict([2], 7, 7, 0) == 7 and o.evict([2], 7, 3, 0) == 3
