"""Pins of the paged cache's oracle against arithmetic written out here (CPU only)."""
import math

import numpy as np
import pytest

from oracle import paged_oracle as po


def test_rope_is_a_rotation_of_complex_pairs():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(3, 8))
    for style in (0, 1):
        z = x[:, 0::2] + 1j * x[:, 1::2] if style else x[:, :4] + 1j * x[:, 4:]
        z = z * np.exp(1j * 7 * 100.0 ** (-np.arange(4) / 4))
        y = po.rope(x, 7, 100.0, style)
        got = y[:, 0::2] + 1j * y[:, 1::2] if style else y[:, :4] + 1j * y[:, 4:]
        np.testing.assert_allclose(got, z, atol=1e-14)


def test_attention_by_hand_and_relative_positions():
    # two slots whose logits differ by ln 3: weights 1/4 and 3/4
    d = 4
    q = np.zeros((2, d))
    q[:, 0] = 1.0
    K, V = np.zeros((3, 1, d)), np.zeros((3, 1, d))
    K[1, 0, 0] = math.log(3) * math.sqrt(d)
    K[2, 0, 0] = 1e9                                # its page is not there
    V[:, 0, 0] = [4.0, 8.0, 1e9]
    out, p = po.attend(q, 0, K, V, np.array([True, True, False]), 10.0)
    np.testing.assert_allclose(p, [[0.25, 0.75, 0.0]] * 2, atol=1e-15)
    np.testing.assert_allclose(out[:, 0], 7.0, atol=1e-14)
    np.testing.assert_allclose(po.list_weights(p, 1), [[0.5, 1.5, 0.0]], atol=1e-15)
    out, p = po.attend(q, 0, K, V, np.zeros(3, bool), 10.0)
    assert not out.any() and not p.any()
    # rotated keys: only the distance of the positions matters, and heads read their group's rows
    rng = np.random.default_rng(2)
    q, k, v = rng.normal(size=(4, 8)), rng.normal(size=(5, 2, 8)), rng.normal(size=(5, 2, 8))
    ys = []
    for shift in (0, 1000):
        kr = np.stack([po.rope(k[t], t + shift, 100.0) for t in range(5)])
        ys.append(po.attend(q, 5 + shift, kr, v, np.ones(5, bool), 100.0)[0])
    np.testing.assert_allclose(ys[0], ys[1], atol=1e-11)
    changed = v.copy()
    changed[:, 1] += 1.0
    y2 = po.attend(q, 5, np.stack([po.rope(k[t], t, 100.0) for t in range(5)]), changed, np.ones(5, bool), 100.0)[0]
    np.testing.assert_allclose(y2[:2], ys[0][:2], atol=1e-13)
    np.testing.assert_allclose(y2[2:], ys[0][2:] + 1.0, atol=1e-12)


def test_slots_of_pages():
    page, row, there = po.slots([5, -1, 7, 9], 3, 8, 9)
    assert page.tolist() == [5, 5, 5, -1, -1, -1, 7, 7] and row.tolist() == [0, 1, 2, 0, 1, 2, 0, 1]
    assert there.tolist() == [True] * 3 + [False] * 3 + [True] * 2
    assert not po.slots([9], 4, 2, 9)[2].any()


@pytest.mark.parametrize("weights,pos,position,n_keep,sink,recent,want", [
    ([5, 1, 4, 2, 3], [0, 1, 2, 3, 4], 4, 5, 0, 0, [0, 1, 2, 3, 4]),          # nothing to do
    ([5, 1, 4, 2, 3], [0, 1, 2, 3, 4], 4, 4, 0, 0, [0, 4, 2, 3]),             # the lightest leaves, the last takes its slot
    ([5, 1, 4, 2, 3], [0, 1, 2, 3, 4], 4, 3, 0, 0, [0, 4, 2]),
    ([5, 1, 4, 2, 3], [0, 1, 2, 3, 4], 4, 3, 2, 1, [0, 1, 4]),                # first two and newest protected
    ([1, 1, 1, 1, 1], [0, 1, 2, 3, 4], 4, 2, 0, 0, [0, 1]),                   # ties: lower slots
    ([0.0, -0.0, 0.0], [0, 1, 2], 2, 2, 0, 0, [0, 1]),
    ([math.nan, 0.0, -1.0, math.inf], [0, 1, 2, 3], 3, 3, 0, 0, [3, 1, 2]),
    ([1, 2, 3, 4], [9, 8, 7, 6], 9, 2, 0, 2, [0, 1]),                         # recent by position, not by slot
    ([1, 2, 3, 4], [0, 1, 2, 3], 3, 2, 4, 0, [0, 1]),                         # more protected ones than stay
    ([1, 9, 2, 8, 3, 7], [0, 1, 2, 3, 4, 5], 5, 3, 0, 0, [3, 1, 5]),          # i-th mover into the i-th free slot
])
def test_eviction_by_hand(weights, pos, position, n_keep, sink, recent, want):
    assert po.evict(weights, pos, position, n_keep, sink, recent) == want
