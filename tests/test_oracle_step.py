"""The oracle of the operators between two layers against values that can be worked out by hand, and its gradients
against differences of its own forward."""
import math

import numpy as np
import pytest

from oracle import step


def tables(n, rot):
    a = np.arange(n)[:, None] * 100.0 ** (-np.arange(rot // 2) / (rot // 2))
    return np.cos(a), np.sin(a)


def test_rotation_of_a_quarter_turn():
    cos, sin = np.array([[0.0, 1.0]]), np.array([[1.0, 0.0]])
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    assert step.norm_rope(x, None, cos, sin, [0], 0, False)[0, 0].tolist() == [-3, 2, 1, 4, 5]       # pairs (0, 2), (1, 3)
    assert step.norm_rope(x, None, cos, sin, [0], 0, True)[0, 0].tolist() == [-2, 1, 3, 4, 5]        # pairs (0, 1), (2, 3)
    n = step.norm_rope(x, np.full(5, 2.0), cos, sin, [0], 0.0, True)
    np.testing.assert_allclose(n[0, 0], 2 / math.sqrt(11) * np.array([-2, 1, 3, 4, 5]))
    assert np.isnan(step.norm_rope(x, None, cos, sin, [1], 0, False)[0, 0][:4]).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("weight", [False, True])
def test_gradients_against_differences(interleaved, weight):
    rng = np.random.default_rng(1)
    x, dy = rng.normal(size=(3, 2, 24)), rng.normal(size=(3, 2, 24))
    w = 1 + 0.3 * rng.normal(size=24) if weight else None
    cos, sin = tables(9, 16)
    pos = [4, 0, 8]
    f = lambda x, w: (step.norm_rope(x, w, cos, sin, pos, 1e-3, interleaved) * dy).sum()  # noqa: E731
    dx, dw, _ = step.norm_rope_backward(dy, x, w, cos, sin, pos, 1e-3, interleaved)
    h = 1e-6
    for at in [(0, 0, 0), (1, 1, 7), (2, 0, 15), (2, 1, 23), (0, 1, 20)]:
        d = np.zeros_like(x)
        d[at] = h
        assert abs((f(x + d, w) - f(x - d, w)) / (2 * h) - dx[at]) < 1e-7
    for j in (0, 9, 23) if weight else ():
        d = np.zeros(24)
        d[j] = h
        assert abs((f(x, w + d) - f(x, w - d)) / (2 * h) - dw[j]) < 1e-7


def test_quantiser_by_hand():
    c, s, lo = step.quantise(np.array([[0.0, 15.0, 7.4, 7.6], [2.0, 2.0, 2.0, 2.0], [-1.0, 0.5, np.nan, 0.0]]))
    assert c[0].tolist() == [0, 15, 7, 8] and s[0] == 1 and lo[0] == 0
    assert c[1].tolist() == [0] * 4 and s[1] == 2.0 ** -24 and lo[1] == 2
    assert c[2].tolist() == [0] * 4 and np.isnan(s[2]) and np.isnan(lo[2])


def test_a_tile_by_hand():
    # token 19 of a tile, head size 40 (padded to 64): its codes 0, 15 at columns 0 and 39, its neighbours' untouched
    tile = np.full(step.tile_bytes(40), 0xFF, np.uint8)
    k, v = np.zeros((1, 40)), np.zeros((1, 40))
    k[0, 39] = v[0, 39] = 15.0
    step.put_tokens(tile, k, v, 40, [19])
    words = tile[:2048].view(np.uint32)
    # keys: token 19 = 16 + 3, column 39 = 32 + 7: word (1, 0, 3, 1), element 7 at bits 28..31
    assert words[((1 * 4 + 0) * 16 + 3) * 2 + 1] == 0xF0000000
    # values: token 19: e / 4 = 1, quad 0, e % 4 = 3, so element 7; column 39 = 32 + 7: word (1, 0, 7, 0)
    assert words[256 + ((1 * 4 + 0) * 16 + 7) * 2] == 0xFFFFFFFF
    assert words[256 + ((0 * 4 + 0) * 16 + 7) * 2] == 0x0FFFFFFF
    got_k, got_v = step.get_tile(tile, 40)
    np.testing.assert_array_equal(got_k[19], k[0])
    np.testing.assert_array_equal(got_v[19], v[0])


def test_attention_by_hand():
    table = np.array([[1, 0]])
    pages = np.zeros((2, 1, 1, step.tile_bytes(8)), np.uint8)
    k, v = np.zeros((40, 1, 8)), np.zeros((40, 1, 8))
    v[:, 0, 0] = np.arange(40)
    step.append(pages, table, [0, 40], [40], k, v, 8)
    q = np.ones((2, 2, 8))
    out, lse, _ = step.attention(q, pages, table, [0, 2], [40], 0.3)
    got = [step.read(pages, table[0], 40, 8)[1][:39, 0, 0].mean(), step.read(pages, table[0], 40, 8)[1][:, 0, 0].mean()]
    np.testing.assert_allclose(out[:, 0, 0], got)
    np.testing.assert_allclose(lse[:, 1], [math.log(39), math.log(40)])
    out, lse, _ = step.attention(q, pages, table, [0, 2], [40], 0.3, window=3, sinks=2)
    vv = step.read(pages, table[0], 40, 8)[1][:, 0, 0]
    np.testing.assert_allclose(out[1, 0, 0], vv[[0, 1, 37, 38, 39]].mean())
    out, lse, _ = step.attention(q, pages, table, [0, 2], [1], 0.3)          # the first row has a negative position
    assert (out[0] == 0).all() and np.isneginf(lse[0]).all() and (lse[1] == 0).all()


def test_sampling_by_hand():
    x = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    one = np.ones(4)
    assert step.sample_row(x, one)[0] == 1
    assert abs(step.sample_row(x, one)[1] - math.log(0.4)) < 1e-12
    e = np.array([1e-3, 1.0, 1.0, 1.0])                         # a small variate makes its token win
    assert step.sample_row(x, e)[0] == 0
    assert step.sample_row(x, e, top_k=3)[0] == 1
    assert step.sample_row(x, e, top_p=0.89)[0] == 1 and step.sample_row(x, e, top_p=0.91)[0] == 0
    assert step.sample_row(x, e, min_p=0.26)[0] == 1 and step.sample_row(x, e, min_p=0.24)[0] == 0
    assert step.sample_row(x, None, t=0.0)[0] == 1
    assert step.sample_row(np.zeros(4), one, top_k=2)[0] == 0 and step.sample_row(np.zeros(4), np.array([1, 1, .1, 1]), top_k=2)[0] == 0
    assert step.sample_row(np.array([0, np.nan]), one[:2])[0] == -1 and step.sample_row(np.full(2, -np.inf), one[:2])[0] == -1
    rng = np.random.default_rng(0)                              # the frequencies are the probabilities
    got = np.bincount([step.sample_row(x, rng.exponential(size=4))[0] for _ in range(4000)], minlength=4) / 4000
    assert np.abs(got - np.exp(x)).max() < 4 * math.sqrt(0.25 / 4000)
