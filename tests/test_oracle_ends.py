"""Pins of oracle/ends.py: published answers of the generator, gradients against differences, closed forms."""
import numpy as np
import pytest

from oracle import ends


@pytest.mark.parametrize("counter,key,want", [       # known answers of the generator's authors
    ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
    ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
    ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))])
def test_philox(counter, key, want):
    assert tuple(ends.philox(counter, key)) == want


def test_bits_of_an_element():
    seed, step, site = -5, 2 ** 33 + 7, 11
    bits = ends.bits16(seed, step, site, 3, 21)
    for row, col in ((0, 0), (2, 20), (1, 13)):
        words = ends.philox((col // 8, row, 7, site), ((seed & (2 ** 64 - 1)) & 0xffffffff, (seed & (2 ** 64 - 1)) >> 32))
        assert bits[row, col] == (words[col % 8 // 2] >> (16 * (col % 2))) & 0xffff


def test_dropout_keeps_its_share_and_its_mean():
    f = ends.factor((3, 4), 0.25, 0, 200, 1000)
    share = (f > 0).mean()
    assert abs(share - 0.75) < 5 * np.sqrt(0.75 * 0.25 / f.size) and np.allclose(np.unique(f), [0, 4 / 3])
    other = ends.factor((3, 5), 0.25, 0, 200, 1000)
    assert abs(((f > 0) & (other > 0)).mean() - 0.75 ** 2) < 0.01


def make(kind, post, gate, seed=0):
    rng = np.random.default_rng(seed)
    t, n = 3, 7
    d = dict(h=rng.normal(size=(t, n)), branch=rng.normal(size=(t, n)), gate=None if gate is None else rng.normal(size=n if gate == "row" else (t, n)),
             post_w=rng.normal(size=n), post_b=rng.normal(size=n), w=rng.normal(size=n), b=rng.normal(size=n))
    drop = ends.factor((1, 2), 0.3, 5, t, n)
    f = lambda a: ends.residual_norm(a["h"], a["branch"], a["gate"], post, a["post_w"], a["post_b"], kind, a["w"], a["b"], 1.3, 0.7, 1e-5, drop)  # noqa: E731
    return rng, d, drop, f


@pytest.mark.parametrize("kind,post,gate", [("rms", None, None), ("layer", None, "row"), ("rms", "layer", "token"), (None, "rms", "row"), ("layer", "rms", None)])
def test_gradients_against_differences(kind, post, gate):
    rng, d, drop, f = make(kind, post, gate)
    total, y = f(d)
    gt, gy = rng.normal(size=total.shape), rng.normal(size=total.shape)

    def loss(a):
        total, y = f(a)
        return (total * gt).sum() + (0.0 if y is None else (y * gy).sum())
    got = ends.residual_norm_backward(gy, gt, total, d["branch"], d["gate"], post, d["post_w"], d["post_b"], kind, d["w"], 1.3, 0.7, 1e-5, drop)
    for name in d:
        if d[name] is None or name not in got:
            continue
        g = got[name] if d[name].ndim == 2 else got[name].sum(0)
        for at in np.ndindex(d[name].shape):
            up, down = dict(d), dict(d)
            up[name], down[name] = d[name].copy(), d[name].copy()
            up[name][at] += 1e-5
            down[name][at] -= 1e-5
            assert abs((loss(up) - loss(down)) / 2e-5 - g[at]) < 1e-7 * max(1, np.abs(g).max()), (name, at)


def test_logprobs_and_gradients():
    rng = np.random.default_rng(2)
    x = rng.normal(size=(4, 9)) * 3
    x[1, 3] = x[1, 5] = x[1].max() + 1           # equal ones: the lower index first
    x[2, 4:] = -np.inf
    t = np.array([2, 5, 1, -100])
    got = ends.token_logprobs(x, t, 0.8, 5)
    p = np.exp(0.8 * x) / np.exp(0.8 * x).sum(-1, keepdims=True)
    assert np.allclose(got["logprob"], [np.log(p[0, 2]), np.log(p[1, 5]), np.log(p[2, 1]), 0])
    with np.errstate(divide="ignore", invalid="ignore"):
        assert np.allclose(got["entropy"], -np.where(p > 0, p * np.log(p), 0).sum(-1))
    assert list(got["top_token"][1, :2]) == [3, 5] and got["top_token"][2, 4] == -1 and got["top_logprob"][2, 4] == -np.inf
    a, h = rng.normal(size=4), rng.normal(size=4)
    g, _ = ends.token_logprobs_backward(a, h, x, t, 0.8)
    f = lambda x: (ends.token_logprobs(x, t, 0.8, 0)["logprob"] * a).sum() + (ends.token_logprobs(x, t, 0.8, 0)["entropy"] * h).sum()  # noqa: E731
    for at in np.ndindex(x.shape):
        if np.isinf(x[at]):
            assert g[at] == 0
            continue
        up, down = x.copy(), x.copy()
        up[at] += 1e-6
        down[at] -= 1e-6
        assert abs((f(up) - f(down)) / 2e-6 - g[at]) < 1e-7


def test_rows_without_a_distribution():
    x = np.array([[1.0, np.nan], [np.inf, 0], [-np.inf, -np.inf], [2.0, 2.0]])
    got = ends.token_logprobs(x, np.array([0, 0, 0, 1]), 1.0, 1)
    assert np.isnan(got["logprob"][:3]).all() and np.isnan(got["stats"][:, :3]).all() and got["top_token"][:, 0].tolist() == [-1, -1, -1, 0]
    assert np.allclose(got["logprob"][3], -np.log(2)) and np.allclose(got["entropy"][3], np.log(2))
    g, _ = ends.token_logprobs_backward(np.array([1.0, 0, 1, 0]), None, x, np.array([0, 0, 0, 1]), 1.0)
    assert np.isnan(g[0]).all() and (g[1] == 0).all() and np.isnan(g[2]).all() and (g[3] == 0).all()
