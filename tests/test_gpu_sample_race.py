"""Sampling: the race is run on distances to the row's largest logit, so neither small temperatures nor a common offset of the
logits decide it.  Tokens and log-probabilities against the binary64 oracle."""
import numpy as np
import pytest

from test_gpu_sample import check, env          # noqa: F401

pytestmark = pytest.mark.gpu
FILTERS = [{}, {"top_k": 50}, {"top_k": 2000}, {"top_p": 0.9}, {"top_k": 600, "top_p": 0.7}]


def filters(f, rows):
    return {n: [v] * rows for n, v in f.items()}


@pytest.mark.parametrize("f", FILTERS, ids=str)
@pytest.mark.parametrize("vocab", [2, 3001])
def test_least_temperatures(env, vocab, f):      # noqa: F811
    # products of raw logits with 1 / T pass the largest binary32 number here
    torch, _ = env
    rng = np.random.default_rng(vocab)
    pairs = [(2.0 ** -126, 3, 20), (1e-37, 24, 30), (2.0 ** -126, -20, -3), (1e-30, 60000, 60032), (1e-37, -30, 5)]
    x = np.empty((len(pairs), vocab))
    for r, (_, low, high) in enumerate(pairs):
        x[r] = low
        x[r, vocab - 1] = high
    e = rng.exponential(size=x.shape).astype(np.float32)
    for dtype in (torch.float16, torch.float32):
        check(env, torch.from_numpy(x).to(dtype).cuda(), torch.from_numpy(e).cuda(), temperature=[p[0] for p in pairs], **filters(f, len(pairs)))


@pytest.mark.parametrize("f", FILTERS, ids=str)
def test_tied_maxima_at_small_temperatures(env, f):      # noqa: F811
    # 40 largest logits of equal size: the variates choose among them
    torch, _ = env
    rng = np.random.default_rng(21)
    rows, vocab = 8, 5000
    x = rng.normal(size=(rows, vocab))
    for r in range(rows):
        x[r, rng.choice(vocab, 40, replace=False)] = 20
    e = rng.exponential(size=x.shape).astype(np.float32)
    for t in (1e-6, 1e-3, 1e-20):
        check(env, torch.from_numpy(x).half().cuda(), torch.from_numpy(e).cuda(), temperature=[t] * rows, **filters(f, rows))


@pytest.mark.parametrize("f", FILTERS + [{"min_p": 0.05}, {"top_p": 0.95, "min_p": 0.05}], ids=str)
@pytest.mark.parametrize("offset", [1e6, -1e6, 3e7])
def test_common_offset(env, offset, f):      # noqa: F811
    # logits in steps of 1/16 or 2 beside a large offset: exact in binary32, their sums with a variate's logarithm are not
    torch, _ = env
    rng = np.random.default_rng(22)
    rows, vocab = 8, 4000
    grid = 2.0 if abs(offset) > 1e7 else 1 / 16
    x = offset - np.floor(rng.exponential(size=(rows, vocab)) * 4 / grid) * grid
    e = rng.exponential(size=x.shape).astype(np.float32)
    check(env, torch.from_numpy(x).float().cuda(), torch.from_numpy(e).cuda(), temperature=[1.0, 0.7, 1.5, 1.0, 3.0, 1.0, 0.5, 1.0], **filters(f, rows))


@pytest.mark.parametrize("f", [{}, {"top_k": 60}, {"top_p": 0.9999}], ids=str)
def test_min_p_beside_an_offset(env, f):      # noqa: F811
    # ln 0.05 = -2.9957: the logit 3 below the largest goes, the one 2.9375 below it stays, whatever they are added to
    torch, _ = env
    x = np.full((4, 3000), -40.0)
    x[:, 100], x[:, 7], x[:, 9] = 0, -3, -2.9375
    e = np.ones((4, 3000), np.float32)
    e[1, 7], e[2, 9], e[3, 7], e[3, 9] = 1e-6, 1e-6, 1e-8, 1e-6
    for offset in (0.0, 1e6, -1e6):
        check(env, torch.from_numpy(x + offset).float().cuda(), torch.from_numpy(e).cuda(), min_p=[0.05] * 4, **filters(f, 4))
