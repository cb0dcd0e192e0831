"""Logits so far apart that their difference is past binary32's largest number, with a scale that makes ordinary numbers of it.  Against the
binary64 oracle, by the tolerances of test_gpu_logprob.py; the scales are binary32 numbers themselves."""
import numpy as np
import pytest

from oracle import ends
from test_gpu_logprob import HALF, U, check, env, host, rounding  # noqa: F401

pytestmark = pytest.mark.gpu
SCALES = [2.0 ** -126, float(np.float32(1.7e-38)), float(np.float32(9e-38))]


def make(torch, rows, vocab, dtype, seed):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy((rng.random((rows, vocab)) * 2 - 1) * 3.38e38).to(getattr(torch, dtype)).cuda()
    x[:, 0], x[:, -1] = -3.38e38, 3.38e38                 # in every row
    targets = torch.from_numpy(rng.integers(0, vocab, size=rows).astype(np.int32)).cuda()
    targets[0] = 0                                        # the one farthest below
    return rng, x, targets


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("shape", [(1, 2), (3, 7), (3, 1003), (2, 20000), (600, 2000)], ids=str)
def test_forward(env, shape, dtype):  # noqa: F811
    torch, B = env
    _, x, targets = make(torch, *shape, dtype, sum(shape))
    for scale in SCALES:
        for top in (0, 2, 64):
            want = check(B.token_logprobs(x, targets, scale, top), x, targets, scale, top)
            assert np.isfinite(want["logprob"]).all()


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("shape", [(1, 2), (3, 1003), (2, 20000)], ids=str)
def test_backward(env, shape, dtype):  # noqa: F811
    torch, B = env
    rows, vocab = shape
    rng, x, targets = make(torch, rows, vocab, dtype, sum(shape))
    # of a size that the smallest scale makes ordinary numbers of
    a, h = (torch.from_numpy((rng.normal(size=rows) * 2.0 ** 110).astype(np.float32)).cuda() for _ in range(2))
    for scale in SCALES:
        stats = B.token_logprobs(x, targets, scale)[3]
        got = host(B.token_logprobs_backward(a, h, x, targets, stats, scale))
        t = targets.cpu().numpy()
        want, size = ends.token_logprobs_backward(host(a), host(h), host(x), t, scale)
        full = ends.token_logprobs(host(x), None, scale, 0)
        s, log_s = rounding(full, vocab)
        entropy = log_s + s * (1 + full["spread"]) + 3 * U * full["spread2"]
        d = scale * np.abs(host(x) - full["stats"][0][:, None])
        p = np.exp(-d - full["stats"][1][:, None])
        tol = HALF[dtype] * np.abs(want) + size * (log_s[:, None] + 6 * U * (d + 2) + 8 * U) * 1.5
        tol += scale * p * np.abs(host(h))[:, None] * (entropy[:, None] + 4 * U * (d + 1))
        tol[np.arange(rows), t] += 4 * U * scale * np.abs(host(a))
        bad = ~(np.abs(got - want) <= tol)
        assert not bad.any(), (scale, np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], tol[bad][:5])
