"""Sampling at temperatures that have no token: infinite ones, and those between 0 and the least normal number."""
import numpy as np
import pytest

from test_gpu_sample import check, env, make          # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("vocab", [5, 4099, 16384, 32768, 65536])          # from 16384 on: rows of whole rounds of a workgroup
def test_infinite_and_subnormal(env, vocab, dtype):      # noqa: F811
    torch, _ = env
    rng = np.random.default_rng(vocab)
    below = np.nextafter(np.float32(2.0 ** -126), np.float32(0))
    t = [float("inf"), 1e-38, 4.4e-39, 2.0 ** -127, below, 1e-45, float("inf"), 2.0 ** -126, 3e38, 1.0]
    x, e = make(torch, rng, len(t), vocab, getattr(torch, dtype))
    check(env, x, e, temperature=t, top_k=[0, 0, 5, 1, 0, 0, 900, 1, 1, 0], top_p=[1, 1, 1, 1, 0.5, 0.9, 0.5, 1, 1, 1])
    check(env, x, e, temperature=[float("inf")] * len(t))
    check(env, x, e, temperature=[1e-38] * len(t))
