"""Sampling where a logarithm's argument is a subnormal number: variates and min_p below 2^-126 count by their own size."""
import numpy as np
import pytest

from test_gpu_sample import check, env          # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("f", [{}, {"top_k": 5}, {"top_k": 800}, {"top_p": 0.999}], ids=str)
def test_variates(env, f):      # noqa: F811
    torch, _ = env
    x = np.zeros((3, 1500))
    e = np.ones((3, 1500), np.float32)
    e[0, [0, 2, 4]] = 1e-39, 1e-44, 3e-39
    e[1, [1, 3]] = 1.4e-45, 1e-37
    e[2, [0, 3]] = 1e-42, 0                     # ln 0: nothing beats it
    check(env, torch.from_numpy(x).half().cuda(), torch.from_numpy(e).cuda(), **{n: [v] * 3 for n, v in f.items()})


@pytest.mark.parametrize("f", [{}, {"top_k": 50}], ids=str)
def test_min_p(env, f):      # noqa: F811
    # ln 1e-40 = -92.1: the logit at -93 goes, though its variate would make it win; the one at -91 stays
    torch, _ = env
    x = np.full((2, 1500), -200.0)
    x[:, 0], x[0, 4], x[1, 4] = 0, -93, -91
    e = np.ones((2, 1500), np.float32)
    e[:, 4] = 1e-43
    check(env, torch.from_numpy(x).float().cuda(), torch.from_numpy(e).cuda(), min_p=[1e-40] * 2, **{n: [v] * 2 for n, v in f.items()})
