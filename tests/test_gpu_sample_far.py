"""Sampling at temperatures near binary32's largest number, which make ordinary numbers of logits at the type's lowest value."""
import numpy as np
import pytest

from test_gpu_sample import check, env          # noqa: F401

pytestmark = pytest.mark.gpu
TEMPERATURES = [8e36, 3e37, 1e38, 2.5e38, 3.4e38]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("vocab", [70, 1500, 20011])
@pytest.mark.parametrize("f", [{"top_k": 50}, {"top_k": 50, "min_p": 0.01}, {"top_k": 300, "top_p": 0.9}, {}], ids=str)
def test_masks_of_the_lowest_value(env, f, vocab, dtype):      # noqa: F811
    # the k-th of the threads' largest logits is a mask: the least candidate lies at the lowest value, not below it
    torch, _ = env
    rng = np.random.default_rng(vocab)
    rows = len(TEMPERATURES)
    x = torch.full((rows, vocab), torch.finfo(getattr(torch, dtype)).min, dtype=getattr(torch, dtype), device="cuda")
    x[:, 3:vocab:40] = torch.from_numpy(rng.normal(size=(rows, len(range(3, vocab, 40))))).to(x.dtype).cuda()
    x[:, -1] = -float("inf")
    e = torch.from_numpy(rng.exponential(size=(rows, vocab)).astype(np.float32)).cuda()
    check(env, x, e, temperature=TEMPERATURES, **{n: [v] * rows for n, v in f.items()})


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("vocab", [2, 70, 1500, 20011])
@pytest.mark.parametrize("f", [{}, {"top_k": 5}, {"top_k": 50, "min_p": 0.2}, {"top_k": 600, "top_p": 0.7}, {"top_p": 0.5}, {"min_p": 0.3}], ids=str)
def test_differences_past_the_largest_number(env, f, vocab, dtype):      # noqa: F811
    # the temperatures make numbers from 1 to 20 of what lies between these logits
    torch, _ = env
    rng = np.random.default_rng(vocab + 1)
    rows = len(TEMPERATURES)
    x = torch.from_numpy((rng.random((rows, vocab)) * 2 - 1) * 3.38e38).to(getattr(torch, dtype)).cuda()
    x[:, 0], x[:, -1] = -3.38e38, 3.38e38
    e = torch.from_numpy(rng.exponential(size=(rows, vocab)).astype(np.float32)).cuda()
    e[::2, 0] = 1e-35                                  # the one farthest below wins where it stays
    check(env, x, e, temperature=[3.5e37, 6e37, 1e38, 2.5e38, 3.4e38], **{n: [v] * rows for n, v in f.items()})
