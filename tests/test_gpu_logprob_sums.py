"""Rows whose first logits are the largest, so that every thread has one, and whose others lie at one distance below: the same term is
added over and over, so that its roundings do not cancel.  Many rows, which few threads each take; every row another distance, beginning
off the 16-byte grid by turns.

Tolerance, in steps of u = 2^-24 relative to S: a batch's 16 terms 16, the batches of 128 threads vocab / 2048 + 1, the join 10, a term
2 and 3 d, the two growths of the largest logit that a thread can see here 8.  ln S adds 2 |ln S|; the entropy is off by that and by W / S,
whose W has the terms' errors again and 2 of its own, of at most d."""
import numpy as np
import pytest

from test_gpu_logprob import U, env, host  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_equal_terms(env, dtype):  # noqa: F811
    torch, B = env
    rows, vocab, tops = 1100, 131077, 1040
    step = 128 if dtype == "float16" else 16
    d = (1 + np.arange(rows) % (8 * step)) / step                        # 8 to 16 less this: exact in both types
    x = (16.0 - torch.from_numpy(d)).to(getattr(torch, dtype)).cuda()[:, None].repeat(1, vocab)
    x[:, :tops] = 16.0
    targets = torch.full((rows,), 70001, dtype=torch.int32, device="cuda")
    targets[::3] = 3
    lp, _, _, stats = (host(t) for t in B.token_logprobs(x, targets))
    rest = (vocab - tops) * np.exp(-d)
    log_s = np.log(tops + rest)
    share = rest / (tops + rest)
    s = (16 + vocab / 2048 + 1 + 10 + 2 + 8 + 3 * d * share) * U
    off = s + 2 * U * log_s
    want = np.where(np.arange(rows) % 3 == 0, 0.0, -d) - log_s
    worst = np.abs(stats[1] - log_s).max() / U
    assert (stats[0] == 16).all() and (np.abs(stats[1] - log_s) <= off).all(), worst
    assert (np.abs(lp - want) <= off + 2 * U * log_s + 4 * U * np.abs(want)).all()
    assert (np.abs(stats[2] - (log_s + d * share)) <= off + (2 * s + 2 * U) * d * share + 2 * U * np.abs(log_s + d * share)).all()
