"""Attention over the 4-bit cache: an infinity in a query makes its row NaN, whichever way it drives the scores."""
import numpy as np
import pytest

from test_gpu_attend import env, filled          # noqa: F401
from test_gpu_cache import i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new,heads", [(1, 1), (3, 2), (90, 1), (80, 128)])          # few rows, blocks of 32, whole spans
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("bf16", [False, True])
def test_infinity_against_keys_of_one_sign(env, new, heads, sign, bf16):      # noqa: F811
    # column 3 is every key's largest element, so its code is 15, and least values are above 0: all scores are sign x infinity
    torch, B = env
    rng = np.random.default_rng(31)
    n, dim = 200, 32
    pages, table = filled(env, rng, [n], heads, dim, 32)
    k = np.abs(rng.normal(size=(n, heads, dim))) + 0.5
    k[..., 3] = 9
    k, v = torch.from_numpy(k).half().cuda(), torch.from_numpy(rng.normal(size=(n, heads, dim))).half().cuda()
    B.cache_append(pages, i32(torch, table), i32(torch, [0, n]), i32(torch, [n]), k, v)
    q = torch.from_numpy(rng.normal(size=(new, 2 * heads, dim))).to(torch.bfloat16 if bf16 else torch.float16).cuda()
    args = (pages, i32(torch, table), i32(torch, [0, new]), i32(torch, [n]))
    for window, sinks in ((0, 0), (40, 3)):
        base, base_lse = B.cache_attention(q, *args, window=window, sinks=sinks, want_lse=True)
        spoilt = q.clone()
        spoilt[::2, 1, 3] = sign * float("inf")
        out, lse = B.cache_attention(spoilt, *args, window=window, sinks=sinks, want_lse=True)
        keep = torch.ones(new, 2 * heads, dtype=torch.bool, device="cuda")
        keep[::2, 1] = False
        assert torch.isnan(out[~keep]).all() and torch.isnan(lse[~keep]).all()
        assert torch.equal(out[keep], base[keep]) and torch.equal(lse[keep], base_lse[keep])
    # a row that sees nothing stays 0 and -infinity
    out, lse = B.cache_attention(spoilt, pages, i32(torch, np.full_like(table, -1)), *args[2:], want_lse=True)
    assert (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("new,heads", [(1, 1), (3, 2), (90, 1), (80, 128)])
def test_scores_far_below_zero(env, new, heads):      # noqa: F811
    # keys that are all alike: every score is the same number near -1e31, and the result the values' mean
    torch, B = env
    rng = np.random.default_rng(32)
    n, dim = 200, 32
    pages, table = filled(env, rng, [n], heads, dim, 32)
    k = torch.full((n, heads, dim), 2.0, device="cuda").half()
    v = torch.from_numpy(rng.normal(size=(n, heads, dim))).half().cuda()
    args = (pages, i32(torch, table), i32(torch, [0, new]), i32(torch, [n]))
    B.cache_append(pages, i32(torch, table), i32(torch, [0, n]), i32(torch, [n]), k, v)
    q = torch.full((new, heads, dim), -2.0 ** 100, device="cuda").to(torch.bfloat16)
    out, lse = B.cache_attention(q, *args, want_lse=True)
    score = -2.0 ** 100 * 2 * dim * dim ** -0.5
    assert ((lse.double() - score).abs() <= 2e-5 * abs(score)).all()
    _, values = B.cache_read(pages, i32(torch, table), i32(torch, [0, n]), n, dim)
    sums = values.double().cumsum(0)
    for i in range(new):
        seen = n - new + 1 + i
        mean = sums[seen - 1] / seen
        # the result's rounding, and fp16 weights on codes 8 from the middle at most
        tol = 2.0 ** -8 * mean.abs() + 2.0 ** -11 * (values.amax() - values.amin()).double() + 1e-5 * values.abs().max().double()
        assert ((out[i].double() - mean).abs() <= tol).all()
