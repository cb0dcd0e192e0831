"""Attention over the 4-bit cache where rows and heads are many enough for whole spans of keys per 128 rows.

Inputs, checks and tolerances as for fewer rows; the heads are many so that every call here takes that form.
"""
import numpy as np
import pytest

from oracle import step
from test_gpu_attend import check, env, filled          # noqa: F401
from test_gpu_cache import i32

pytestmark = pytest.mark.gpu

CASES = [  # lengths, new, q heads, kv heads, dim, page, window, sinks, bf16
    ([65], [65], 128, 128, 32, 32, 0, 0, False), ([200, 129, 0, 70], [129, 129, 0, 66], 32, 16, 128, 64, 0, 0, True),
    ([300, 90], [33, 2], 192, 64, 96, 32, 40, 5, False), ([700], [90], 256, 256, 24, 64, 0, 0, False),
    ([620, 530], [70, 1], 140, 140, 64, 32, 100, 33, True), ([20, 100], [90, 100], 64, 64, 40, 32, 0, 0, False),
    ([400], [260], 80, 80, 64, 128, 1, 0, False), ([512], [260], 60, 60, 128, 32, 33, 70, False),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_attention(env, case):      # noqa: F811
    torch, B = env
    lengths, news, hq, hk, dim, page, window, sinks, bf16 = case
    rng = np.random.default_rng(sum(lengths) + hq)
    pages, table = filled(env, rng, lengths, hk, dim, page)
    starts = np.cumsum([0] + news)
    x = torch.from_numpy(rng.normal(size=(int(starts[-1]), hq + 1, dim)) * 1.5).to(torch.bfloat16 if bf16 else torch.float16).cuda()
    q = x[:, 1:]
    out, lse = B.cache_attention(q, pages, i32(torch, table), i32(torch, starts), i32(torch, lengths), window=window, sinks=sinks,
                                 max_new=max(news), max_len=max(max(lengths), max(news)), want_lse=True)
    want = step.attention(q.double().cpu().numpy(), pages.cpu().numpy(), table, starts, lengths, dim ** -0.5, window, sinks)
    check(env, out, lse, want, bf16)


@pytest.mark.parametrize("q_scale,v_scale", [(1e-4, 1.0), (40.0, 1.0), (1.0, 1e-6), (1.0, 3000.0), (0.0, 1.0)])
def test_magnitudes(env, q_scale, v_scale):      # noqa: F811
    torch, B = env
    rng = np.random.default_rng(15)
    pages, table = filled(env, rng, [400], 128, 32, 32, v_scale)
    q = torch.from_numpy(rng.normal(size=(70, 128, 32)) * q_scale).half().cuda()
    out, lse = B.cache_attention(q, pages, i32(torch, table), i32(torch, [0, 70]), i32(torch, [400]), want_lse=True)
    want = step.attention(q.double().cpu().numpy(), pages.cpu().numpy(), table, [0, 70], [400], 32 ** -0.5)
    check(env, out, lse, want, False)


@pytest.mark.parametrize("down", [False, True])
def test_rising_and_falling_scores(env, down):      # noqa: F811
    # every key's score lies beyond the one before by more than the reference's slack; step sizes of the values differ by 2^20
    torch, B = env
    rng = np.random.default_rng(16)
    n, dim, heads = 300, 32, 128
    pages = B.cache_empty(10, 32, heads, dim)
    pages.fill_(0xFF)
    table = np.arange(10, dtype=np.int32)[None]
    k = np.linspace(0, 35, n)[:, None, None] * np.ones((1, heads, dim))
    v = rng.normal(size=(n, heads, dim)) * 2.0 ** rng.integers(-10, 10, size=(n, heads, 1))
    kt, vt = (torch.from_numpy(np.ascontiguousarray(a)).half().cuda() for a in (k[::-1] if down else k, v))
    B.cache_append(pages, i32(torch, table), i32(torch, [0, n]), i32(torch, [n]), kt, vt)
    q = torch.from_numpy(np.abs(rng.normal(size=(70, heads, dim))) + 0.5).half().cuda()
    out, lse = B.cache_attention(q, pages, i32(torch, table), i32(torch, [0, 70]), i32(torch, [n]), want_lse=True)
    want = step.attention(q.double().cpu().numpy(), pages.cpu().numpy(), table, [0, 70], [n], 32 ** -0.5)
    check(env, out, lse, want, False)


def test_masked_keys_missing_pages_and_spoilt_rows(env):      # noqa: F811
    torch, B = env
    rng = np.random.default_rng(17)
    n, new, heads = 300, 80, 128
    pages, table = filled(env, rng, [n], heads, 32, 32)
    table[0, 4] = -1
    args = (pages, i32(torch, table), i32(torch, [0, new]), i32(torch, [n]))
    q = torch.from_numpy(rng.normal(size=(new, heads, 32))).half().cuda()
    base, lse = B.cache_attention(q, *args, window=100, sinks=3, want_lse=True)
    check(env, base, lse, step.attention(q.double().cpu().numpy(), pages.cpu().numpy(), table, [0, new], [n], 32 ** -0.5, 100, 3), False)
    for factor in (300.0, -300.0, 0.0, float("nan"), float("inf")):
        q2 = q.clone()
        q2[::3] *= factor
        got = B.cache_attention(q2, *args, window=100, sinks=3)
        keep = torch.arange(new, device="cuda") % 3 != 0
        assert torch.equal(got[keep], base[keep]), factor
        assert factor - factor == 0 or torch.isnan(got[::3]).all()
    # NaN in keys that no row sees, and in the last row's own key
    bad = torch.full((1, heads, 32), float("nan"), device="cuda").half()
    for t in (50, n - 1):
        B.cache_append(pages, i32(torch, table), i32(torch, [0, 1]), i32(torch, [t + 1]), bad, bad)
    got = B.cache_attention(q, *args, window=100, sinks=3)
    assert torch.equal(got[:-1], base[:-1]) and torch.isnan(got[-1]).all()


@pytest.mark.parametrize("case", [  # one token each: heads and spans that take eight waves, four, ranges
    ([350], 8, 2, 128, 0, 0, False), ([1000, 300], 40, 20, 64, 0, 0, True), ([1500, 290, 900, 64] * 4, 32, 16, 32, 0, 0, False),
    ([900, 2000] * 4, 64, 32, 32, 500, 3, False), ([700, 33] * 9, 32, 32, 24, 0, 0, True), ([9000], 2, 1, 96, 0, 0, False),
], ids=lambda c: "%d to %d, %d heads" % (len(c[0]), max(c[0]), c[2]))
def test_single_tokens(env, case):      # noqa: F811
    torch, B = env
    lengths, hq, hk, dim, window, sinks, bf16 = case
    rng = np.random.default_rng(sum(lengths) + hq)
    pages, table = filled(env, rng, lengths, hk, dim, 64)
    n = len(lengths)
    q = torch.from_numpy(rng.normal(size=(n, hq, dim)) * 1.5).to(torch.bfloat16 if bf16 else torch.float16).cuda()
    starts = np.arange(n + 1)
    out, lse = B.cache_attention(q, pages, i32(torch, table), i32(torch, starts), i32(torch, lengths), window=window, sinks=sinks,
                                 max_new=1, max_len=max(lengths), want_lse=True)
    want = step.attention(q.double().cpu().numpy(), pages.cpu().numpy(), table, starts, lengths, dim ** -0.5, window, sinks)
    check(env, out, lse, want, bf16)
