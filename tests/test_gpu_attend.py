"""Attention over the 4-bit cache on the GPU against the binary64 oracle, reading the same bytes.

Tolerance of an output: the softmax weights times step sizes are rounded to fp16, 2^-11 of each, on codes measured from 8 of
0..15, so at most 2^-11 of the largest spread of a visible head's values; the result is rounded once (2^-11 or 2^-8 of it);
binary32's share is in the oracle's bound (1e-5 of the largest value, more where scores are large).  lse: 2e-5 of its size.
"""
import numpy as np
import pytest

from oracle import step
from test_gpu_cache import i32, make_table

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2306_02272_amd import binding
    binding.lib()
    torch.cuda.set_device(0)
    return torch, binding


def filled(env, rng, lengths, heads, dim, page, v_scale=1.0):
    torch, B = env
    table, n_pages = make_table(rng, lengths, page)
    pages = B.cache_empty(n_pages, page, heads, dim)
    pages.fill_(0xFF)                                           # garbage scales are NaN wherever nothing is written
    rows = sum(lengths)
    k = torch.from_numpy(rng.normal(size=(rows, heads, dim))).half().cuda()
    k[..., ::7] *= 4
    v = torch.from_numpy(rng.normal(size=(rows, heads, dim)) * v_scale + v_scale * 0.5).half().cuda()
    B.cache_append(pages, i32(torch, table), i32(torch, np.cumsum([0] + lengths)), i32(torch, lengths), k, v, max_new=max(1, max(lengths)))
    torch.cuda.synchronize()
    return pages, table


def check(env, got, lse, want, bf16):
    out, ref_lse, bound = want
    got, lse = got.double().cpu().numpy(), lse.double().cpu().numpy()
    nan = np.isnan(out)
    assert (np.isnan(got) == nan).all()
    tol = bound[..., None] + (2.0 ** -8 if bf16 else 2.0 ** -11) * np.abs(out) + 2.0 ** -25
    bad = ~nan & ~(np.abs(got - out) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], out[bad][:5], tol[bad][:5])
    inf = np.isneginf(ref_lse)
    assert (np.isneginf(lse) == inf).all() and (got[inf] == 0).all()
    ok = ~inf & ~np.isnan(ref_lse)
    assert (np.isnan(lse) == np.isnan(ref_lse)).all()
    assert (np.abs(lse[ok] - ref_lse[ok]) <= 2e-5 * (1 + np.abs(ref_lse[ok]))).all()


CASES = [  # lengths, new, q heads, kv heads, dim, page, window, sinks, bf16
    ([1], [1], 1, 1, 8, 32, 0, 0, False), ([33], [1], 4, 2, 128, 32, 0, 0, False), ([700, 1, 32, 31], [1] * 4, 8, 8, 64, 64, 0, 0, True),
    ([300, 17], [3, 2], 12, 3, 80, 32, 0, 0, False), ([257], [5], 8, 1, 96, 256, 0, 0, False),       # 40 rows of a key head
    ([100, 513], [9, 1], 14, 2, 128, 64, 0, 0, True),                                               # 63 rows
    ([210, 64, 3], [100, 64, 3], 4, 2, 128, 64, 0, 0, False), ([333], [200], 3, 1, 40, 32, 0, 0, True),
    ([1200], [1], 2, 2, 128, 128, 0, 0, False), ([900, 40], [2, 2], 6, 2, 64, 32, 65, 0, False),
    ([900, 40, 64], [2, 2, 1], 6, 2, 64, 32, 65, 5, True), ([500], [300], 2, 1, 128, 32, 33, 70, False),
    ([400, 5], [130, 5], 4, 4, 32, 32, 1, 0, False), ([250], [1], 3, 3, 128, 32, 7, 300, False),
    ([10, 0, 40], [12, 0, 40], 4, 2, 64, 32, 0, 0, False),      # rows before the first token, an empty sequence
    ([4, 90], [80, 70], 2, 2, 64, 32, 20, 2, False), ([3000], [1], 16, 1, 128, 64, 0, 0, False), ([2500], [2], 72, 36, 64, 64, 0, 0, False),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_attention(env, case):
    torch, B = env
    lengths, news, hq, hk, dim, page, window, sinks, bf16 = case
    rng = np.random.default_rng(sum(lengths) + hq)
    pages, table = filled(env, rng, lengths, hk, dim, page)
    starts = np.cumsum([0] + news)
    x = torch.from_numpy(rng.normal(size=(int(starts[-1]), hq + 1, dim)) * 1.5).to(torch.bfloat16 if bf16 else torch.float16).cuda()
    q = x[:, 1:]                                                # strided rows
    args = (q, pages, i32(torch, table), i32(torch, starts), i32(torch, lengths))
    out, lse = B.cache_attention(*args, window=window, sinks=sinks, max_new=max(news), max_len=max(lengths), want_lse=True)
    torch.cuda.synchronize()
    want = step.attention(q.double().cpu().numpy(), pages.cpu().numpy(), table, starts, lengths, dim ** -0.5, window, sinks)
    check(env, out, lse, want, bf16)
    # other bounds give another split of the work and the same result to rounding
    out, lse = B.cache_attention(*args, window=window, sinks=sinks, want_lse=True)
    check(env, out, lse, want, bf16)


LONG = [  # many sequences, ranges of keys over several of them, more ranges of a head than lanes
    ([3000, 700, 64, 2000], [1, 2, 0, 3], 8, 4, 64, 64, 0, 0, False), ([1] + [13 * b % 800 for b in range(149)], [1] * 150, 2, 1, 32, 32, 0, 0, False),
    ([30000], [1], 1, 1, 32, 256, 0, 0, True), ([4000, 3000], [20, 1], 3, 1, 64, 32, 0, 0, False), ([5000, 40], [2, 2], 2, 1, 128, 64, 2200, 70, False),
    ([600 + 2 * b for b in range(70)], [b % 3 for b in range(70)], 4, 4, 32, 32, 400, 3, False),
    ([900, 1100], [700, 5], 2, 1, 32, 32, 0, 0, False), ([130] * 3, [129] * 3, 5, 5, 48, 64, 50, 0, True),
]


@pytest.mark.parametrize("case", LONG, ids=lambda c: "%d sequences to %d, %d rows" % (len(c[0]), max(c[0]), max(c[1])))
def test_long_and_many(env, case):
    torch, B = env
    lengths, news, hq, hk, dim, page, window, sinks, bf16 = case
    lengths = [max(a, b) for a, b in zip(lengths, news)]
    rng = np.random.default_rng(len(lengths) + hq)
    pages, table = filled(env, rng, lengths, hk, dim, page)
    starts = np.cumsum([0] + news)
    q = torch.from_numpy(rng.normal(size=(int(starts[-1]), hq, dim))).to(torch.bfloat16 if bf16 else torch.float16).cuda()
    out, lse = B.cache_attention(q, pages, i32(torch, table), i32(torch, starts), i32(torch, lengths), window=window, sinks=sinks,
                                 max_new=max(news), max_len=max(lengths), want_lse=True)
    want = step.attention(q.double().cpu().numpy(), pages.cpu().numpy(), table, starts, lengths, dim ** -0.5, window, sinks)
    check(env, out, lse, want, bf16)


@pytest.mark.parametrize("q_scale,v_scale", [(1e-4, 1.0), (40.0, 1.0), (1.0, 1e-6), (1.0, 3000.0), (0.0, 1.0)])
@pytest.mark.parametrize("new", [1, 90])
def test_magnitudes(env, q_scale, v_scale, new):
    # sharp and flat softmax, values near the ends of fp16's range
    torch, B = env
    rng = np.random.default_rng(5)
    pages, table = filled(env, rng, [400], 2, 64, 32, v_scale)
    q = torch.from_numpy(rng.normal(size=(new, 4, 64)) * q_scale).half().cuda()
    out, lse = B.cache_attention(q, pages, i32(torch, table), i32(torch, [0, new]), i32(torch, [400]), want_lse=True)
    want = step.attention(q.double().cpu().numpy(), pages.cpu().numpy(), table, [0, new], [400], 0.125)
    check(env, out, lse, want, False)


@pytest.mark.parametrize("new", [1, 90])
def test_rising_scores_and_uneven_step_sizes(env, new):
    # every key's score lies above the one before by more than the reference's slack, and step sizes of the values differ by 2^20
    torch, B = env
    rng = np.random.default_rng(6)
    n, dim = 300, 64
    pages = B.cache_empty(10, 32, 1, dim)
    pages.fill_(0xFF)
    table = np.arange(10, dtype=np.int32)[None]
    ramp = np.linspace(0, 25, n)[:, None, None] * np.ones((1, 1, dim))
    for k, v in ((ramp, rng.normal(size=(n, 1, dim)) * 2.0 ** rng.integers(-10, 10, size=(n, 1, 1))),
                 (ramp[::-1], rng.normal(size=(n, 1, dim))), (ramp * 0, np.full((n, 1, dim), -3.25)),
                 (ramp * 0, np.where(np.arange(n)[:, None, None] % 2, 0.0, rng.normal(size=(n, 1, dim)) * 1e-3))):
        kt, vt = (torch.from_numpy(np.ascontiguousarray(a)).half().cuda() for a in (k, v))
        args = (i32(torch, table),)
        B.cache_append(pages, *args, i32(torch, [0, n]), i32(torch, [n]), kt, vt)
        q = torch.from_numpy(np.abs(rng.normal(size=(new, 2, dim))) + 0.5).half().cuda()
        out, lse = B.cache_attention(q, pages, *args, i32(torch, [0, new]), i32(torch, [n]), want_lse=True)
        want = step.attention(q.double().cpu().numpy(), pages.cpu().numpy(), table, [0, new], [n], 0.125)
        check(env, out, lse, want, False)


@pytest.mark.parametrize("new", [2, 90])
def test_what_is_masked_has_no_effect(env, new):
    torch, B = env
    rng = np.random.default_rng(7)
    n = 200
    pages, table = filled(env, rng, [n], 2, 64, 32)
    q = torch.from_numpy(rng.normal(size=(new, 4, 64))).half().cuda()
    args = (i32(torch, table), i32(torch, [0, new]))
    base = B.cache_attention(q, pages, *args, i32(torch, [n - 1]), window=30, sinks=3)
    # NaN heads outside the window, past the end, and at a position that only the last row does not see
    bad = torch.full((1, 2, 64), float("nan"), device="cuda").half()
    for t in (5, n - 1):
        B.cache_append(pages, i32(torch, table), i32(torch, [0, 1]), i32(torch, [t + 1]), bad, bad)
    got = B.cache_attention(q, pages, *args, i32(torch, [n - 1]), window=30, sinks=3)
    torch.cuda.synchronize()
    pos = n - 1 - new + np.arange(new)
    clean = torch.from_numpy(pos - 30 >= 5).cuda()
    assert torch.equal(got[clean], base[clean]) and torch.isnan(got[~clean]).all()
    # a query of NaN or infinity spoils its own row only
    q2 = q.clone()
    q2[0, 1, 3], q2[1, 0, 9] = float("nan"), float("inf")
    got2 = B.cache_attention(q2, pages, *args, i32(torch, [n - 1]), window=30, sinks=3)
    assert torch.isnan(got2[0, 1]).all() and torch.isnan(got2[1, 0]).all()
    assert torch.equal(got2[2:][clean[2:]], got[2:][clean[2:]])


@pytest.mark.parametrize("new", [1, 5, 13, 90])
def test_rows_do_not_show_in_each_other(env, new):
    # sharp and NaN rows move their own reference, at other tiles than their neighbours: these keep every bit
    torch, B = env
    rng = np.random.default_rng(10)
    pages, table = filled(env, rng, [700], 1, 64, 32)
    args = (pages, i32(torch, table), i32(torch, [0, new]), i32(torch, [700]))
    q = torch.from_numpy(rng.normal(size=(new, 4, 64))).half().cuda()
    base = B.cache_attention(q, *args)
    for factor in (300.0, -300.0, 0.0, float("nan")):
        q2 = q.clone()
        q2[:, 1] *= factor
        q2[::3, 2] *= factor
        got = B.cache_attention(q2, *args)
        same = torch.ones(new, 4, dtype=torch.bool, device="cuda")
        same[:, 1], same[::3, 2] = False, False
        assert torch.equal(got[same], base[same]), factor


def test_no_page_is_no_key(env):
    torch, B = env
    rng = np.random.default_rng(8)
    lengths = [150, 100]
    pages, table = filled(env, rng, lengths, 2, 64, 32)
    table[0, 1], table[1, 0] = -1, pages.shape[0]
    for new in (1, 80):
        q = torch.from_numpy(rng.normal(size=(2 * new, 4, 64))).half().cuda()
        out, lse = B.cache_attention(q, pages, i32(torch, table), i32(torch, [0, new, 2 * new]), i32(torch, lengths), max_new=new, want_lse=True)
        check(env, out, lse, step.attention(q.double().cpu().numpy(), pages.cpu().numpy(), table, [0, new, 2 * new], lengths, 0.125), False)


def test_same_bits_twice_on_another_stream_and_in_a_graph(env):
    torch, B = env
    rng = np.random.default_rng(9)
    lengths = [1500, 700]
    pages, table = filled(env, rng, lengths, 2, 128, 64)
    q = torch.from_numpy(rng.normal(size=(2, 8, 128))).half().cuda()
    kv = torch.from_numpy(rng.normal(size=(2, 2, 128))).half().cuda()
    t, s, n = i32(torch, table), i32(torch, [0, 1, 2]), i32(torch, lengths)
    work = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")

    def calls():
        B.cache_append(pages, t, s, n, kv, kv, max_new=1)
        return [B.cache_attention(q, pages, t, s, n, max_new=1, max_len=1500, workspace=work), *B.cache_read(pages, t, s, 2, 128)]
    first = calls()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        second = calls()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            third = calls()
        for _ in range(3):
            for x in third:
                x.fill_(3)
            work.random_()
            stream.synchronize()
            graph.replay()
            stream.synchronize()
            for a, b, c in zip(first, second, third):
                assert torch.equal(a, b) and torch.equal(a, c)
