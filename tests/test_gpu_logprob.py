"""Log-probabilities of tokens, entropies, alternatives and the gradient on the GPU against the binary64 oracle.

Tolerances, in binary32 steps of u = 2^-24.  A term e^d carries the rounding of d = scale (x - m) in log2 units, 3 u |d|, and the
instruction's, 2 u; a thread adds up to vocab / 1024 of them one after the other and scales its sum when its maximum grows (at
most as often as it takes a batch of 16, 4 u each); 10 additions join the threads.  Relative to S that is
(vocab / 1024 (1 + 4 / 16) + 40) u and 3 u times the softmax's mean of |d| (`spread`); ln S adds 2 u |ln S|.  A log-probability
adds 3 u |d|.  W = sum e^d d has the same relative errors per term, weighted by |d|: W / S is off by that of S times spread, and
by 3 u times the mean of d^2."""
import numpy as np
import pytest

from oracle import ends

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8, "float32": 2.0 ** -24}


@pytest.fixture(scope="module")
def env():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2306_02272_amd import binding
    binding.lib()
    torch.cuda.set_device(0)
    return torch, binding


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


def make(torch, rows, vocab, dtype, seed, off=0, spread=3.0):
    rng = np.random.default_rng(seed)
    wide = torch.from_numpy(rng.normal(size=(rows, vocab + off + 2)) * spread).to(getattr(torch, dtype)).cuda()
    x = wide[:, off:off + vocab]
    targets = torch.from_numpy(rng.integers(0, vocab, size=rows).astype(np.int32)).cuda()
    return rng, x, targets


def rounding(want, vocab):
    s = (vocab / 1024 * 1.25 + 40) * U + 3 * U * want["spread"]
    log_s = s + 2 * U * np.abs(want["stats"][1])
    return s, log_s


def check(got, x, targets, scale, top):
    lp, token, token_lp, stats = (host(t) for t in got)
    want = ends.token_logprobs(host(x), None if targets is None else targets.cpu().numpy(), scale, top)
    vocab = x.shape[1]
    s, log_s = rounding(want, vocab)
    assert np.array_equal(np.isnan(stats), np.isnan(want["stats"]))
    ok = ~np.isnan(want["stats"][0])
    assert (stats[0][ok] == want["stats"][0][ok]).all()
    assert (np.abs(stats[1] - want["stats"][1]) <= log_s)[ok].all()
    assert (np.abs(stats[2] - want["entropy"]) <= log_s + s * (1 + want["spread"]) + 3 * U * want["spread2"])[ok].all()

    def near(got, want):
        fine = np.isfinite(want)
        assert np.array_equal(got[~fine], want[~fine], equal_nan=True)
        # d is the log-probability plus ln S
        l = np.broadcast_to((log_s + 2 * U * np.abs(stats[1]))[(...,) + (None,) * (want.ndim - 1)], want.shape)
        assert (np.abs(got[fine] - want[fine]) <= (l + 4 * U * np.abs(want))[fine]).all()
    if targets is None:
        assert lp is None
    else:
        near(lp, want["logprob"])
    if top:
        assert np.array_equal(token, want["top_token"])
        near(token_lp, want["top_logprob"])
    return want


SHAPES = [(1, 1), (3, 2), (2, 7), (5, 64), (1, 1000), (4, 1023), (3, 1025), (2, 8193), (2, 16391), (7, 32003), (2, 50272), (1, 131072), (1, 200001), (900, 40)]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(env, shape, dtype):
    torch, B = env
    for off, scale, top in ((0, 1.0, 0), (1, 1.0, 5), (3, 0.7, 20), (2, 1.9, 1)):
        _, x, targets = make(torch, *shape, dtype, sum(shape) + off, off)
        check(B.token_logprobs(x, targets, scale, top), x, targets, scale, top)
    check(B.token_logprobs(x, None, 1.0, 2), x, None, 1.0, 2)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_backward(env, shape, dtype):
    torch, B = env
    rows, vocab = shape
    for off, scale, parts in ((0, 1.0, "lh"), (1, 0.7, "l"), (3, 1.3, "h")):
        rng, x, targets = make(torch, rows, vocab, dtype, sum(shape) + off, off)
        targets[rows // 2] = (-100, vocab, 2 ** 31 - 1)[off % 3]
        a = torch.from_numpy(rng.normal(size=rows).astype(np.float32)).cuda() if "l" in parts else None
        h = torch.from_numpy(rng.normal(size=rows).astype(np.float32)).cuda() if "h" in parts else None
        t = targets if a is not None else None
        stats = B.token_logprobs(x, t, scale)[3]
        got = host(B.token_logprobs_backward(a, h, x, t, stats, scale))
        want, size = ends.token_logprobs_backward(host(a), host(h), host(x), None if t is None else t.cpu().numpy(), scale)
        full = ends.token_logprobs(host(x), None, scale, 0)
        s, log_s = rounding(full, vocab)
        entropy = log_s + s * (1 + full["spread"]) + 3 * U * full["spread2"]
        with np.errstate(divide="ignore"):
            d = scale * np.abs(host(x) - full["stats"][0][:, None])
        # p is off by that of ln S and of d, the entropy by its own, the operations by 8 u; 2^-126: the exponential of less is 0
        p = np.exp(-d - full["stats"][1][:, None])
        tol = HALF[dtype] * np.abs(want) + size * (log_s[:, None] + 6 * U * (d + 2) + 8 * U) * 1.5
        tol += scale * p * (0 if h is None else np.abs(host(h))[:, None] * (entropy[:, None] + 4 * U * (d + 1)))
        at = np.zeros_like(want)
        if t is not None:
            inside = (t.cpu().numpy() >= 0) & (t.cpu().numpy() < vocab)
            at[np.arange(rows)[inside], t.cpu().numpy()[inside]] = scale * np.abs(host(a))[inside]
        tol += 4 * U * at + (2.0 ** -25 if dtype == "float16" else 2.0 ** -120)
        bad = ~(np.abs(got - want) <= tol)
        assert not bad.any(), (off, np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], tol[bad][:5])


def test_gradients_against_differences(env):
    torch, B = env
    rng, x, targets = make(torch, 4, 50, "float32", 3, spread=1.0)
    x = x.contiguous()
    targets[1] = -1
    a, h = (torch.from_numpy(rng.normal(size=4).astype(np.float32)).cuda() for _ in range(2))
    stats = B.token_logprobs(x, targets, 0.8)[3]
    g = B.token_logprobs_backward(a, h, x, targets, stats, 0.8)

    def f():
        lp, _, _, stats = B.token_logprobs(x, targets, 0.8)
        return ((lp * a).double() + (stats[2] * h).double()).sum().item()
    for at in ((0, 0), (0, int(targets[0])), (1, 7), (3, 49)):
        old = x[at].item()
        x[at] = old + 0.03
        hi, up = x[at].item(), f()
        x[at] = old - 0.03
        lo, down = x[at].item(), f()
        x[at] = old
        # rounding of the outputs (a few of size 5) over the step; the third derivative's share, (0.03)^2 / 6 of at most 4
        assert abs((up - down) / (hi - lo) - g[at].item()) < 64 * U * 5 / 0.06 + 0.0006 * 4, at


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
def test_masked_and_unfinished_rows(env, dtype):
    torch, B = env
    rows, vocab = 12, 3001
    _, x, targets = make(torch, rows, vocab, dtype, 8)
    x = x.contiguous()
    lowest = torch.finfo(x.dtype).min
    x[0] = -float("inf")                                  # nothing left
    x[1, 5:] = -float("inf")                              # five left
    x[2] = lowest                                         # all at the type's lowest value
    x[3, 3:] = lowest
    x[4, 17] = float("nan")
    x[5, 2000] = float("inf")
    x[6, 1:] = -float("inf")                              # one left
    x[7] = 2.5                                            # all equal
    x[8, ::2] = 4.0                                       # many equal above others
    x[9, :] = torch.arange(vocab, device="cuda") % 3      # three values
    x[10] = float("inf")
    targets[:] = torch.arange(rows, dtype=torch.int32)
    targets[11] = -100
    for top in (0, 1, 7, 64, 512):
        for scale in (1.0, 0.25):
            want = check(B.token_logprobs(x, targets, scale, top), x, targets, scale, top)
    assert np.isnan(want["stats"][0][[0, 4, 5, 10]]).all() and np.isfinite(want["stats"][:, [1, 2, 3, 6, 7, 8, 9, 11]]).all()
    stats = B.token_logprobs(x, targets)[3]
    a = torch.ones(rows, device="cuda")
    h = torch.full((rows,), 0.5, device="cuda")
    a[4] = h[4] = 0                                       # not counted: 0 whatever the row holds
    got = host(B.token_logprobs_backward(a, h, x, targets, stats))
    want, _ = ends.token_logprobs_backward(host(a), host(h), host(x), targets.cpu().numpy(), 1.0)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and (got[4] == 0).all()
    ok = [1, 2, 3, 6, 7, 8, 9, 11]
    assert (np.abs(got[ok] - want[ok]) <= HALF[dtype] * np.abs(want[ok]) + 2e-5).all() and (got[1, 5:] == 0).all()
    # a masked token that is asked for keeps its 1 - p, all others of the row nothing
    assert (np.delete(got[6], [0, 6]) == 0).all() and got[6, 6] == 1
    out = x.clone()
    assert B.token_logprobs_backward(a, h, out, targets, stats, out=out) is out
    assert np.array_equal(host(out), got, equal_nan=True)


def test_ties_go_to_the_lower_index_in_every_way(env):
    torch, B = env
    # more equal logits than are listed (1024), in one row with some above them; alternatives in descending order
    for vocab, above in ((40000, 3), (5000, 0), (1500, 600)):
        x = torch.zeros(2, vocab, device="cuda", dtype=torch.bfloat16)
        x[0, torch.arange(above, device="cuda") * 2 + 1] = (8 - torch.arange(above, device="cuda") % 4).to(torch.bfloat16)
        x[1, 7:] = -1
        for top in (1, 6, 300, 512):
            check(B.token_logprobs(x, None, 1.0, top), x, None, 1.0, top)
    # minus zero equals zero
    x = torch.zeros(1, 64, device="cuda")
    x[0, ::2] = -0.0
    check(B.token_logprobs(x, None, 1.0, 10), x, None, 1.0, 10)


def test_offsets_of_all_logits_and_far_scales(env):
    torch, B = env
    _, x, targets = make(torch, 3, 5000, "float32", 4)
    x = x.contiguous()
    x = (x * 64).round() / 64                             # exact beside the offset
    base = B.token_logprobs(x, targets, 1.0, 4)
    far = B.token_logprobs(x + 65536.0, targets, 1.0, 4)
    for a, b in zip(base[:3], far[:3]):
        assert torch.equal(a, b)
    assert torch.equal(base[3][1:], far[3][1:])
    for scale in (1e-30, 1e-3, 40.0, 1e30):
        check(B.token_logprobs(x, targets, scale, 4), x, targets, scale, 4)


def test_offsets_past_32_bits(env):
    # rows that lie further apart than 2^31 bytes and elements: the last row by itself
    torch, B = env
    rows, vocab, stride = 5, 300, 2 ** 29 + 1
    store = torch.zeros(4 * stride + vocab, dtype=torch.bfloat16, device="cuda")
    x = store.as_strided((rows, vocab), (stride, 1))
    x.normal_()
    targets = torch.arange(rows, dtype=torch.int32, device="cuda")
    check(B.token_logprobs(x, targets, 1.0, 3), x, targets, 1.0, 3)
    stats = B.token_logprobs(x, targets)[3]
    a = torch.ones(rows, device="cuda")
    packed = x.contiguous()
    assert torch.equal(B.token_logprobs_backward(a, a, x, targets, stats), B.token_logprobs_backward(a, a, packed, targets, stats))


def test_same_bits_twice_on_another_stream_and_in_a_graph(env):
    torch, B = env
    rng, x, targets = make(torch, 40, 9001, "float16", 9)
    a = torch.from_numpy(rng.normal(size=40).astype(np.float32)).cuda()

    def calls():
        lp, token, token_lp, stats = B.token_logprobs(x, targets, 1.0, 12)
        return [lp, token, token_lp, stats, B.token_logprobs_backward(a, a, x, targets, stats)]
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
            for t in third:
                t.fill_(7)
            stream.synchronize()
            graph.replay()
            stream.synchronize()
            for p, q, r in zip(first, second, third):
                assert torch.equal(p, q) and torch.equal(p, r)


def test_no_rows(env):
    torch, B = env
    x = torch.empty(0, 100, device="cuda")
    t = torch.empty(0, dtype=torch.int32, device="cuda")
    lp, token, token_lp, stats = B.token_logprobs(x, t, 1.0, 3)
    assert lp.shape == (0,) and token.shape == (0, 3) and stats.shape == (3, 0)
    assert B.token_logprobs_backward(lp, lp, x, t, stats).shape == (0, 100)
