"""Sampling on the GPU against the binary64 oracle on the same random numbers: equal tokens, log-probabilities to 2e-5 (a sum of up to
70 000 fp32 terms and one logarithm)."""
import numpy as np
import pytest

from oracle import step

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


def check(env, logits, noise, **kw):
    torch, B = env
    dev = {n: None if v is None else torch.from_numpy(np.asarray(v, np.int32 if n == "top_k" else np.float32)).cuda() for n, v in kw.items()}
    token, logprob = B.sample(logits, noise, **dev)
    token, logprob = token.cpu().numpy(), logprob.cpu().numpy()
    x = logits.double().cpu().numpy()
    e = None if noise is None else noise.double().cpu().numpy()
    for r in range(len(x)):
        pick = lambda n, d: d if kw.get(n) is None else (int if n == "top_k" else lambda v: float(np.float32(v)))(kw[n][r])  # noqa: E731
        want = step.sample_row(x[r], None if e is None else e[r], pick("temperature", 1.0), pick("top_k", 0), pick("top_p", 1.0), pick("min_p", 0.0))
        assert token[r] == want[0], (r, token[r], want, {n: v[r] for n, v in kw.items() if v is not None})
        assert np.isnan(want[1]) == np.isnan(logprob[r]) and (np.isnan(want[1]) or abs(logprob[r] - want[1]) <= 2e-5)


def make(torch, rng, rows, vocab, dtype, spread=2.0):
    x = torch.from_numpy(rng.normal(size=(rows, vocab)) * spread + 9 * rng.random(size=(rows, vocab)) ** 40).to(dtype).cuda()
    return x, torch.from_numpy(rng.exponential(size=(rows, vocab)).astype(np.float32)).cuda()


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("vocab", [1, 2, 63, 1000, 1025, 32000, 50272, 70001])
def test_mixed_rows(env, vocab, dtype):
    torch, _ = env
    rng = np.random.default_rng(vocab)
    rows = 12
    x, e = make(torch, rng, rows, vocab, getattr(torch, dtype))
    check(env, x, e, temperature=rng.choice([0.0, 0.6, 1.0, 1.7], size=rows), top_k=rng.choice([0, 1, 5, 50, 3 * vocab // 4 + 1], size=rows),
          top_p=rng.choice([0.0, 0.3, 0.9, 0.999, 1.0], size=rows), min_p=rng.choice([0.0, 0.02, 0.5, 1.0], size=rows))
    check(env, x, e)
    check(env, x, e, top_p=np.full(rows, 0.8))
    check(env, x, e, top_k=np.arange(rows) * 17 % (vocab + 3))


@pytest.mark.parametrize("spread", [0.0, 0.05, 30.0])
def test_flat_and_sharp_rows(env, spread):
    torch, _ = env
    rng = np.random.default_rng(11)
    for dtype in (torch.float16, torch.float32):
        x, e = make(torch, rng, 6, 5000, dtype, spread)
        if spread < 1:
            x = (x - 9 * 0).clamp(-0.2, 0.2)
        check(env, x, e, top_k=[0, 7, 300, 0, 4000, 2], top_p=[0.5, 0.7, 0.9, 0.01, 1.0, 0.6])


def test_ties_go_to_the_lower_index(env):
    torch, _ = env
    rng = np.random.default_rng(12)
    x = torch.from_numpy(rng.integers(0, 4, size=(8, 3001)).astype(np.float32)).half().cuda()
    _, e = make(torch, rng, 8, 3001, torch.float16)
    check(env, x, e, temperature=[0, 1, 1, 1, 2, 1, 0.5, 1], top_k=[0, 3, 400, 1000, 2500, 0, 0, 10])
    check(env, torch.zeros_like(x), torch.ones_like(e), top_k=[0, 1, 2, 3, 64, 65, 1024, 3001])
    check(env, -torch.zeros_like(x) * (torch.arange(3001, device="cuda") % 2), e, top_k=[0, 1, 2, 3, 64, 65, 1024, 3001])


def test_masked_and_hopeless_rows(env):
    torch, _ = env
    rng = np.random.default_rng(13)
    x, e = make(torch, rng, 9, 4099, torch.float16)
    x[0, 100:] = -float("inf")                  # all but some masked, fewer than top_k
    x[1] = -float("inf")                        # nothing left
    x[2, 4098] = float("nan")
    x[3, 7] = float("inf")
    x[4, 1:] = -65504                           # masks of the type's lowest value
    x[5, :4098] = -float("inf")
    x[6] = -65504
    check(env, x, e, top_k=[200, 5, 5, 5, 5, 5, 9, 0, 0], top_p=[0.9] * 7 + [1.0, 1.0], temperature=[1, 1, 1, 1, 1, 1, 1, -1.0, float("nan")])
    check(env, x[4:9], e[4:9], temperature=[float("inf"), 1e-40, 2.0 ** -126, 1e30, 1e-3], top_p=[0.5] * 5)
    check(env, x[:7], None, temperature=[0.0] * 7)
    check(env, x[:2], None, temperature=[0.0, 1.0])


def test_strides_streams_and_graph(env):
    torch, B = env
    rng = np.random.default_rng(14)
    x, e = make(torch, rng, 5, 5001, torch.bfloat16)
    check(env, x[:, 3:4000], e[:, 5:4002], top_k=[0, 4, 0, 9, 1000], top_p=[0.5, 1, 0.9, 0.8, 0.99])
    check(env, x[::2], e[1:4], top_p=[0.5, 0.9, 0.8])
    p = torch.full((5,), 0.9, device="cuda")
    first = B.sample(x, e, top_p=p)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        second = B.sample(x, e, top_p=p)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            third = B.sample(x, e, top_p=p)
        for _ in range(3):
            for t in third:
                t.fill_(5)
            stream.synchronize()
            graph.replay()
            stream.synchronize()
            for a, b, c in zip(first, second, third):
                assert torch.equal(a, b) and torch.equal(a, c)
    token, logprob = B.sample(x[:0], e[:0])
    assert token.numel() == 0 and logprob.numel() == 0
