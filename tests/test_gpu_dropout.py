"""Dropout on the GPU against the binary64 oracle: the same elements stay, bit by bit, whatever the strides.

Tolerances.  The factor is rounded to binary32 (2^-24), as are the product and the sum; the result is rounded once: half a step,
2^-11 of it in fp16, 2^-8 in bf16, and 2^-25 in fp16's subnormal range.  In fp16 the nearest of 65520 = (65504 + 65536) / 2 and above is
infinity: an element times 65536 is, where p leaves so few."""
import numpy as np
import pytest

from oracle import ends

pytestmark = pytest.mark.gpu
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
    return t.detach().double().cpu().numpy()


def key(torch, seed, step):
    wrap = lambda v: v - 2 ** 64 if v >= 2 ** 63 else v  # noqa: E731
    return torch.tensor([wrap(seed), wrap(step)], dtype=torch.int64, device="cuda")


def check(got, x, res, f, dtype):
    want = ends.times(x, f) + (0 if res is None else res)
    size = np.abs(ends.times(x, f)) + (0 if res is None else np.abs(res))
    tol = HALF[dtype] * np.abs(want) + 4 * 2.0 ** -24 * size + (2.0 ** -25 if dtype == "float16" else 0)
    if dtype == "float16":
        over = np.abs(want) >= 65520 * (1 + 4 * 2.0 ** -24)
        assert (got[over] == np.sign(want[over]) * np.inf).all()
        got, want, tol = (np.where(over, 0.0, a) for a in (got, want, tol))
    assert (np.abs(got - want) <= tol).all()
    if res is None and not (dtype == "float16" and over.any()):
        assert ((got != 0) == ((f != 0) & (x != 0))).all()


CASES = [(1, 1), (1, 7), (1, 8), (3, 9), (5, 64), (2, 100), (33, 127), (40, 768), (7, 2048), (3, 2049), (2, 5003), (700, 24), (9000, 3), (1, 70001)]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("shape", CASES, ids=str)
def test_against_the_oracle(env, shape, dtype):
    torch, B = env
    rows, width = shape
    rng = np.random.default_rng(rows + width)
    t = lambda: torch.from_numpy(rng.normal(size=(rows, width + 3)) + 3).to(getattr(torch, dtype)).cuda()  # noqa: E731
    x, res = t(), t()
    for p, site, seed, step in ((0.1, 0, 1, 2), (0.5, 2 ** 31 - 1, 2 ** 64 - 3, 2 ** 40 + 5), (65535 / 65536, -1, 2 ** 33, 0), (0.0, 1, 0, 0)):
        f = ends.factor((seed, step), p, site, rows, width)
        # slices that begin off every boundary, and packed
        got = B.dropout(x[:, 1:1 + width], key(torch, seed, step), p, site)
        check(host(got), host(x[:, 1:1 + width]), None, f, dtype)
        xp, rp = x[:, :width].contiguous(), res[:, 2:2 + width]
        got = B.dropout(xp, key(torch, seed, step), p, site, residual=rp)
        check(host(got), host(xp), host(rp), f, dtype)


def test_in_place_without_rows_and_without_a_key(env):
    torch, B = env
    k = key(torch, 5, 6)
    x = torch.randn(17, 333, device="cuda").half()
    res = torch.randn(17, 333, device="cuda").half()
    want, want_sum = B.dropout(x, k, 0.3), B.dropout(x, k, 0.3, residual=res)
    y = x.clone()
    assert B.dropout(y, k, 0.3, out=y) is y and torch.equal(y, want)
    y = res.clone()
    B.dropout(x, k, 0.3, residual=y, out=y)
    assert torch.equal(y, want_sum)
    assert torch.equal(B.dropout(x, None, 0.0), x)
    assert B.dropout(x[:0], k, 0.3).shape == (0, 333) and B.dropout(x[:, :0], k, 0.3).shape == (17, 0)


def test_what_is_dropped_may_be_anything(env):
    torch, B = env
    k = key(torch, 9, 1)
    x = torch.full((4, 100), float("nan"), device="cuda")
    f = ends.factor((9, 1), 0.5, 3, 4, 100)
    got = host(B.dropout(x, k, 0.5, 3))
    assert (got[f == 0] == 0).all() and np.isnan(got[f > 0]).all()
    got = host(B.dropout(x, k, 0.5, 3, residual=torch.ones_like(x)))
    assert (got[f == 0] == 1).all()


def test_the_gradient_drops_the_same(env):
    # linear in x: the difference of two outputs is the gradient applied to the difference, up to fp32's rounding
    torch, B = env
    k = key(torch, 3, 3)
    x, dy = torch.randn(9, 55, device="cuda"), torch.randn(9, 55, device="cuda")
    dx = B.dropout(dy, k, 0.2, 4)
    step = torch.randn(9, 55, device="cuda")
    up, down = B.dropout(x + step, k, 0.2, 4), B.dropout(x - step, k, 0.2, 4)
    width = (x + step).double() - (x - step).double()
    assert abs(((up.double() - down.double()) * dy.double()).sum() - (dx.double() * width).sum()) < 1e-6 * (dx.double() * width).abs().sum() + 1e-6 * 500


def test_other_streams_and_graphs_with_a_step_that_moves(env):
    torch, B = env
    k = key(torch, 12, 0)
    x = torch.randn(130, 1000, device="cuda").to(torch.bfloat16)
    eager = []
    for step in range(3):
        k[1] = step
        eager.append(B.dropout(x, k, 0.1, 7).clone())
    assert not torch.equal(eager[0], eager[1])
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        k[1] = 0
        out = torch.empty_like(x)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            B.dropout(x, k, 0.1, 7, out=out)
            k[1].add_(1)
        for step in range(3):
            out.fill_(3)
            stream.synchronize()
            graph.replay()
            stream.synchronize()
            assert torch.equal(out, eager[step])
