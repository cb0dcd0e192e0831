"""Head norm with rotation and its gradients on the GPU against the binary64 oracle.

Tolerances.  Outputs are rounded once: half a unit in the last place of the result (2^-11 of it in fp16, 2^-8 in bf16,
2^-25 in the subnormal range of fp16) plus binary32's share, 16 operations of 2^-24 on values of the row's size: 1e-6 of the row's
largest magnitude (4e-6 in the backward, whose terms cancel).  Gradients of the weights are fp32 sums: 2e-6 of the sum of magnitudes.
"""
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


def tables(n, rot):
    a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(rot // 2) / (rot // 2))
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def host(t):
    return t.detach().double().cpu().numpy()


def close(got, want, bf16, slack):
    assert got.shape == want.shape
    nan = np.isnan(want)
    assert (np.isnan(got) == nan).all()
    size = np.nanmax(np.where(nan, 0, np.abs(want)), axis=-1, keepdims=True)
    tol = (2.0 ** -8 if bf16 else 2.0 ** -11) * np.abs(want) + slack * size + 2.0 ** -25
    bad = ~(np.abs(got - want) <= tol) & ~nan
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


CASES = [  # tokens, q heads, kv heads, dim, rotary, interleaved, weights, bf16
    (1, 1, 1, 16, 16, False, "qk", False), (1, 40, 40, 128, 128, False, "", False), (3, 32, 8, 128, 128, True, "qk", False),
    (5, 12, 12, 64, 32, False, "qk", True), (33, 5, 5, 80, 80, False, "q", False), (7, 7, 1, 80, 32, True, "k", True),
    (2, 3, 2, 256, 256, False, "qk", True), (9, 4, 4, 256, 128, True, "qk", False), (4, 6, 3, 24, 16, False, "qk", False),
    (1, 72, 72, 128, 64, False, "", True), (700, 9, 2, 96, 96, False, "qk", False), (6, 1, 0, 48, 48, True, "qk", False),
    (130, 33, 31, 248, 16, False, "qk", True), (2500, 2, 1, 32, 32, False, "qk", False),
]


def make(env, tokens, hq, hk, dim, rot, weights, bf16, seed, slices):
    torch, _ = env
    rng = np.random.default_rng(seed)
    dtype = torch.bfloat16 if bf16 else torch.float16
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()  # noqa: E731
    x = dev(rng.normal(size=(tokens, hq + 2 * hk + 1, dim)) * rng.choice([1e-3, 1.0, 30.0], size=(tokens, 1, 1)))
    q, k = x[:, :hq], x[:, hq:hq + hk]
    if not slices:
        q, k = q.contiguous(), k.contiguous()
    w = dev(1 + 0.3 * rng.normal(size=(2, dim)))
    n = tokens + 17
    cos, sin = tables(n, rot)
    pos = rng.integers(0, n, size=tokens).astype(np.int32)
    return rng, dev, q, k, w[0] if "q" in weights else None, w[1] if "k" in weights else None, cos, sin, pos


@pytest.mark.parametrize("slices", [False, True])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward(env, case, slices):
    torch, B = env
    tokens, hq, hk, dim, rot, inter, weights, bf16 = case
    rng, dev, q, k, wq, wk, cos, sin, pos = make(env, tokens, hq, hk, dim, rot, weights, bf16, 1, slices)
    got = B.qk_norm_rope(q, k, torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), torch.from_numpy(pos).cuda(), wq, wk, 1e-6, inter)
    torch.cuda.synchronize()
    for x, w, y in ((q, wq, got[0]), (k, wk, got[1])):
        if x.shape[1]:
            close(host(y), step.norm_rope(host(x), None if w is None else host(w), cos, sin, pos, 1e-6, inter), bf16, 1e-6)


@pytest.mark.parametrize("slices", [False, True])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_backward(env, case, slices):
    torch, B = env
    tokens, hq, hk, dim, rot, inter, weights, bf16 = case
    rng, dev, q, k, wq, wk, cos, sin, pos = make(env, tokens, hq, hk, dim, rot, weights, bf16, 2, slices)
    dy = dev(0.1 * rng.normal(size=(tokens, hq + 3 * hk, dim)))
    dq, dk = dy[:, :hq], dy[:, hq + hk:hq + 2 * hk]
    got = B.qk_norm_rope_backward(dq, dk, q, k, torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), torch.from_numpy(pos).cuda(),
                                  wq, wk, 1e-6, inter)
    torch.cuda.synchronize()
    for d, x, w, dx, dw in ((dq, q, wq, got[0], got[2]), (dk, k, wk, got[1], got[3])):
        if not x.shape[1]:
            continue
        want, want_w, terms = step.norm_rope_backward(host(d), host(x), None if w is None else host(w), cos, sin, pos, 1e-6, inter)
        close(host(dx), want, bf16, 4e-6)
        assert (dw is None) == (w is None)
        if w is not None:
            assert (np.abs(host(dw) - want_w) <= 2e-6 * terms + 1e-30).all()


def test_gradients_against_differences(env):
    # the kernel's own forward, differenced in fp16-exact steps along one element, against its backward
    torch, B = env
    rng = np.random.default_rng(3)
    cos, sin = (torch.from_numpy(t).cuda() for t in tables(40, 64))
    pos = torch.arange(8, dtype=torch.int32).cuda()
    q, k = (torch.from_numpy(rng.normal(size=(8, 2, 64))).half().cuda() for _ in range(2))
    w = torch.from_numpy(1 + 0.2 * rng.normal(size=64)).half().cuda()
    dy = torch.from_numpy(rng.normal(size=(8, 2, 64))).half().cuda()
    dq, _, dwq, _ = B.qk_norm_rope_backward(dy, torch.zeros_like(dy), q, k, cos, sin, pos, w, None)
    f = lambda x, w: (B.qk_norm_rope(x, k, cos, sin, pos, w, None)[0].double() * dy.double()).sum().item()  # noqa: E731
    step_, noise = 0.25, 2.0 ** -12 * 3 * np.sqrt(128) * 4        # rounding of 64 outputs on either side, four sigma
    for at in [(0, 0, 0), (3, 1, 20), (7, 0, 63)]:
        up, down = q.clone(), q.clone()
        up[at] += step_
        down[at] -= step_
        width = (up[at] - down[at]).item()
        # the third derivative's share of a step of 1/4 on a row of norm sqrt(64): below 1 % of the row's largest gradient
        assert abs((f(up, w) - f(down, w)) / width - dq[at].item()) < noise / width + 0.01 * dq[at[0], at[1]].abs().max().item()
    for j in (0, 33, 63):
        up, down = w.clone(), w.clone()
        up[j] += step_
        down[j] -= step_
        width = (up[j] - down[j]).item()
        assert abs((f(q, up) - f(q, down)) / width - dwq[j].item()) < noise * 4 / width


def test_positions_outside_the_table_and_in_place(env):
    torch, B = env
    rng, dev, q, k, wq, wk, cos, sin, pos = make(env, 6, 4, 2, 64, 32, "qk", False, 4, False)
    pos[:] = [0, -1, 22, 23, 2 ** 31 - 1, -2 ** 31]
    want = step.norm_rope(host(q), host(wq), cos, sin, pos, 1e-6, False), step.norm_rope(host(k), host(wk), cos, sin, pos, 1e-6, False)
    args = (torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), torch.from_numpy(pos).cuda(), wq, wk)
    B.qk_norm_rope(q, k, *args, out=(q, k))
    torch.cuda.synchronize()
    close(host(q), want[0], False, 1e-6)
    close(host(k), want[1], False, 1e-6)
    empty = q[:0]
    out = B.qk_norm_rope(empty, k[:0], *args)
    assert out[0].shape == (0, 4, 64)
    grads = B.qk_norm_rope_backward(empty, k[:0], empty, k[:0], *args)
    torch.cuda.synchronize()
    assert (host(grads[2]) == 0).all() and (host(grads[3]) == 0).all()


def test_zero_rows_and_infinities_stay_in_their_row(env):
    torch, B = env
    rng, dev, q, k, wq, wk, cos, sin, pos = make(env, 4, 3, 1, 128, 128, "qk", False, 5, False)
    q[1, 0] = 0
    q[2, 1, 5] = float("inf")
    args = (torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), torch.from_numpy(pos).cuda(), wq, wk)
    y = host(B.qk_norm_rope(q, k, *args)[0])
    assert (y[1, 0] == 0).all() and np.isfinite(np.delete(y.reshape(12, -1), 7, 0)).all() and not np.isfinite(y[2, 1]).all()


def test_same_bits_twice_on_another_stream_and_in_a_graph(env):
    torch, B = env
    rng, dev, q, k, wq, wk, cos, sin, pos = make(env, 300, 12, 4, 128, 128, "qk", True, 6, False)
    dy, dk = dev(rng.normal(size=(300, 12, 128))), dev(rng.normal(size=(300, 4, 128)))
    args = (torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), torch.from_numpy(pos).cuda(), wq, wk)
    work = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")

    def calls():
        return [*B.qk_norm_rope(q, k, *args), *B.qk_norm_rope_backward(dy, dk, q, k, *args, workspace=work)]
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
            work.random_()
            stream.synchronize()
            graph.replay()
            stream.synchronize()
            for a, b, c in zip(first, second, third):
                assert torch.equal(a, b) and torch.equal(a, c)
