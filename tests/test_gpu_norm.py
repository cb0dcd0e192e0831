"""Residual sum with norms and its gradients on the GPU against the binary64 oracle.

Tolerances.  Results are rounded once: half a step, 2^-11 of the result in fp16 (2^-25 below its normal range), 2^-8 in bf16,
2^-24 in fp32.  Binary32's share: a sum over a row passes at most 16 additions in a thread, 6 across a wave's lanes, 4 across
waves, 26 of 2^-24 or 1.6e-6 of the sum of magnitudes; half of that in 1 / size; the mean's, against the deviation, counts
|mean| / deviation times.  With ten more operations per element 4e-6 (1 + |mean| / deviation) of the row's largest magnitude
covers the forward, and three times that the backward, whose terms pass two such sums more.  Sums over tokens add to that 64
additions (4e-6) of the sum of magnitudes."""
import numpy as np
import pytest

from oracle import ends

pytestmark = pytest.mark.gpu
HALF = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8, "float32": 2.0 ** -24}
EPS = 1e-5


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


CASES = [  # tokens, width, norm, post, gate, bias, p, dtype, fp32 residual, off the 16-byte grid
    (1, 1, "rms", None, None, False, 0.0, "float16", False, False),
    (1, 4096, "rms", None, None, False, 0.0, "float16", False, False),
    (3, 7, "layer", "layer", "row", True, 0.3, "float16", False, False),
    (2, 8, "layer", None, "token", True, 0.0, "bfloat16", True, False),
    (5, 100, "rms", "rms", "row", False, 0.1, "float16", True, True),
    (4, 511, "layer", "rms", None, True, 0.5, "bfloat16", False, True),
    (9, 512, None, "layer", "token", True, 0.1, "float16", False, False),
    (6, 513, "rms", "layer", "row", True, 0.0, "bfloat16", False, True),
    (700, 64, "layer", "rms", "row", True, 0.2, "float16", False, False),
    (1300, 96, "rms", None, None, True, 0.1, "bfloat16", True, False),
    (33, 1003, "layer", None, "row", False, 0.25, "float16", False, True),
    (2, 5003, "rms", "rms", "token", True, 0.1, "bfloat16", False, False),
    (3, 8191, "layer", "layer", "row", True, 0.0, "float16", False, True),
    (2, 8193, "rms", "layer", "row", True, 0.1, "float16", True, True),
    (5, 9216, "layer", "rms", "row", True, 0.1, "bfloat16", False, False),
    (2, 12288, "layer", "layer", "row", True, 0.0, "float16", False, False),
    (3, 16384, "rms", "rms", "token", False, 0.1, "bfloat16", True, False),
    (2, 16383, "layer", "layer", "row", True, 0.1, "float16", True, True),
    (1, 16384, "layer", None, None, True, 0.0, "float16", False, False),
]


class Case:
    def __init__(self, env, case, seed, backward=False):
        torch, self.B = env
        self.torch = torch
        tokens, width, self.norm, self.post, gate, bias, self.p, dtype, h32, off = case
        self.dtype, self.h_dtype = dtype, "float32" if h32 else dtype
        rng = np.random.default_rng(seed)

        def dev(a, dtype=dtype):
            a = np.asarray(a)
            t = torch.from_numpy(a).to(getattr(torch, dtype))
            if off and a.ndim == 2:              # rows that begin anywhere
                wide = torch.zeros(a.shape[0], a.shape[1] + 3, dtype=t.dtype)
                wide[:, 1:1 + a.shape[1]] = t
                return wide.cuda()[:, 1:1 + a.shape[1]]
            return t.cuda()
        size = rng.choice([0.02, 1.0, 40.0], size=(tokens, 1))
        columns = np.where(rng.random(width) < 0.01, 15.0, 1.0)
        self.h = dev(rng.normal(size=(tokens, width)) * size * columns + 0.5, self.h_dtype)
        self.branch = dev(rng.normal(size=(tokens, width)) * rng.choice([0.1, 1.0], size=(tokens, 1)) - 0.2)
        self.gate = None if gate is None else dev(0.5 + rng.normal(size=width if gate == "row" else (tokens, width)))
        vec = lambda there, about: dev(about + 0.3 * rng.normal(size=width)) if there else None  # noqa: E731
        self.w, self.b = vec(self.norm, 1), vec(self.norm and bias, 0)
        self.pw, self.pb = vec(self.post, 1), vec(self.post and bias, 0)
        self.rng = torch.tensor([seed * 977 - 10 ** 12, 41], dtype=torch.int64, device="cuda")
        self.drop = ends.factor((seed * 977 - 10 ** 12, 41), self.p, 6, tokens, width) if self.p else None
        self.options = dict(gate=self.gate, post=self.post, post_weight=self.pw, post_bias=self.pb, norm=self.norm, weight=self.w, bias=self.b,
                            h_scale=1.25, branch_scale=0.6, eps=EPS, rng=self.rng, p=self.p, site=6)
        if backward:
            self.dy = dev(0.1 * rng.normal(size=(tokens, width))) if self.norm else None
            self.dtotal = dev(0.1 * rng.normal(size=(tokens, width)), self.h_dtype)

    def forward(self, **more):
        return self.B.residual_norm(self.h, self.branch, **self.options, **more)

    def want(self):
        return ends.residual_norm(host(self.h), host(self.branch), host(self.gate), self.post, host(self.pw), host(self.pb), self.norm, host(self.w),
                                  host(self.b), 1.25, 0.6, EPS, self.drop)

    def backward(self, **more):
        return self.B.residual_norm_backward(self.dy, self.dtotal, self.h, self.branch, **self.options, **more)

    def want_backward(self):
        return ends.residual_norm_backward(host(self.dy), host(self.dtotal), host(self.h), host(self.branch), host(self.gate), self.post, host(self.pw),
                                           host(self.pb), self.norm, host(self.w), 1.25, 0.6, EPS, self.drop)


def spread(x, kind):
    """1 + |mean| / deviation of every row, for a norm that takes the mean off."""
    return 1 + (np.abs(x.mean(-1, keepdims=True)) / np.sqrt(x.var(-1, keepdims=True) + EPS) if kind == "layer" else 0 * x[:, :1])


def close(got, want, dtype, slack):
    assert got.shape == want.shape
    size = np.abs(want).max(-1, keepdims=True)
    tol = HALF[dtype] * np.abs(want) + slack * size + (2.0 ** -25 if dtype == "float16" else 0)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward(env, case):
    c = Case(env, case, 1)
    total, y = c.forward()
    want_total, want_y = c.want()
    slack = 4e-6 * spread(host(c.branch), c.post)
    terms = np.abs(1.25 * host(c.h)).max(-1, keepdims=True) + np.abs(want_total - 1.25 * host(c.h)).max(-1, keepdims=True)
    close(host(total), want_total, c.h_dtype, slack * terms / np.abs(want_total).max(-1, keepdims=True))
    if c.norm is None:
        assert y is None
    else:
        n = spread(want_total, c.norm)
        deviation = np.sqrt((want_total.var(-1, keepdims=True) if c.norm == "layer" else (want_total ** 2).mean(-1, keepdims=True)) + EPS)
        # what the total is off by counts against its deviation, times the weight
        carried = slack * terms / deviation * np.abs(host(c.w)).max() / np.abs(want_y).max(-1, keepdims=True)
        close(host(y), want_y, c.dtype, 4e-6 * n + carried)


@pytest.mark.parametrize("case", CASES, ids=str)
def test_backward(env, case):
    c = Case(env, case, 2, backward=True)
    dh, dbranch, dgate, dpw, dpb, dw, db = (host(t) for t in c.backward())
    want = c.want_backward()
    n = spread(host(c.h), c.norm)
    pn = spread(host(c.branch), c.post)
    # the sum that dh ends with may cancel: both its parts count
    part = np.abs(host(c.dtotal)).max(-1, keepdims=True) + np.abs(want["h"] / 1.25 - host(c.dtotal)).max(-1, keepdims=True)
    off = 1.2e-5 * n * part * 1.25
    close(dh, want["h"], c.h_dtype, off / np.abs(want["h"]).max(-1, keepdims=True))
    # through the gate, the dropping and the branch's norm: relative to the row's gradient there
    e = 0.6 * np.abs(want["h"] / 1.25)
    g = 1.0 if c.gate is None else np.abs(host(c.gate))
    stay = 1.0 if c.drop is None else c.drop.max()
    q = e * g * stay * (1.0 if c.pw is None else np.abs(host(c.pw)))
    if c.post:
        x, r = ends.normalised(host(c.branch), c.post, EPS)
        q = (q + np.abs(x) * (q * np.abs(x)).mean(-1, keepdims=True) + q.mean(-1, keepdims=True)) * r
    v = g * stay * 0.6 * off / 1.25 * (1.0 if c.pw is None else np.abs(host(c.pw)).max()) * (r * (1 + np.abs(x).max(-1, keepdims=True) ** 2) if c.post else 1.0)
    tol = 1.2e-5 * pn * q.max(-1, keepdims=True) + np.broadcast_to(v, dbranch.shape).max(-1, keepdims=True)
    close(dbranch, want["branch"], c.dtype, tol / np.maximum(np.abs(want["branch"]).max(-1, keepdims=True), 1e-30))
    assert (dgate is None) == (c.gate is None)
    u = ends.norm(host(c.branch), c.post, host(c.pw), host(c.pb), EPS)
    u_off = (4e-6 * pn * np.abs(u).max(-1, keepdims=True)) * stay
    if c.gate is not None and c.gate.dim() == 2:
        tol = 1e-6 * np.abs(want["gate"]).max(-1, keepdims=True) + (e * u_off + 0.6 * off / 1.25 * np.abs(u) * stay).max(-1, keepdims=True)
        close(dgate, want["gate"], c.dtype, tol / np.maximum(np.abs(want["gate"]).max(-1, keepdims=True), 1e-30))
    elif c.gate is not None:
        tol = 8e-6 * np.abs(want["gate"]).sum(0) + (e * u_off + 0.6 * off / 1.25 * np.abs(u) * stay).sum(0)
        assert (np.abs(dgate - want["gate"].sum(0)) <= tol).all()

    def sums(got, terms, row_off):
        assert (got is None) == (terms is None)
        if got is not None:
            assert (np.abs(got - terms.sum(0)) <= 8e-6 * np.abs(terms).sum(0) + row_off.sum(0) + 1e-30).all()
    there = lambda k, x: want[k] if x is not None else None  # noqa: E731
    if c.norm:
        x, _ = ends.normalised(host(c.h), c.norm, EPS)
        sums(dw, there("w", c.w), np.abs(host(c.dy)) * 4e-6 * n * np.abs(x).max(-1, keepdims=True))
        sums(db, there("b", c.b), 0 * x)
    if c.post:
        x, _ = ends.normalised(host(c.branch), c.post, EPS)
        dv = 0.6 * off / 1.25 * g * stay
        sums(dpw, there("post_w", c.pw), np.abs(want["post_b"]) * 4e-6 * pn * np.abs(x).max(-1, keepdims=True) + dv * np.abs(x))
        sums(dpb, there("post_b", c.pb), dv + 0 * x)


def test_gradients_against_differences(env):
    # fp32 residual: its output carries no 16-bit rounding, so that differences of it show the gradients of the branch and the gate
    c = Case(env, (6, 40, None, "layer", "row", True, 0.2, "float16", True, False), 3, backward=True)
    torch = c.torch
    dh, dbranch, dgate, dpw, dpb, _, _ = c.backward()
    f = lambda: (c.forward()[0].double() * c.dtotal.double()).sum().item()  # noqa: E731
    noise = 6 * 40 * 2.0 ** -23 * c.h.abs().max().item() * 0.4 * 2

    def difference(x, at, step):
        old = x[at].item()
        x[at] = old + step
        hi, up = x[at].item(), f()
        x[at] = old - step
        lo, down = x[at].item(), f()
        x[at] = old
        return (up - down) / (hi - lo), noise / (hi - lo)
    for x, g, at in ((c.gate, dgate, 3), (c.gate, dgate, 39), (c.pw, dpw, 0), (c.pb, dpb, 17), (c.h, dh, (2, 5))):      # linear ones: a wide step
        got, n = difference(x, at, 0.5)
        assert abs(got - g[at].item()) < n + 1e-5 * g.abs().max().item(), at
    for at in ((0, 0), (3, 20), (5, 39)):
        step = 0.02 * c.branch[at[0]].float().std().item()
        got, n = difference(c.branch, at, step)
        # the third derivative's share: (step / deviation)^2, of the row's largest gradient; half a step of the gradient itself
        assert abs(got - dbranch[at].item()) < n + (0.0004 + 2.0 ** -11) * dbranch[at[0]].abs().max().item() * 2, at


def test_without_a_branch_and_without_outputs(env):
    torch, B = env
    h = (torch.randn(5, 777, device="cuda") * 3).half()
    w = (1 + 0.1 * torch.randn(777, device="cuda")).half()
    total, y = B.residual_norm(h, weight=w, eps=EPS)
    assert torch.equal(total, h)
    close(host(y), ends.norm(host(h), "rms", host(w), None, EPS), "float16", 4e-6)
    none, y2 = B.residual_norm(h, weight=w, eps=EPS, want_total=False)
    assert none is None and torch.equal(y, y2)
    branch = torch.randn(5, 777, device="cuda").half()
    total, none = B.residual_norm(h, branch, norm=None)
    assert none is None
    close(host(total), host(h) + host(branch), "float16", 1e-6)
    dy = torch.randn(5, 777, device="cuda").half()
    dh, *rest = B.residual_norm_backward(dy, None, h, weight=w, eps=EPS)
    want = ends.residual_norm_backward(host(dy), None, host(h), None, None, None, None, None, "rms", host(w), 1.0, 1.0, EPS)
    close(host(dh), want["h"], "float16", 1.2e-5)
    assert [r is None for r in rest] == [True] * 4 + [False, True]
    # a gradient of the sum alone
    dh, dbranch, *_, dw, db = B.residual_norm_backward(None, dy, h, branch, weight=w, h_scale=2.0, branch_scale=0.5, eps=EPS)
    assert torch.equal(dh, dy * 2) and torch.equal(dbranch, dy * 0.5) and (dw == 0).all() and db is None
    # nothing comes in: nothing comes out
    dh, dbranch, *_ = B.residual_norm_backward(None, None, h, branch, weight=w, eps=EPS)
    assert (dh == 0).all() and (dbranch == 0).all()


def test_in_place_and_no_tokens(env):
    for case in ((37, 1003, "layer", "rms", "row", True, 0.2, "float16", False, False), (5, 9216, "rms", None, None, False, 0.1, "bfloat16", False, False)):
        c = Case(env, case, 5, backward=True)
        torch, B = env
        total, y = c.forward()
        grads = c.backward()
        h, branch = c.h.clone(), c.branch.clone()
        got = B.residual_norm(h, branch, **c.options, out=(h, branch))
        assert got[0] is h and torch.equal(h, total) and torch.equal(branch, y)
        empty = [t[:0] for t in (c.dy, c.dtotal, c.h, c.branch)]
        total, y = B.residual_norm(empty[2], empty[3], **c.options)
        assert total.shape == y.shape == (0, c.h.shape[1])
        none = B.residual_norm_backward(*empty, **c.options)
        assert none[0].shape == (0, c.h.shape[1])
        for g, n in zip(grads[2:], none[2:]):
            assert (g is None) == (n is None) and (n is None or (n.shape == g.shape and (n == 0).all()))


def test_what_is_not_finite_stays_in_its_row(env):
    c = Case(env, (6, 300, "layer", "rms", None, True, 0.0, "float16", False, False), 6, backward=True)
    total, y = c.forward()
    grads = c.backward()
    c.h[1, 7], c.branch[3, 299] = float("nan"), float("inf")
    total2, y2 = c.forward()
    keep = [0, 2, 4, 5]
    assert c.torch.equal(total[keep], total2[keep]) and c.torch.equal(y[keep], y2[keep])
    assert not host(y2)[1].any() or np.isnan(host(y2)[1]).all()
    assert np.isnan(host(y2)[[1, 3]]).all()
    again = c.backward()
    for a, b in zip(grads[:2], again[:2]):
        assert c.torch.equal(a[keep], b[keep])


def test_rows_of_zeros_and_a_large_offset(env):
    torch, B = env
    h = torch.zeros(3, 640, device="cuda").half()
    h[1] = 1000
    h[2] = (1000 + torch.randn(640, device="cuda")).half()
    for kind in ("rms", "layer"):
        y = host(B.residual_norm(h, norm=kind, eps=EPS)[1])
        want = ends.norm(host(h), kind, None, None, EPS)
        assert (y[0] == 0).all()
        if kind == "layer":
            # a constant row's deviation is 0: what is left of the mean's rounding, 26 2^-24 of 1000, over sqrt(eps)
            assert np.abs(y[1]).max() <= 1.6e-6 * 1000 / np.sqrt(EPS)
            close(y[2:], want[2:], "float16", 4e-6 * spread(host(h)[2:], kind))
        else:
            close(y[1:], want[1:], "float16", 4e-6)


def test_same_bits_twice_on_another_stream_and_in_a_graph(env):
    for case in ((300, 1024, "layer", "rms", "row", True, 0.1, "bfloat16", False, False), (70, 9216, "rms", "layer", "row", True, 0.1, "float16", True, False)):
        c = Case(env, case, 7, backward=True)
        torch, B = env
        work = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
        calls = lambda: [*c.forward(), *(t for t in c.backward(workspace=work) if t is not None)]  # noqa: E731
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
                for a, b, d in zip(first, second, third):
                    assert torch.equal(a, b) and torch.equal(a, d)


def test_more_tokens_than_workgroups_in_turn(env):
    # more rows than a launch has workgroups: rows in turn
    torch, B = env
    h = torch.randn(70001, 16, device="cuda").half()
    y = host(B.residual_norm(h, eps=EPS)[1])
    close(y, ends.norm(host(h), "rms", None, None, EPS), "float16", 4e-6)


@pytest.mark.parametrize("post,gate", [(None, None), ("layer", None), ("rms", "row"), (None, "token")])
def test_teams_without_a_row_add_nothing(env, post, gate):
    # two teams a workgroup and an odd number of rows: the last team has none, and without eps a row of zeros is no number
    torch, B = env
    g = torch.Generator("cuda").manual_seed(9)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").half()  # noqa: E731
    rows, width = 301, 72
    total, branch, dy, dt = (rand(rows, width) for _ in range(4))
    options = dict(gate=None if gate is None else rand(width) if gate == "row" else rand(rows, width), post=post, post_weight=rand(width) if post else None,
                   norm="layer", weight=rand(width), bias=rand(width), eps=0.0)
    _, dbranch, dgate, dpw, _, dw, db = B.residual_norm_backward(dy, dt, total, branch, **options)
    want = ends.residual_norm_backward(host(dy), host(dt), host(total), host(branch), host(options["gate"]), post, host(options["post_weight"]), None,
                                       "layer", host(options["weight"]), 1.0, 1.0, 0.0)
    for got, terms in ((dw, want["w"]), (db, want["b"]), (dpw, want.get("post_w")), (dgate if gate == "row" else None, want.get("gate"))):
        if got is not None:
            # against the terms' sizes: twelve roundings of a row's statistics and sums (2^-24 each) and 64 additions
            assert (np.abs(host(got) - terms.sum(0)) <= 1.2e-5 * np.abs(terms).max(1, keepdims=True).sum(0) * np.ones(width) + 1e-5 * np.abs(terms).sum(0)).all()
    assert torch.isfinite(dbranch).all()


def test_offsets_past_32_bits(env):
    # rows that lie further apart than 2^31 bytes: bit for bit what packed rows give
    torch, B = env
    rows, width, stride = 4, 200, 2 ** 30 + 3

    def far():
        return torch.zeros((rows - 1) * stride + width, dtype=torch.float16, device="cuda").as_strided((rows, width), (stride, 1)).normal_()
    h, branch = far(), far()
    w = (1 + 0.1 * torch.randn(width, device="cuda")).half()
    key = torch.tensor([1, 2], dtype=torch.int64, device="cuda")
    options = dict(norm="layer", weight=w, post="rms", rng=key, p=0.2)
    got = B.residual_norm(h, branch, **options)
    want = B.residual_norm(h.contiguous(), branch.contiguous(), **options)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    got = B.residual_norm_backward(branch, h, h, branch, **options)
    packed = h.contiguous(), branch.contiguous()
    want = B.residual_norm_backward(packed[1], packed[0], packed[0], packed[1], **options)
    for a, b in zip(got, want):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b))
    assert torch.equal(B.dropout(h, key, 0.3, residual=branch), B.dropout(packed[0], key, 0.3, residual=packed[1]))
