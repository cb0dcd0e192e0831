"""Log-probabilities of many rows, which the launch rule gives to fewer threads each: 64 to 512, with alternatives 256.  By the check of
test_gpu_logprob.py, with a tolerance for these launches.

Steps of u = 2^-24 relative to S: a batch of 16 logits a thread (8 of fp32 with alternatives) adds its terms by themselves, 16; every batch then
adds 1, and 4 where a thread's largest logit grew (a product and the exponential of a difference); what lies beside a row's units is a
batch more; the join 10 + 4 + 4; a term 2, and 3 |d| (`spread`)."""
import numpy as np
import pytest

import test_gpu_logprob as L
from test_gpu_logprob import U, env, host, make  # noqa: F401

pytestmark = pytest.mark.gpu


def threads_of(rows, vocab, top):
    if top:
        return 256 if rows > 512 and top <= (64 if vocab <= 8192 else 16) else 1024
    threads = 1024
    while threads > 64 and (threads * 16 > vocab or (threads > 128 and threads * rows > 2 ** 18)):
        threads //= 2
    return threads


def check(monkeypatch, B, x, targets, scale, top, threads, rows=None):
    """All rows, or those of a list, checked; rows of the launch decide the tolerance."""
    assert threads == threads_of(*x.shape, top)
    batch = threads * (8 if top and x.element_size() == 4 else 16)

    def rounding(want, vocab):
        s = (5 * (vocab // batch + 2) + 16 + 18 + 2) * U + 3 * U * want["spread"]
        return s, s + 2 * U * np.abs(want["stats"][1])
    monkeypatch.setattr(L, "rounding", rounding)
    got = B.token_logprobs(x, targets, scale, top)
    if rows is not None:
        got = [None if t is None else t[:, rows] if t.shape[0] == 3 and t.dim() == 2 and t.shape[1] == x.shape[0] else t[rows] for t in got]
        x, targets = x[rows], targets[rows]
    return L.check(got, x, targets, scale, top)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("rows,vocab,top,threads", [
    (600, 8192, 5, 256), (513, 8192, 64, 256), (600, 8193, 16, 256), (520, 32003, 16, 256), (600, 8192, 65, 1024), (600, 8193, 17, 1024),
    (512, 5000, 3, 1024), (4100, 300, 7, 256)])
def test_alternatives(env, monkeypatch, rows, vocab, top, threads, dtype):  # noqa: F811
    torch, B = env
    _, x, targets = make(torch, rows, vocab, dtype, rows + vocab, 1)
    some = list(range(0, rows, 1 + rows // 150)) + [rows - 1]
    check(monkeypatch, B, x, targets, 1.0, top, threads, some)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("rows,vocab,threads", [(2048, 50272, 128), (1025, 32003, 128), (768, 32000, 256), (300, 32003, 512), (5000, 1501, 64),
                                                (5000, 2049, 128), (2000, 1024, 64), (70, 12000, 512)])
def test_no_alternatives(env, monkeypatch, rows, vocab, threads, dtype):  # noqa: F811
    torch, B = env
    g = torch.Generator("cuda").manual_seed(rows)
    wide = 3 * torch.randn(rows, vocab + 3, generator=g, device="cuda")
    wide[: rows // 2] = wide[: rows // 2].sort(-1).values        # the largest grows from batch to batch
    x = wide.to(getattr(torch, dtype))[:, 2:2 + vocab]
    targets = torch.randint(-1, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    some = list(range(0, rows, 1 + rows // 24)) + [rows // 2 - 1, rows // 2, rows - 1]
    check(monkeypatch, B, x, targets, 1.0, 0, threads, some)


def kinds(torch, rows, vocab, dtype):
    """Rows by turns: masked in part or whole, ties, not finite."""
    _, x, targets = make(torch, rows, vocab, dtype, 8)
    x = x.contiguous()
    inf, lowest = float("inf"), torch.finfo(x.dtype).min
    x[0::14] = -inf
    x[1::14, 5:] = -inf
    x[2::14] = lowest
    x[3::14, 3:] = lowest
    x[4::14, vocab // 3] = float("nan")
    x[5::14, vocab - 1] = inf
    x[6::14, 1:] = -inf
    x[7::14] = 2.5                                                       # all equal
    x[8::14, ::2] = 4.0                                                  # many equal above others
    x[9::14] = (torch.arange(vocab, device="cuda") % 3).to(x.dtype)      # three values
    x[10::14] = torch.where(torch.arange(vocab, device="cuda") % 5 == 0, x[10::14], torch.full_like(x[10::14], -inf))
    x[11::14] = (torch.arange(vocab, device="cuda") // 300).to(x.dtype)  # runs of equal ones, the largest last
    x[12::14, -1] = 60.0                                                 # one far above
    targets[13::14] = -100
    return x, targets


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("rows,vocab,tops", [(602, 3001, (1, 7, 64)), (602, 20001, (1, 16)), (1103, 700, (5, 64)), (515, 263, (64,))])
def test_ties_and_masks_with_alternatives(env, monkeypatch, rows, vocab, tops, dtype):  # noqa: F811
    # more candidates than a list of 256 holds in the rows of equal logits
    torch, B = env
    x, targets = kinds(torch, rows, vocab, dtype)
    some = list(range(0, 42)) + list(range(rows - 15, rows))
    for top in tops:
        want = check(monkeypatch, B, x, targets, 1.0, top, 256, some)
        assert np.isnan(want["stats"][0][[0, 4, 5]]).all() and np.isfinite(want["stats"][:, [1, 2, 3, 6, 7, 8, 9, 10, 11, 12, 13]]).all()
        # all rows of a kind without random numbers in them are alike
        token = host(B.token_logprobs(x, targets, 1.0, top)[1])
        for kind in (0, 2, 7, 9, 11):
            assert (token[kind::14] == token[kind]).all(), kind


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("rows,vocab", [(1103, 3001), (1400, 20001)])
def test_masks_without_alternatives(env, monkeypatch, rows, vocab, dtype):  # noqa: F811
    torch, B = env
    x, targets = kinds(torch, rows, vocab, dtype)
    check(monkeypatch, B, x, targets, 0.5, 0, 128, list(range(0, 42)) + list(range(rows - 15, rows)))


def test_many_rows_twice_and_in_a_graph(env):  # noqa: F811
    torch, B = env
    x, targets = kinds(torch, 1200, 4001, "bfloat16")
    a = torch.rand(1200, device="cuda")

    def calls():
        lp, token, token_lp, stats = B.token_logprobs(x, targets, 1.0, 9)
        return [lp, token, token_lp, stats, *(t for t in B.token_logprobs(x, targets) if t is not None), B.token_logprobs_backward(a, a, x, targets, stats)]
    first = calls()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            captured = calls()
        for _ in range(3):
            for t in captured:
                t.fill_(7)
            stream.synchronize()
            graph.replay()
            stream.synchronize()
            for p, q in zip(first, captured):
                assert torch.equal(torch.nan_to_num(p.double(), 5.0, 6.0, 7.0), torch.nan_to_num(q.double(), 5.0, 6.0, 7.0))
