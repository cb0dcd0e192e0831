"""What the entry points at the ends of a block and of a tuning step refuse, before anything reaches a GPU."""
import os

import pytest

B = pytest.importorskip("paper_2306_02272_amd.binding")
P = 4096                                         # any aligned address: every call here is refused, or has nothing to do
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return B.lib()


def status(f, *a):
    try:
        f(*a)
    except B.OwqError as e:
        return e.status
    return B.OWQ_OK


@pytest.mark.parametrize("kw,want", [
    (dict(n_rows=-1), B.OWQ_ERR_SHAPE), (dict(width=-1), B.OWQ_ERR_SHAPE), (dict(type=3), B.OWQ_ERR_TYPE), (dict(type=-1), B.OWQ_ERR_TYPE),
    (dict(p=-0.1), B.OWQ_ERR_SHAPE), (dict(p=1.0), B.OWQ_ERR_SHAPE), (dict(p=0.999999), B.OWQ_ERR_SHAPE), (dict(p=NAN), B.OWQ_ERR_SHAPE),
    (dict(x=0), B.OWQ_ERR_NULL), (dict(out=0), B.OWQ_ERR_NULL), (dict(rng=0), B.OWQ_ERR_NULL), (dict(x=P + 1), B.OWQ_ERR_BUFFER),
    (dict(residual=P + 1), B.OWQ_ERR_BUFFER), (dict(out=P + 1), B.OWQ_ERR_BUFFER), (dict(rng=P + 4), B.OWQ_ERR_BUFFER),
    (dict(x=P + 2, type=2), B.OWQ_ERR_BUFFER), (dict(n_rows=0, x=0, out=0), B.OWQ_OK), (dict(width=0, x=0, rng=0), B.OWQ_OK)])
def test_dropout(lib, kw, want):
    d = dict(x=P, residual=0, type=0, n_rows=2, width=16, x_row=16, residual_row=16, rng=P, p=0.5, site=0, out=P)
    d.update(kw)
    assert status(B.owq_dropout, *d.values()) == want


def norm(**kw):
    d = dict(n_tokens=2, width=64, type=0, h_type=0, post=1, norm=2, gate=1, site=0, eps=1e-6, h_scale=1.0, branch_scale=1.0, p=0.5, h_row=64,
             branch_row=64, gate_row=64, total_row=64, dy_row=64, dtotal_row=64)
    d.update(kw)
    return B.NormDesc(**d)


@pytest.mark.parametrize("kw,want", [
    (dict(n_tokens=-1), B.OWQ_ERR_SHAPE), (dict(width=0), B.OWQ_ERR_SHAPE), (dict(width=16385), B.OWQ_ERR_UNSUPPORTED), (dict(type=2), B.OWQ_ERR_TYPE),
    (dict(type=-1), B.OWQ_ERR_TYPE), (dict(h_type=1), B.OWQ_ERR_TYPE), (dict(type=1, h_type=0), B.OWQ_ERR_TYPE), (dict(h_type=3), B.OWQ_ERR_TYPE),
    (dict(post=3), B.OWQ_ERR_SHAPE), (dict(post=-1), B.OWQ_ERR_SHAPE), (dict(norm=3), B.OWQ_ERR_SHAPE), (dict(gate=3), B.OWQ_ERR_SHAPE),
    (dict(gate=-1), B.OWQ_ERR_SHAPE), (dict(eps=-1.0), B.OWQ_ERR_SHAPE), (dict(eps=NAN), B.OWQ_ERR_SHAPE), (dict(h_scale=NAN), B.OWQ_ERR_SHAPE),
    (dict(branch_scale=NAN), B.OWQ_ERR_SHAPE), (dict(p=1.0), B.OWQ_ERR_SHAPE), (dict(p=-1.0), B.OWQ_ERR_SHAPE), (dict(p=NAN), B.OWQ_ERR_SHAPE),
    (dict(n_tokens=0), B.OWQ_OK)])
def test_norm(lib, kw, want):
    d = norm(**kw)
    assert status(B.owq_residual_norm, d, *[P] * 10) == want
    if want != B.OWQ_OK:
        assert status(B.owq_residual_norm_backward_workspace_bytes, d) == want
        assert status(B.owq_residual_norm_backward, d, *[P] * 17, 1 << 30) == want


def test_norm_pointers(lib):
    names = ("h", "branch", "gate", "post_weight", "post_bias", "weight", "bias", "rng", "total", "y")
    for i, name in enumerate(names):
        a = [P] * 10
        a[i] = 0
        if name in ("h", "branch", "gate", "rng", "y"):
            assert status(B.owq_residual_norm, norm(), *a) == B.OWQ_ERR_NULL, name
        a[i] = P + 1
        assert status(B.owq_residual_norm, norm(), *a) == B.OWQ_ERR_BUFFER, name
    assert status(B.owq_residual_norm, norm(h_type=2), P + 2, *[P] * 9) == B.OWQ_ERR_BUFFER
    # no branch: nothing that acts on one
    for kw in (dict(post=0, gate=0), dict(post=0, p=0.0), dict(gate=0, p=0.0)):
        assert status(B.owq_residual_norm, norm(**kw), P, 0, *[P] * 8) == B.OWQ_ERR_NULL


def test_norm_backward_pointers(lib):
    names = ("dy", "dtotal", "total", "branch", "gate", "post_weight", "post_bias", "weight", "rng", "dh", "dbranch", "dgate", "dpost_weight",
             "dpost_bias", "dweight", "dbias", "workspace")
    need = B.owq_residual_norm_backward_workspace_bytes(norm())
    assert need >= 5 * 64 * 4 and B.owq_residual_norm_backward_workspace_bytes(norm(n_tokens=0)) == 0
    assert B.owq_residual_norm_backward_workspace_bytes(norm(post=0, norm=0, gate=2)) == 0
    for i, name in enumerate(names):
        a = [P] * 17
        a[i] = 0
        if name in ("total", "branch", "gate", "rng", "workspace"):
            assert status(B.owq_residual_norm_backward, norm(), *a, need) == B.OWQ_ERR_NULL, name
        a[i] = P + 1
        assert status(B.owq_residual_norm_backward, norm(), *a, need) == B.OWQ_ERR_BUFFER, name
    assert status(B.owq_residual_norm_backward, norm(), *[P] * 17, need - 1) == B.OWQ_ERR_BUFFER
    a = [P] * 17
    a[11] = P + 2                                # a row gate's gradient is fp32, a token gate's is not
    assert status(B.owq_residual_norm_backward, norm(), *a, need) == B.OWQ_ERR_BUFFER


@pytest.mark.parametrize("kw,want", [
    (dict(n_rows=-1), B.OWQ_ERR_SHAPE), (dict(vocab=0), B.OWQ_ERR_SHAPE), (dict(vocab=(1 << 24) + 1), B.OWQ_ERR_SHAPE), (dict(type=3), B.OWQ_ERR_TYPE),
    (dict(scale=0.0), B.OWQ_ERR_SHAPE), (dict(scale=-1.0), B.OWQ_ERR_SHAPE), (dict(scale=3e38), B.OWQ_ERR_SHAPE), (dict(scale=1e-39), B.OWQ_ERR_SHAPE), (dict(scale=INF), B.OWQ_ERR_SHAPE), (dict(scale=NAN), B.OWQ_ERR_SHAPE),
    (dict(logits=0), B.OWQ_ERR_NULL), (dict(stats=0), B.OWQ_ERR_NULL), (dict(logits=P + 1), B.OWQ_ERR_BUFFER), (dict(logits=P + 2, type=2), B.OWQ_ERR_BUFFER),
    (dict(targets=P + 2), B.OWQ_ERR_BUFFER), (dict(stats=P + 2), B.OWQ_ERR_BUFFER), (dict(n_rows=0, logits=0), B.OWQ_OK)])
def test_logprobs(lib, kw, want):
    d = dict(logits=P, type=0, n_rows=2, vocab=100, logits_row=100, targets=P, scale=1.0)
    d.update({k: v for k, v in kw.items() if k != "stats"})
    stats = kw.get("stats", P)
    assert status(B.owq_token_logprobs, *d.values(), 3, P, P, P, stats) == want
    assert status(B.owq_token_logprobs_backward, *d.values(), stats, P, P, P) == want


def test_logprobs_outputs(lib):
    front = (P, 0, 2, 100, 100, P, 1.0)
    for top, outs, want in ((-1, (P, P, P, P), B.OWQ_ERR_SHAPE), (513, (P, P, P, P), B.OWQ_ERR_SHAPE), (1, (0, P, P, P), B.OWQ_ERR_NULL),
                            (1, (P, 0, P, P), B.OWQ_ERR_NULL), (1, (P, P, 0, P), B.OWQ_ERR_NULL), (1, (P + 2, P, P, P), B.OWQ_ERR_BUFFER),
                            (1, (P, P + 2, P, P), B.OWQ_ERR_BUFFER), (1, (P, P, P + 2, P), B.OWQ_ERR_BUFFER)):
        assert status(B.owq_token_logprobs, *front, top, *outs) == want, (top, outs)
    back = (P, P, P, P)                          # stats, dlogprob, dentropy, dlogits
    assert status(B.owq_token_logprobs_backward, P, 0, 2, 100, 100, 0, 1.0, *back) == B.OWQ_ERR_NULL      # log-probabilities of no tokens
    for i, want in ((3, B.OWQ_ERR_NULL),):
        a = list(back)
        a[i] = 0
        assert status(B.owq_token_logprobs_backward, *front, *a) == want
    for i in range(4):
        a = list(back)
        a[i] = P + (1 if i == 3 else 2)
        assert status(B.owq_token_logprobs_backward, *front, *a) == B.OWQ_ERR_BUFFER, i
