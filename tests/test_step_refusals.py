"""What the entry points between two layers refuse, before anything reaches a GPU."""
import os

import pytest

B = pytest.importorskip("paper_2306_02272_amd.binding")
P = 4096                                         # any aligned address: every call here is refused, or has nothing to do


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


def rope(**kw):
    d = dict(n_tokens=2, q_heads=4, kv_heads=2, head_dim=64, rotary_dim=32, interleaved=0, type=0, n_positions=9, eps=1e-6, reserved=0,
             q_token=512, q_head=64, k_token=512, k_head=64, dq_token=512, dq_head=64, dk_token=512, dk_head=64)
    d.update(kw)
    return B.RopeDesc(**d)


@pytest.mark.parametrize("kw,want", [
    (dict(n_tokens=-1), B.OWQ_ERR_SHAPE), (dict(q_heads=0), B.OWQ_ERR_SHAPE), (dict(kv_heads=-1), B.OWQ_ERR_SHAPE),
    (dict(n_positions=0), B.OWQ_ERR_SHAPE), (dict(eps=-1.0), B.OWQ_ERR_SHAPE), (dict(eps=float("nan")), B.OWQ_ERR_SHAPE),
    (dict(type=2), B.OWQ_ERR_TYPE), (dict(type=-1), B.OWQ_ERR_TYPE), (dict(head_dim=264, rotary_dim=16), B.OWQ_ERR_UNSUPPORTED),
    (dict(head_dim=60), B.OWQ_ERR_UNSUPPORTED), (dict(rotary_dim=80), B.OWQ_ERR_UNSUPPORTED), (dict(rotary_dim=24), B.OWQ_ERR_UNSUPPORTED),
    (dict(rotary_dim=0), B.OWQ_ERR_UNSUPPORTED), (dict(q_token=516), B.OWQ_ERR_BUFFER), (dict(k_head=63), B.OWQ_ERR_BUFFER),
    (dict(n_tokens=0), B.OWQ_OK)])
def test_rope(lib, kw, want):
    d = rope(**kw)
    assert status(B.owq_qk_norm_rope, d, P, P, P, P, P, P, P, P, P) == want
    if want != B.OWQ_OK:
        assert status(B.owq_qk_norm_rope_backward, d, P, P, P, P, P, P, P, P, P, P, P, P, P, P, 1 << 20) == want


def test_rope_pointers(lib):
    d = rope()
    good = [P] * 9
    for i in range(9):
        a = list(good)
        a[i] = 0
        if i not in (2, 3):                      # the weights may be NULL
            assert status(B.owq_qk_norm_rope, d, *a) == B.OWQ_ERR_NULL, i
        a[i] = P + 2
        assert status(B.owq_qk_norm_rope, d, *a) == B.OWQ_ERR_BUFFER, i
    need = B.owq_qk_norm_rope_backward_workspace_bytes(d)
    assert need >= 2 * 64 * 4
    assert status(B.owq_qk_norm_rope_backward, d, *[P] * 13, 0, need) == B.OWQ_ERR_NULL
    assert status(B.owq_qk_norm_rope_backward, d, *[P] * 13, P, need - 1) == B.OWQ_ERR_BUFFER
    assert status(B.owq_qk_norm_rope_backward, d, *[P] * 13, P + 4, need) == B.OWQ_ERR_BUFFER
    for i in (0, 1, 2, 3, 6, 7, 8, 9, 10):
        a = [P] * 13
        a[i] = 0
        assert status(B.owq_qk_norm_rope_backward, d, *a, P, need) == B.OWQ_ERR_NULL, i
    assert lib.owq_qk_norm_rope(None, *[P] * 9, None) == B.OWQ_ERR_NULL


def cache(**kw):
    d = dict(n_pages=4, page_size=64, kv_heads=2, head_dim=64, n_seqs=2, table_stride=3)
    d.update(kw)
    return B.CacheDesc(**d)


BAD_CACHE = [
    (dict(n_pages=0), B.OWQ_ERR_SHAPE), (dict(kv_heads=0), B.OWQ_ERR_SHAPE), (dict(kv_heads=70000), B.OWQ_ERR_SHAPE), (dict(n_seqs=-1), B.OWQ_ERR_SHAPE),
    (dict(n_seqs=65536), B.OWQ_ERR_SHAPE), (dict(table_stride=0), B.OWQ_ERR_SHAPE), (dict(head_dim=136), B.OWQ_ERR_UNSUPPORTED),
    (dict(head_dim=60), B.OWQ_ERR_UNSUPPORTED), (dict(head_dim=0), B.OWQ_ERR_UNSUPPORTED), (dict(page_size=16), B.OWQ_ERR_UNSUPPORTED),
    (dict(page_size=96), B.OWQ_ERR_UNSUPPORTED), (dict(page_size=1 << 17), B.OWQ_ERR_UNSUPPORTED)]


def att(**kw):
    d = dict(q_heads=4, type=0, n_rows=5, max_new=3, max_len=100, window=0, sinks=0, scale=0.1, q_row=256, q_head=64)
    d.update(kw)
    return B.AttentionDesc(**d)


@pytest.mark.parametrize("kw,want", BAD_CACHE)
def test_cache_geometry(lib, kw, want):
    d = cache(**kw)
    assert status(B.owq_cache_append, d, P, P, P, P, P, P, 0, 5, 5, 128, 64, 128, 64) == want
    assert status(B.owq_cache_read, d, P, P, P, P, P, 0, 5, 5) == want
    assert status(B.owq_cache_attention, d, att(), P, P, P, P, P, P, P, P, 1 << 30) == want
    if not {"n_pages", "n_seqs", "table_stride"} & set(kw):
        assert status(B.owq_cache_page_bytes, d) == want


def test_cache_pages_and_pointers(lib):
    assert B.owq_cache_page_bytes(cache()) == 2 * 2 * (32 * 64 + 256)
    assert B.owq_cache_page_bytes(cache(head_dim=80, page_size=32)) == 2 * (32 * 96 + 256)
    d = cache()
    for i in range(6):
        for bad, want in ((0, B.OWQ_ERR_NULL), (P + 2, B.OWQ_ERR_BUFFER)):
            a = [P] * 6
            a[i] = bad
            assert status(B.owq_cache_append, d, *a, 0, 5, 5, 128, 64, 128, 64) == want, (i, bad)
            if i < 5:
                assert status(B.owq_cache_read, d, *a[:5], 0, 5, 5) == want, (i, bad)
            assert status(B.owq_cache_attention, d, att(), *a, P, P, 1 << 30) == want, (i, bad)
    assert status(B.owq_cache_append, d, *[P] * 6, 0, 5, 5, 127, 64, 128, 64) == B.OWQ_ERR_BUFFER
    assert status(B.owq_cache_append, d, *[P] * 6, 0, 5, 5, 128, 64, 128, 4) == B.OWQ_ERR_BUFFER
    assert status(B.owq_cache_append, d, *[P] * 6, 2, 5, 5, 128, 64, 128, 64) == B.OWQ_ERR_TYPE
    assert status(B.owq_cache_append, d, *[P] * 6, 0, -1, 5, 128, 64, 128, 64) == B.OWQ_ERR_SHAPE
    assert status(B.owq_cache_read, d, *[P] * 5, 3, 5, 5) == B.OWQ_ERR_TYPE
    assert status(B.owq_cache_append, d, *[0] * 6, 0, 0, 5, 128, 64, 128, 64) == B.OWQ_OK
    assert status(B.owq_cache_read, cache(n_seqs=0), *[0] * 5, 0, 5, 5) == B.OWQ_OK


@pytest.mark.parametrize("kw,want", [
    (dict(q_heads=3), B.OWQ_ERR_SHAPE), (dict(q_heads=0), B.OWQ_ERR_SHAPE), (dict(type=2), B.OWQ_ERR_TYPE), (dict(n_rows=-1), B.OWQ_ERR_SHAPE),
    (dict(window=-1), B.OWQ_ERR_SHAPE), (dict(sinks=-1), B.OWQ_ERR_SHAPE), (dict(scale=float("nan")), B.OWQ_ERR_SHAPE),
    (dict(q_row=250), B.OWQ_ERR_BUFFER), (dict(max_new=0), B.OWQ_OK), (dict(n_rows=0), B.OWQ_OK)])
def test_attention(lib, kw, want):
    assert status(B.owq_cache_attention, cache(), att(**kw), P, P, P, P, P, P, P, P, 1 << 30) == want


def test_attention_workspace(lib):
    d, a = cache(n_pages=4096, n_seqs=1, table_stride=2048), att(n_rows=1, max_new=1, max_len=100000)
    need = B.owq_cache_attention_workspace_bytes(d, a)
    assert need > 0
    assert status(B.owq_cache_attention, d, a, *[P] * 7, 0, need) == B.OWQ_ERR_NULL
    assert status(B.owq_cache_attention, d, a, *[P] * 7, P, need - 1) == B.OWQ_ERR_BUFFER
    assert status(B.owq_cache_attention, d, a, *[P] * 7, P + 16, need) == B.OWQ_ERR_BUFFER


@pytest.mark.parametrize("rows,vocab,type,want", [(-1, 5, 0, B.OWQ_ERR_SHAPE), (2, 0, 0, B.OWQ_ERR_SHAPE), (2, (1 << 24) + 1, 0, B.OWQ_ERR_SHAPE),
                                                  (2, 5, 3, B.OWQ_ERR_TYPE), (0, 5, 0, B.OWQ_OK)])
def test_sample(lib, rows, vocab, type, want):
    assert status(B.owq_sample, P, type, rows, vocab, 5, P, 5, P, P, P, P, P, P) == want


def test_sample_pointers(lib):
    good = dict(logits=P, type=2, rows=2, vocab=5, lrow=5, noise=P, nrow=5, t=P, k=P, p=P, m=P, token=P, lp=P)
    call = lambda **kw: status(B.owq_sample, *{**good, **kw}.values())  # noqa: E731
    assert call(logits=0) == B.OWQ_ERR_NULL and call(token=0) == B.OWQ_ERR_NULL and call(noise=0, t=0) == B.OWQ_ERR_NULL
    for name in ("logits", "noise", "t", "k", "p", "m", "token", "lp"):
        assert call(**{name: P + 2}) == B.OWQ_ERR_BUFFER, name
