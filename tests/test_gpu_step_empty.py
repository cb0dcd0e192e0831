"""The operators between two layers on tensors without elements, whose strides may be anything."""
import pytest

from test_gpu_cache import env, i32          # noqa: F401

pytestmark = pytest.mark.gpu


def test_no_rows(env):      # noqa: F811
    torch, B = env

    def none(*shape, dtype=torch.float16):
        return torch.empty(0, device="cuda", dtype=dtype).as_strided(shape, (3,) * len(shape))
    cos = torch.ones(4, 16, device="cuda")
    w = torch.ones(32, device="cuda").half()
    q, k, pos = none(0, 4, 32), none(0, 2, 32), i32(torch, [])
    out = B.qk_norm_rope(q, k, cos, cos, pos, w, w)
    assert out[0].shape == q.shape and out[1].shape == k.shape
    dq, dk, dwq, dwk = B.qk_norm_rope_backward(q, k, q, k, cos, cos, pos, w, w)
    assert dq.shape == q.shape and dk.shape == k.shape and (dwq == 0).all() and (dwk == 0).all()
    pages = B.cache_empty(1, 32, 2, 32)
    before = pages.fill_(5).clone()
    args = (i32(torch, [[0]]), i32(torch, [0, 0]), i32(torch, [9]))
    B.cache_append(pages, *args, k, k)
    assert torch.equal(pages, before)
    assert B.cache_attention(q, pages, *args).shape == q.shape
    token, logprob = B.sample(none(0, 9), none(0, 9, dtype=torch.float32))
    assert token.numel() == 0 and logprob.numel() == 0
