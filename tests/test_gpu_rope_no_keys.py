"""Head norm with rotation where there are no key heads: the keys' weight has a gradient, of nothing: zero."""
import numpy as np
import pytest

from test_gpu_rope import env, make          # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [0, 1, 700])
@pytest.mark.parametrize("weights", ["k", "qk"])
def test_key_weight_without_key_heads(env, tokens, weights):      # noqa: F811
    torch, B = env
    _, dev, q, k, wq, wk, cos, sin, pos = make(env, max(tokens, 1), 3, 0, 48, 48, weights, False, 7, False)
    q, k, pos = q[:tokens], k[:tokens], torch.from_numpy(pos[:tokens]).cuda()
    cos, sin = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    dy = dev(np.ones((tokens, 3, 48)))
    # what the call's results are allocated from holds no zeros
    torch.cuda.synchronize()
    stale = [torch.full((48,), 7.0, device="cuda") for _ in range(64)]
    torch.cuda.synchronize()
    del stale
    dq, dk, dwq, dwk = B.qk_norm_rope_backward(dy, k, q, k, cos, sin, pos, wq, wk)
    assert dk.shape == (tokens, 0, 48) and dwk.shape == (48,) and (dwk == 0).all()
    # the rest is what it is without that weight
    want = B.qk_norm_rope_backward(dy, k, q, k, cos, sin, pos, wq, None)
    assert torch.equal(dq, want[0]) and want[3] is None
    assert (dwq is None) == (wq is None) and (wq is None or torch.equal(dwq, want[2]))


def test_null_keys_through_the_c_entry(env):      # noqa: F811
    torch, B = env
    _, dev, q, _, wq, wk, cos, sin, pos = make(env, 5, 2, 0, 64, 32, "qk", True, 8, False)
    pos, cos, sin = (torch.from_numpy(t).cuda() for t in (pos, cos, sin))
    dy, dq = dev(np.ones((5, 2, 64))), torch.empty_like(q)
    dw = torch.full((2, 64), 7.0, device="cuda")
    d = B.RopeDesc(5, 2, 0, 64, 32, 0, B.OWQ_TYPE_BF16, cos.shape[0], 1e-6, 0, 128, 64, 0, 0, 128, 64, 0, 0)
    work = torch.empty(B.owq_qk_norm_rope_backward_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    B.owq_qk_norm_rope_backward(d, dy.data_ptr(), 0, q.data_ptr(), 0, wq.data_ptr(), wk.data_ptr(), cos.data_ptr(), sin.data_ptr(),
                                pos.data_ptr(), dq.data_ptr(), 0, dw[0].data_ptr(), dw[1].data_ptr(), work.data_ptr(), work.numel(),
                                torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert (dw[1] == 0).all() and not (dw[0] == 7).any()
