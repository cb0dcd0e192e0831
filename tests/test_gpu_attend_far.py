"""Attention and cache where counts come near 2^31: first tokens kept beyond any length, positions at the end of the range."""
import numpy as np
import pytest

from oracle import step
from test_gpu_attend import check, env, filled          # noqa: F401
from test_gpu_cache import i32

pytestmark = pytest.mark.gpu
LAST = 2 ** 31 - 1


@pytest.mark.parametrize("sinks", [LAST, LAST - 30, LAST - 31])
@pytest.mark.parametrize("new,heads,length", [(1, 1, 300), (2, 2, 3000), (90, 1, 300), (80, 128, 200)])
def test_all_tokens_are_first_tokens(env, new, heads, length, sinks):      # noqa: F811
    torch, B = env
    rng = np.random.default_rng(41)
    pages, table = filled(env, rng, [length], heads, 32, 32)
    q = torch.from_numpy(rng.normal(size=(new, heads, 32))).half().cuda()
    out, lse = B.cache_attention(q, pages, i32(torch, table), i32(torch, [0, new]), i32(torch, [length]), window=10, sinks=sinks, want_lse=True)
    want = step.attention(q.double().cpu().numpy(), pages.cpu().numpy(), table, [0, new], [length], 32 ** -0.5, 10, sinks)
    check(env, out, lse, want, False)
