"""Attention over the 4-bit cache, single tokens: batches whose spans are cut into ranges, in the forms that few or short sequences
do not take.  Which form a call takes is read from its launches and from what its first launch leaves for the second, so that
another rule of choosing cannot leave these forms without a test."""
import numpy as np
import pytest

from launches import launches
from oracle import step
from test_gpu_attend import check, env, filled          # noqa: F401
from test_gpu_cache import i32

pytestmark = pytest.mark.gpu

CASES = {  # lengths, q heads, kv heads, dim, window, sinks, bf16; which forms it must take
    "70 uneven sequences": ([2200] + [31 * b % 2100 + 1 for b in range(69)], 2, 1, 32, 0, 0, False, {"more sequences than lanes"}),
    "130 uneven sequences, window": ([2600] + [57 * b % 2500 + 1 for b in range(129)], 2, 1, 32, 2300, 40, True, {"more sequences than lanes"}),
    "400 heads": ([2300, 2200] + [11 * b % 60 + 1 for b in range(98)], 8, 4, 32, 0, 0, False, {"more heads than half the ranges", "more sequences than lanes"}),
    "one long among 400": ([9 * b % 30 + 1 for b in range(257)] + [30000] + [5] * 142, 2, 1, 32, 0, 0, False,
                           {"more heads than half the ranges", "more sequences than lanes", "more ranges than lanes"}),
}


@pytest.mark.parametrize("name", CASES)
def test_ranges(env, name):      # noqa: F811
    torch, B = env
    lengths, hq, hk, dim, window, sinks, bf16, forms = CASES[name]
    n = len(lengths)
    rng = np.random.default_rng(n)
    pages, table = filled(env, rng, lengths, hk, dim, 64)
    q = torch.from_numpy(rng.normal(size=(n, hq, dim)) * 1.5).to(torch.bfloat16 if bf16 else torch.float16).cuda()
    starts = np.arange(n + 1)
    work = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")
    args = (q, pages, i32(torch, table), i32(torch, starts), i32(torch, lengths))
    call = lambda: B.cache_attention(*args, window=window, sinks=sinks, max_new=1, max_len=max(lengths), want_lse=True, workspace=work)  # noqa: E731
    out, lse = call()

    # two launches: ranges, then the join.  At the workspace's end, each sequence's first workgroup and ranges per head
    d = B.CacheDesc(pages.shape[0], 64, hk, dim, n, table.shape[1])
    a = B.AttentionDesc(hq, int(bf16), n, 1, max(lengths), window, sinks, dim ** -0.5, hq * dim, dim)
    need = B.owq_cache_attention_workspace_bytes(d, a)
    first, ranges = work[need - 8 * n:need].view(torch.int32).view(n, 2).cpu().numpy().T
    kernels = launches(torch, call)
    assert len(kernels) == 2 and kernels[0][1] == 256
    assert (first == np.concatenate([[0], np.cumsum(ranges * hk)[:-1]])).all() and kernels[0][0] >= (ranges * hk).sum()
    tiles = -(-np.asarray(lengths) // 32)
    assert ranges.max() > 1 and (ranges <= tiles).all()
    taken = set()
    if n > 64 and (ranges[64:] > 0).all():
        taken.add("more sequences than lanes")
    if 2 * n * hk > 3 * 256:
        taken.add("more heads than half the ranges")
    if ranges.max() > 64:
        taken.add("more ranges than lanes")
    assert taken == forms, (taken, ranges.max())

    want = step.attention(q.double().cpu().numpy(), pages.cpu().numpy(), table, starts, lengths, dim ** -0.5, window, sinks)
    check(env, out, lse, want, bf16)
