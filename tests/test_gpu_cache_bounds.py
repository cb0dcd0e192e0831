"""The 4-bit cache: rows past max_new (append) and tokens past max_len (read) are not written, wherever in a tile they lie."""
import numpy as np
import pytest

from oracle import step
from test_gpu_cache import env, i32, make_table          # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", [  # tokens, new rows of them, bound
    ([5], [5], 1), ([50], [20], 3), ([40, 70, 9], [40, 6, 9], 7), ([100, 33], [90, 33], 33), ([100, 64], [90, 64], 32),
    ([3, 40], [10, 39], 8),                              # rows with negative positions count towards the bound
], ids=str)
@pytest.mark.parametrize("dim", [64, 72])
def test_append(env, case, dim):      # noqa: F811
    torch, B = env
    lengths, news, most = case
    rng = np.random.default_rng(sum(lengths))
    table, n_pages = make_table(rng, lengths, 32)
    starts = np.cumsum([0] + news)
    k = torch.from_numpy(rng.normal(size=(int(starts[-1]), 2, dim))).half().cuda()
    pages = B.cache_empty(n_pages, 32, 2, dim)
    pages.random_(0, 256)
    want = pages.cpu().numpy()
    B.cache_append(pages, i32(torch, table), i32(torch, starts), i32(torch, lengths), k, -k, max_new=most)
    torch.cuda.synchronize()
    for b, (n, m) in enumerate(zip(lengths, news)):
        got = min(m, most)                               # a sequence's first rows, ending where they end
        step.append(want, table[b:b + 1], [starts[b], starts[b] + got], [n - m + got], k.float().cpu().numpy(), -k.float().cpu().numpy(), dim)
    np.testing.assert_array_equal(pages.cpu().numpy(), want)


@pytest.mark.parametrize("most", [1, 31, 32, 33, 60])
@pytest.mark.parametrize("bf16", [False, True])
def test_read(env, most, bf16):      # noqa: F811
    torch, B = env
    rng = np.random.default_rng(most)
    lengths, dim = [50, 7, 100], 40
    table, n_pages = make_table(rng, lengths, 64)
    ends = np.cumsum([0] + lengths)
    rows = int(ends[-1])
    k = torch.from_numpy(rng.normal(size=(rows, 2, dim))).half().cuda()
    pages = B.cache_empty(n_pages, 64, 2, dim)
    B.cache_append(pages, i32(torch, table), i32(torch, ends), i32(torch, lengths), k, -k)
    dtype, kind = (torch.bfloat16, B.OWQ_TYPE_BF16) if bf16 else (torch.float16, B.OWQ_TYPE_F16)
    whole = B.cache_read(pages, i32(torch, table), i32(torch, ends), rows, dim, dtype=dtype)
    out = [torch.full((rows, 2, dim), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    d = B.CacheDesc(n_pages, 64, 2, dim, len(lengths), table.shape[1])
    t, s = i32(torch, table), i32(torch, ends)
    B.owq_cache_read(d, pages.data_ptr(), t.data_ptr(), s.data_ptr(), out[0].data_ptr(), out[1].data_ptr(), kind, rows, most,
                     torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for b, n in enumerate(lengths):
        a, m, z = ends[b], ends[b] + min(n, most), ends[b + 1]
        for got, w in zip(out, whole):
            assert torch.equal(got[a:m], w[a:m]) and (got[m:z] == 7).all(), b
