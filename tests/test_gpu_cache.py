"""The 4-bit cache on the GPU: bytes against the oracle's packer, bit for bit, and values read back, exactly."""
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


def i32(torch, a):
    return torch.from_numpy(np.asarray(a, np.int32)).cuda()


def make_table(rng, lengths, page, spare=1):
    per = [max(1, -(-n // page)) for n in lengths]
    n_pages = sum(per) + spare
    ids = rng.permutation(n_pages)
    table = np.full((len(lengths), max(per) + 1), -1, np.int32)
    at = 0
    for b, n in enumerate(per):
        table[b, :n] = ids[at:at + n]
        at += n
    return table, n_pages


CASES = [  # lengths, new, kv heads, dim, page, bf16
    ([1], [1], 1, 8, 32, False), ([33, 1, 64], [1, 1, 1], 2, 128, 32, False), ([70, 32, 31], [70, 3, 31], 3, 64, 64, True),
    ([129], [100], 1, 80, 128, False), ([40, 0, 7], [35, 0, 7], 2, 96, 32, True), ([65, 200], [2, 9], 5, 128, 256, False),
    ([5, 90], [8, 1], 2, 40, 32, False),                      # more new rows than tokens: the first have negative positions
]


@pytest.mark.parametrize("slices", [False, True])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_append_bytes_and_read(env, case, slices):
    torch, B = env
    lengths, news, heads, dim, page, bf16 = case
    rng = np.random.default_rng(dim + len(lengths))
    table, n_pages = make_table(rng, lengths, page)
    rows = sum(news)
    x = torch.from_numpy(rng.normal(size=(rows, 2 * heads + 1, dim)) * rng.choice([1e-4, 1.0, 500.0], size=(rows, 1, 1)))
    x = x.to(torch.bfloat16 if bf16 else torch.float16).cuda()
    x[rows // 2, 0] = 0.75                                     # a constant head
    k, v = x[:, :heads], x[:, heads:2 * heads]
    if not slices:
        k, v = k.contiguous(), v.contiguous()
    starts = np.cumsum([0] + news)
    pages = B.cache_empty(n_pages, page, heads, dim)
    pages.random_(0, 256)
    want = pages.cpu().numpy()
    assert want.shape[3] == step.tile_bytes(dim)
    B.cache_append(pages, i32(torch, table), i32(torch, starts), i32(torch, lengths), k, v, max_new=max(news))
    torch.cuda.synchronize()
    step.append(want, table, starts, lengths, k.float().cpu().numpy(), v.float().cpu().numpy(), dim)
    np.testing.assert_array_equal(pages.cpu().numpy(), want)
    # and back; what older tokens' bytes stand for is garbage here, and read as it is
    for dtype in (torch.float16, torch.bfloat16):
        ends = np.cumsum([0] + lengths)
        got = B.cache_read(pages, i32(torch, table), i32(torch, ends), int(ends[-1]), dim, max_len=max(lengths), dtype=dtype)
        torch.cuda.synchronize()
        for b, n in enumerate(lengths):
            rk, rv, _ = step.read(want, table[b], n, dim)
            for a, r in zip(got, (rk, rv)):
                with np.errstate(all="ignore"):
                    r = torch.from_numpy(r.astype(np.float32)).to(dtype)
                a = a[ends[b]:ends[b + 1]].cpu()
                assert torch.equal(torch.nan_to_num(a, nan=7), torch.nan_to_num(r, nan=7))


def test_rows_outside_pages_tables_and_tensors_are_left_out(env):
    torch, B = env
    rng = np.random.default_rng(0)
    heads, dim, page = 2, 64, 32
    pages = torch.zeros((3, heads, 1, step.tile_bytes(dim)), dtype=torch.uint8, device="cuda")
    table = np.array([[2, 7], [-1, 1], [0, -5]], np.int32)      # 7 and negative entries are no pages
    lengths, starts = [80, 40, 20], [0, 80, 120, 140]            # sequence 0 also passes its table; row 130 and on do not exist
    k = torch.from_numpy(rng.normal(size=(130, heads, dim))).half().cuda()
    want = pages.cpu().numpy()
    B.cache_append(pages, i32(torch, table), i32(torch, starts), i32(torch, lengths), k, k)
    torch.cuda.synchronize()
    kn = np.concatenate([k.float().cpu().numpy(), np.zeros((10, heads, dim), np.float32)])
    table_cut = table.copy()
    step.append(want, table_cut, [0, 80, 120, 130], [80, 40, 10], kn, kn, dim)
    np.testing.assert_array_equal(pages.cpu().numpy(), want)
    out = B.cache_read(pages, i32(torch, table), i32(torch, starts), 130, dim)
    torch.cuda.synchronize()
    assert (out[0][32:80].cpu() == 0).all() and (out[0][80:112].cpu() == 0).all() and (out[0][112:120].cpu() != 0).any()


def test_non_finite_heads(env):
    torch, B = env
    k = torch.ones((3, 2, 32), dtype=torch.float16, device="cuda")
    k[0, 0, 3], k[1, 1, 31], k[2, 0, 0] = float("nan"), float("inf"), -65504
    k[2, 0, 1] = 65504
    pages = torch.zeros((1, 2, 1, step.tile_bytes(32)), dtype=torch.uint8, device="cuda")
    want = pages.cpu().numpy()
    args = i32(torch, [[0]]), i32(torch, [0, 3])
    B.cache_append(pages, *args, i32(torch, [3]), k, k)
    got = B.cache_read(pages, *args, 3, 32)[0].cpu()
    step.append(want, np.array([[0]]), [0, 3], [3], k.float().cpu().numpy(), k.float().cpu().numpy(), 32)
    np.testing.assert_array_equal(pages.cpu().numpy(), want)
    assert torch.isnan(got[0, 0]).all() and torch.isnan(got[1, 1]).all() and (got[0, 1] == 1).all()
    assert got[2, 0, 0] == -65504 and got[2, 0, 1] > 65000


def test_pages_past_two_gigabytes(env):
    torch, B = env
    heads, dim, page = 1, 128, 65536
    n_pages = 260                                               # 260 pages of 8.9 MB
    pages = B.cache_empty(n_pages, page, heads, dim)
    assert pages.numel() > 1 << 31
    k = torch.randn(3, heads, dim, device="cuda").half()
    table = i32(torch, [[n_pages - 1]])
    pages[n_pages - 1].zero_()
    B.cache_append(pages, table, i32(torch, [0, 3]), i32(torch, [65536]), k, k)
    torch.cuda.synchronize()
    want = np.zeros((1, 1, 1, step.tile_bytes(dim)), np.uint8)
    step.append(want, np.array([[0]]), [0, 3], [32], k.float().cpu().numpy(), k.float().cpu().numpy(), dim)
    np.testing.assert_array_equal(pages[n_pages - 1, 0, 2047].cpu().numpy(), want[0, 0, 0])
    assert (pages[n_pages - 1, 0, 2046] == 0).all()
    out, = (B.cache_attention(k, pages, table, i32(torch, [0, 3]), i32(torch, [65536]), window=2),)
    ref = step.attention(k.double().cpu().numpy(), want, np.array([[0]]), [0, 3], [32], dim ** -0.5, window=2)
    assert np.abs(out[1:].double().cpu().numpy() - ref[0][1:]).max() <= ref[2].max() + 2.0 ** -11 * np.abs(ref[0]).max()
