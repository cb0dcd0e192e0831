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


@pytest.mark.parametrize("new,heads", [(1, 1), (3, 2), (45, 1), (80, 128)])
@pytest.mark.parametrize("short_of", [0, 1, 31, 32])
def test_last_positions(env, new, heads, short_of):      # noqa: F811
    # the sequence's pages are all the same one: the bytes and the results are those of a sequence 32767 pages shorter
    torch, B = env
    rng = np.random.default_rng(42)
    page, dim, window, sinks = 65536, 16, 50, 5
    pages = torch.zeros((1, heads, page // 32, step.tile_bytes(dim)), dtype=torch.uint8, device="cuda")
    near = torch.zeros_like(pages)
    far, short = LAST - short_of, LAST - short_of - 32767 * page
    k, v = (torch.from_numpy(rng.normal(size=(160, heads, dim))).half().cuda() for _ in range(2))
    table = torch.zeros((1, 32768), dtype=torch.int32, device="cuda")
    for x, n in ((pages, far), (near, short)):
        B.cache_append(x, table, i32(torch, [0, 20]), i32(torch, [20]), k[:20], v[:20])
        B.cache_append(x, table, i32(torch, [0, 140]), i32(torch, [n]), k[20:], v[20:])
    assert torch.equal(pages, near)
    q = torch.from_numpy(rng.normal(size=(new, heads, dim))).half().cuda()
    got = B.cache_attention(q, pages, table, i32(torch, [0, new]), i32(torch, [far]), window=window, sinks=sinks, max_len=LAST, want_lse=True)
    # the oracle on the tiles that are seen: the first ones, then the last 256 tokens
    tiles = np.concatenate([pages[0, :, :2].cpu().numpy(), pages[0, :, -8:].cpu().numpy()], 1)
    cut = short - (page - 320)
    pos = cut - new + np.arange(new)
    assert pos[0] - window >= 64                         # all tokens between the two pieces are outside the window
    want = step.attention(q.double().cpu().numpy(), np.ascontiguousarray(tiles.transpose(1, 0, 2)[:, :, None]),
                          np.arange(10)[None], [0, new], [cut], dim ** -0.5, window, sinks)
    check(env, *got, want, False)


def test_tables_of_more_than_the_largest_length(env):      # noqa: F811
    # no bound given: the table's capacity, which is more than a length can be
    torch, B = env
    rng = np.random.default_rng(43)
    page, dim = 65536, 16
    pages = torch.zeros((1, 1, page // 32, step.tile_bytes(dim)), dtype=torch.uint8, device="cuda")
    table = torch.full((1, 32769), -1, dtype=torch.int32, device="cuda")
    table[0, 0] = 0
    args = (table, i32(torch, [0, 40]), i32(torch, [40]))
    k = torch.from_numpy(rng.normal(size=(40, 1, dim))).half().cuda()
    B.cache_append(pages, *args, k, k)
    out, lse = B.cache_attention(k, pages, *args, want_lse=True)
    want = step.attention(k.double().cpu().numpy(), pages[:, :, :2].cpu().numpy(), np.array([[0]]), [0, 40], [40], dim ** -0.5)
    check(env, out, lse, want, False)
