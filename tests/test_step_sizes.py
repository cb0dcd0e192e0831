"""The entry points between two layers at sizes near 2^31: workspaces that hold, refusals where a launch could not."""
import pytest

from test_step_refusals import P, att, cache, lib, rope, status          # noqa: F401

B = pytest.importorskip("paper_2306_02272_amd.binding")


@pytest.mark.parametrize("tokens", [2 ** 31 - 1, 2 ** 31 - 1000, 2 ** 31 - 5000, 2 ** 30])
def test_rotation_gradients(lib, tokens):      # noqa: F811
    # a row of sums for each of 4096 workgroups at most, and no fewer than for fewer tokens
    need = B.owq_qk_norm_rope_backward_workspace_bytes(rope(n_tokens=tokens))
    assert B.owq_qk_norm_rope_backward_workspace_bytes(rope(n_tokens=1)) <= need <= 4096 * 2 * 64 * 4


@pytest.mark.parametrize("kw,rows", [
    (dict(n_seqs=65535, kv_heads=65535, head_dim=8), 1), (dict(n_seqs=65535, kv_heads=32769, head_dim=8), 20), (dict(n_seqs=65535, kv_heads=300), 1)])
def test_attention_of_too_many_workgroups(lib, kw, rows):      # noqa: F811
    d = cache(table_stride=4096, **kw)
    for length in (32, 100000):
        a = att(q_heads=d.kv_heads, n_rows=65535 * rows, max_new=rows, max_len=length, q_row=d.kv_heads * 64)
        assert status(B.owq_cache_attention_workspace_bytes, d, a) == B.OWQ_ERR_SHAPE
        assert status(B.owq_cache_attention, d, a, P, P, P, P, P, P, P, P, 1 << 30) == B.OWQ_ERR_SHAPE
    # as many as a batch has
    d = cache(n_seqs=4096, kv_heads=128, table_stride=4096)
    assert status(B.owq_cache_attention_workspace_bytes, d, att(q_heads=128, n_rows=4096, max_new=1, max_len=100000)) == B.OWQ_OK
