"""The entry points between two layers at sizes near 2^31: workspaces that hold."""
import pytest

from test_step_refusals import lib, rope          # noqa: F401

B = pytest.importorskip("paper_2306_02272_amd.binding")


@pytest.mark.parametrize("tokens", [2 ** 31 - 1, 2 ** 31 - 1000, 2 ** 31 - 5000, 2 ** 30])
def test_rotation_gradients(lib, tokens):      # noqa: F811
    # a row of sums for each of 4096 workgroups at most, and no fewer than for fewer tokens
    need = B.owq_qk_norm_rope_backward_workspace_bytes(rope(n_tokens=tokens))
    assert B.owq_qk_norm_rope_backward_workspace_bytes(rope(n_tokens=1)) <= need <= 4096 * 2 * 64 * 4
