"""Residual sum with norms and its gradients where a workgroup takes several rows: three at least for every team of the gradients' kernels with
one, two and three pieces of a row to a thread and of the rolled ones, with every pairing of a norm of the branch and a gate; the last
workgroups have fewer rows than the others, or teams without one.  By the oracle and tolerances of test_gpu_norm.py: a sum over tokens passes at
most rows of a team + 16 teams + 4 + 16 + 2 of the second kernel, fewer than the 64 additions that they count."""
import pytest

import test_gpu_norm as N
from test_gpu_norm import env  # noqa: F401

pytestmark = pytest.mark.gpu

# the sizes: pieces of a thread, rows of a team of the gradients' kernel (with the branch's side; without it where no post and no gate)
#   9001 x 72     one piece, ten teams, four rows (16 teams, three)         1801 x 2000   one piece, two teams, four rows (four teams, two)
#   1031 x 5003   one piece, one team, five rows                            601 x 6001, 8191   two pieces, three rows (one piece)
#   601 x 9216, 10007, 12000   three pieces, three rows                     1031 x 12289, 601 x 12296   rolled, five rows, three
# forward: 1031 x 5003 and 601 x 8191 with a norm of the branch, 601 x 9216 (two pieces), 601 x 12000 (three), 1031 x 12289 (rolled): three rows
CASES = [  # tokens, width, norm, post, gate, bias, p, dtype, fp32 residual, off the 16-byte grid
    (9001, 72, "layer", None, None, True, 0.1, "float16", False, False),
    (9001, 72, "rms", "layer", None, True, 0.1, "bfloat16", False, False),
    (9001, 72, "rms", None, "row", False, 0.0, "float16", True, True),
    (9001, 72, "layer", "rms", "row", True, 0.2, "bfloat16", False, True),
    (1801, 2000, "rms", "rms", "token", False, 0.1, "float16", False, False),
    (1801, 2000, "layer", "layer", "row", True, 0.1, "bfloat16", True, False),
    (1801, 2000, "layer", None, None, True, 0.0, "bfloat16", True, False),
    (1031, 5003, "rms", None, None, False, 0.1, "bfloat16", True, False),
    (1031, 5003, "layer", "rms", None, True, 0.1, "float16", False, False),
    (1031, 5003, "layer", None, "row", True, 0.0, "bfloat16", False, False),
    (1031, 5003, "rms", "rms", "row", False, 0.0, "float16", False, False),
    (1031, 5003, "rms", "layer", "token", True, 0.1, "float16", True, False),
    (601, 8191, "layer", None, None, True, 0.1, "float16", False, True),
    (601, 6001, "rms", "layer", None, True, 0.1, "bfloat16", False, False),
    (601, 8191, "layer", "rms", None, True, 0.0, "float16", True, False),
    (601, 6001, "layer", None, "row", True, 0.1, "float16", True, False),
    (601, 8192, "rms", None, "token", False, 0.0, "bfloat16", False, False),
    (601, 6001, "rms", "rms", "row", True, 0.1, "bfloat16", True, False),
    (601, 8191, "layer", "layer", "row", True, 0.1, "float16", False, True),
    (601, 9216, "rms", None, None, False, 0.0, "float16", False, False),
    (601, 10007, "layer", None, None, True, 0.1, "bfloat16", True, True),
    (601, 9216, "layer", "rms", None, True, 0.1, "bfloat16", False, False),
    (601, 12000, "rms", "layer", None, True, 0.0, "float16", True, False),
    (601, 9216, "rms", None, "row", True, 0.1, "bfloat16", True, False),
    (601, 12000, "layer", None, "token", True, 0.0, "float16", False, False),
    (601, 9217, "layer", "layer", "row", True, 0.1, "float16", False, False),
    (601, 12000, "rms", "rms", "row", True, 0.1, "bfloat16", True, False),
    (1031, 12289, "layer", None, None, True, 0.1, "float16", False, False),
    (1031, 12289, "rms", "layer", None, True, 0.0, "bfloat16", True, False),
    (601, 12296, "layer", None, "row", True, 0.1, "bfloat16", False, False),
    (601, 12289, "layer", "rms", "row", True, 0.1, "float16", False, True),
    (520, 16384, None, "rms", "token", True, 0.1, "float16", True, False),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward(env, case):  # noqa: F811
    N.test_forward(env, case)


@pytest.mark.parametrize("case", CASES, ids=str)
def test_backward(env, case):  # noqa: F811
    N.test_backward(env, case)
