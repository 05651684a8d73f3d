"""Selection over rows with finite logits of any magnitude, as masks by a large negative number leave them."""
import numpy as np
import pytest
import torch

from test_beam_select_gpu import TYPES, _built, _logits, _run, _scores      # noqa: F401  (_built: the fixture)

pytestmark = pytest.mark.gpu
VALUES = [-1e4, -65000.0, -1e5, -1e6, -1e7, -1e9, -3e9, -1e10, -1e12, -1e15, -1e20, -9.9e29, -1e30, -1.1e30, -1e38, 1e5, 1e10, 1e15, 1e20, 1e38]
CASES = [(d, v) for d in TYPES for v in VALUES if d != "fp16" or abs(v) < 65504]


@pytest.mark.parametrize("dtype,value", CASES)
def test_rows_masked_by_a_finite_number(dtype, value):
    V = 20011
    t = torch.arange(V, device="cuda:0")
    x = _logits(10, V, dtype, 3)
    for g in range(2):
        x[5 * g] = value                                    # wholly
        x[5 * g + 1, 9:] = value                            # all but a few tokens
        x[5 * g + 2, V - 4000:] = value                     # the padded end of a vocabulary
        x[5 * g + 3, t // 64 % 2 == g] = value              # every other stretch
        x[5 * g + 4, 12345] = value                         # one token
    _run(x, _scores(2, 5, 3), K=10)


@pytest.mark.parametrize("dtype,value", CASES)
def test_a_row_of_one_large_number(dtype, value):
    # every candidate is the same, and the sum of exponentials the number of tokens
    for V in (5, 700, 9000):
        op, _ = _run(torch.full((1, V), value, device="cuda:0").to(TYPES[dtype]), np.array([[-1.5]]), K=4)
        assert op.token[0].tolist() == [0, 1, 2, 3] and op.parent[0].tolist() == [0] * 4


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("middle", [-3e4, -5000.0, 5000.0, 3e4])
def test_ordinary_rows_far_from_zero(dtype, middle):
    # 16 bits hold whole numbers or less there: spread them so that they differ
    x = (_logits(6, 9001, "fp32", 5, 300.0) + middle).to(TYPES[dtype])
    _run(x, _scores(2, 3, 5), K=8)
