"""Selection among beams with the same logits and the same score, as copies of one beam have them: their candidates are equal, wherever
in its 16 bytes each row begins, and come in order of the beams."""
import numpy as np
import pytest
import torch

from test_beam_select_gpu import TYPES, _built, _logits, _run      # noqa: F401  (_built: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [1, 3, 17, 131, 1001, 8195, 30001, 100003])
@pytest.mark.parametrize("W,K", [(2, 8), (8, 16), (32, 64)])
def test_copies_of_a_beam(dtype, V, W, K):
    for seed in range(3):
        x = _logits(3, V, dtype, seed)[:, None].expand(3, W, V).reshape(3 * W, V).contiguous()
        op, _ = _run(x, np.full((3, W), -0.7), K=K)
        if dtype == "fp32":                                       # (no two tokens are equal: each is taken from all beams in turn)
            n = min(K, W * V) // W * W
            assert (op.parent[:, :n].cpu().numpy() == np.arange(n) % W).all(), (seed, op.parent[:, :n])


def test_copies_among_others():
    x = _logits(16, 5003, "bf16", 5)
    x[3], x[6], x[7] = x[1], x[1], x[4]
    score = np.array([[0.0, -1.0, -2.0, -1.0, -0.5, -0.2, -1.0, -0.5]])
    _run(x[:8].contiguous(), score, K=32)
    x[8:] = x[8]
    _run(x, np.concatenate([score, np.full((1, 8), -3.0)]), K=32, done=np.array([[0, 0, 0, 0, 0, 0, 0, 0], [0, 1, 0, 0, 1, 0, 0, 0]]), eos=7)
