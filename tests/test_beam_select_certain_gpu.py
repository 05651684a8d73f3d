"""Selection where a token is certain: its logarithm of a probability is 0, and its score the beam's, bit for bit."""
import numpy as np
import pytest
import torch

from test_beam_select_gpu import TYPES, _built, _logits, _run      # noqa: F401  (_built: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [1, 5, 300, 20011])
@pytest.mark.parametrize("others", [-float("inf"), -6e4])
def test_the_only_token_that_is_allowed(dtype, V, others):
    # e^-50,000 and less beside 1: nothing
    rng = np.random.default_rng(V)
    x = torch.full((24, V), others, device="cuda:0").to(TYPES[dtype])
    at = torch.from_numpy(rng.integers(0, V, size=24)).cuda()
    x[torch.arange(24, device="cuda:0"), at] = _logits(24, 1, dtype, V, 100.0)[:, 0]
    scores = -rng.uniform(0, 9, size=(3, 8)).astype(np.float32)
    scores[1] = -2.7182817
    scores[2] = -1e9
    op, _ = _run(x, scores, K=8)
    for g in range(3):
        order = np.argsort(-scores[g], kind="stable")
        assert op.score[g].tolist() == scores[g][order].tolist()
        assert op.parent[g].tolist() == order.tolist()
        assert op.token[g].tolist() == at.view(3, 8)[g].cpu().numpy()[order].tolist()
