"""Selection where no threshold is known and more tokens are candidates than the lists hold: fewer sets of tokens (128 of an fp32
row, 256 of a 16-bit one, at most) hold a candidate than are to be selected, and together they hold thousands."""
import numpy as np
import pytest
import torch

from test_beam_select_gpu import TYPES, _built, _logits, _run, _scores      # noqa: F401  (_built: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("W,V,K", [(1, 1537, 50), (1, 1600, 64), (1, 2000, 64), (1, 2016, 64), (2, 769, 50), (2, 900, 64), (2, 1008, 64), (4, 400, 60),
                                   (4, 480, 64), (4, 504, 64), (8, 200, 64), (8, 224, 57), (8, 252, 64), (1, 40, 64), (32, 60, 64)])
def test_small_vocabularies_and_many_to_select(dtype, W, V, K):
    _run(_logits(3 * W, V, dtype, W + V), _scores(3, W, V), K=K, eos=V // 2)
    _run(torch.round(_logits(3 * W, V, "fp32", V, 1.0)).to(TYPES[dtype]), np.zeros((3, W)), K=K)      # a few values only


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("off", range(8))
def test_at_any_alignment(dtype, off):
    # rows 1,003 + 5 elements apart that begin anywhere in their 16 bytes; what lies around them would win
    buf = torch.full((8, 1008), 3e4, device="cuda:0").to(TYPES[dtype])
    x = buf.view(-1)[off:off + 3 * 1008 + 1003].as_strided((4, 1003), (1008, 1))
    x.copy_(_logits(4, 1003, dtype, off))
    _run(x, _scores(2, 2, off), K=64)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("W", [1, 2, 5])
def test_masks_that_leave_few_sets_full(dtype, W):
    # what is left of the rows lies in a few whole sets: a set's pieces are 1,024 (fp32) or 2,048 (16-bit) tokens apart
    for V, period, allowed, K in ((8192, 1024, 208, 16), (16384, 2048, 224, 8), (16384, 2048, 224, 50), (40001, 2048, 96, 64)):
        x = _logits(2 * W, V, dtype, V + allowed)
        x[:, torch.arange(V, device="cuda:0") % period >= allowed] = -np.inf
        _run(x, _scores(2, W, V), K=K)


@pytest.mark.parametrize("dtype", TYPES)
def test_finished_beams_among_them(dtype):
    done = np.array([[0, 1, 0, 0], [1, 1, 0, 1], [0, 0, 0, 0]])
    scores = _scores(3, 4, 3)
    scores[1, 2] -= 4.0
    for V in (520, 1700):
        _run(_logits(12, V, dtype, V), scores, done=done, K=64, eos=5, pad=3)
    # all logits equal: the finished beams' scores fall among thousands of ties
    x = torch.zeros((12, 1700), device="cuda:0", dtype=TYPES[dtype])
    scores = np.where(done == 1, -7.0, 0.0)
    _run(x, scores, done=done, K=64, pad=3)
