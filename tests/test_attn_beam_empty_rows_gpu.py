"""Beams without a slot beside others that have some: nothing of theirs is looked at, neither their query nor its position."""
import numpy as np
import pytest
import torch

import paper_2512_16822_b200 as M
from beam_helpers import BeamCase
from test_attn_beam_gpu import _built      # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,fp8", [(64, False), (128, False), (128, True)])
@pytest.mark.parametrize("W,Hq", [(3, 4), (8, 4), (12, 6)])
@pytest.mark.parametrize("q_pos", [-1, 1 << 30, -(1 << 31), (1 << 31) - 1])
def test_an_empty_rows_position_is_not_looked_at(D, fp8, W, Hq, q_pos):
    # the contexts end at the last position that the rope table has
    specs = [(48, 1), (500, 13), (0, 30)]
    lens = np.repeat([c + g for c, g in specs], W)
    empty = np.zeros(3 * W, dtype=bool)
    empty[[0, W + 1, W + 2, 2 * W, 3 * W - 1]] = True
    lens[empty] = 0
    case = BeamCase(71 + W, Hq=Hq, Hkv=2, D=D, P=16, width=W, specs=specs, lens=lens, fp8=fp8)
    case.pos_base[:] = np.arange(case.pos_base.shape[1]) * 16
    case.finish()
    case.max_position = int(case.q_pos.max())
    case.cfg = M.Config(16, Hq, 2, D, case.num_pages, case.max_position, case.theta)
    case.q_pos[empty] = q_pos
    case.q[empty] = 0x7fc0
    case.poison()
    case.device()
    case.batch()
    out = case.run(0.09)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    case.check(out, 0.09)


@pytest.mark.parametrize("q_pos", [-(1 << 31), 1 << 30])
def test_a_position_out_of_reach_of_a_row_with_slots_is_reported(q_pos):
    case = BeamCase(72, Hq=4, Hkv=2, D=128, P=16, width=3, specs=[(48, 1)])
    case.q_pos[1] = q_pos
    case.device()
    case.batch()
    out = case.run(0.09)
    torch.cuda.synchronize()
    assert case.dev.read_status() == M.MEPIC_DEV_BAD_POSITION
    case.check(out, 0.09, which=[0, 2])
