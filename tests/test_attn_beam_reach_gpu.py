"""Attention of beams at the end of what the rope table reaches, with pages of several tiles that are barely filled."""
import numpy as np
import pytest
import torch

import paper_2512_16822_b200 as M
from beam_helpers import BeamCase
from test_attn_beam_gpu import _built      # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,fp8", [(64, False), (128, False), (128, True)])
@pytest.mark.parametrize("P,filled,base,reach", [(64, 20, 150, 176), (64, 1, 176, 176), (128, 17, 160, 176), (512, 3, 500, 511)])
def test_the_empty_end_of_a_page_needs_no_angles(P, filled, base, reach, D, fp8):
    # the query stands at 0, the last filled slot within reach of it, the page's last tiles beyond
    case = BeamCase(51 + P, Hq=4, Hkv=2, D=D, P=P, width=2, specs=[(P + filled, 0), (0, filled)], fp8=fp8)
    case.pos_base[:2, :2] = [-P // 2, base]
    case.pos_base[2:, 0] = base
    case.q_pos[:] = 0
    assert base + filled - 1 <= reach
    case.max_position = reach
    case.cfg = M.Config(P, 4, 2, D, case.num_pages, reach, case.theta)
    case.poison()
    case.device()
    case.batch()
    out = case.run(0.09)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    case.check(out, 0.09)


def test_a_filled_slot_out_of_reach_is_reported():
    case = BeamCase(52, Hq=4, Hkv=2, D=128, P=64, width=2, specs=[(60, 0)])
    case.pos_base[:, 0] = 200
    case.q_pos[:] = 0
    case.cfg = M.Config(64, 4, 2, 128, case.num_pages, 176, case.theta)
    case.device()
    case.batch()
    case.run(0.09)
    torch.cuda.synchronize()
    assert case.dev.read_status() == M.MEPIC_DEV_BAD_POSITION
