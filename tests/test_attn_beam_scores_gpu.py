"""Attention of beams where the scores themselves show: references that rise by hundreds again and again, and the score of one key
read off a weight."""
import numpy as np
import pytest
import torch

from mepic_inputs import bf16_bits_to_f64, f32_to_bf16_bits
from oracle import mepic_oracle as O
from paper_2512_16822_b200 import runtime as RT
from beam_helpers import BeamCase
from test_attn_beam_gpu import _built      # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def _point_at(case, r, head, slot, factor):
    """The key of row r's `slot` becomes `factor` times the query of that row and head, as seen from there."""
    e, s = slot // case.P, slot % case.P
    back = int(case.q_pos[r]) - (int(case.pos_base[r, e]) + s)
    q = bf16_bits_to_f64(case.q[r, head * (case.Hq // case.Hkv)])
    case.kp[case.page_ids[r, e], head, s] = f32_to_bf16_bits((factor * O.rope_rotate(q, np.array(back), case.theta)).astype(np.float32))


@pytest.mark.parametrize("D,W,fp8", [(64, 2, False), (128, 2, False), (128, 12, False), (128, 2, True), (128, 12, True)])
@pytest.mark.parametrize("falling", [False, True])
def test_references_that_rise_again_and_again(D, W, fp8, falling):
    # 41 keys that point at the query, a seventh longer from one to the next, a tile each and one beside it, in the middle of a long
    # context: every worker there (five to seven tiles each) meets several scores that are hundreds above all before them.  The last
    # one leads by 13 % of a score of thousands, so that the output is its V: the weight and the output are rounded once each.
    case = BeamCase(61, Hq=2, Hkv=2, D=D, P=16, width=W, specs=[(16000, 0)] * 4, theta=5e5, fp8=fp8)
    case.q[:] = np.repeat(case.q[::W], W, axis=0)                   # the beams of a group ask the same
    leads = np.zeros((4, 2), dtype=np.int64)
    for g in range(4):
        for h in range(2):
            for i in range(41):
                slot = 16 * (300 + 7 * g + (40 - i if falling else i)) + (5 * i + h) % 16
                _point_at(case, g * W, h, slot, 1.15 ** i)
                leads[g, h] = slot
    case.device()
    case.batch()
    out = case.run(1.0)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    got = bf16_bits_to_f64(RT.bf16_bits(out))
    if fp8:
        V = O.dequantize_pages(case.pools.v_codes.cpu().numpy(), case.pools.v_scales.cpu().numpy())
    else:
        V = bf16_bits_to_f64(case.vp)
    for r in range(4 * W):
        for h in range(2):
            slot = leads[r // W, h]
            want = V[case.page_ids[r, slot // 16], h, slot % 16]
            assert (np.abs(got[r, h] - want) <= np.abs(want) * ((1 + 2.0 ** -8) ** 2 - 1 + 2.0 ** -16)).all(), (r, h)


def test_the_scores_are_right_in_the_mean():
    # All keys of a context are zero, but for one that points at the query (score 30, V = 0), and all V are, but for a slot's among
    # the former: the output is 2^44 e^-30 or so, and its logarithm less the true one is what the score is off by.  A factor of a
    # product loses less than 2^-10 of itself, and the score gets (1 + 7.05e-4) back; the weight and the output are rounded (2^-8).
    Hkv, groups, n = 8, 40, 800
    case = BeamCase(62, Hq=Hkv, Hkv=Hkv, D=128, P=16, width=1, specs=[(n, 0)] * groups)
    case.kp[:], case.vp[:] = 0, 0
    sm_scale, at = 0.25, case.rng.integers(16, n, size=(groups, Hkv))
    for g in range(groups):
        case.vp[case.page_ids[g, 0], :, 3] = f32_to_bf16_bits(np.full((Hkv, 128), 2.0 ** 44, dtype=np.float32))
        for h in range(Hkv):
            q = bf16_bits_to_f64(case.q[g, h])
            _point_at(case, g, h, int(at[g, h]), 30.0 / (sm_scale * float(q @ q)))
    case.device()
    case.batch()
    out = case.run(sm_scale)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    got, off, score = bf16_bits_to_f64(RT.bf16_bits(out)), [], []
    for g in range(groups):
        want, _ = case.want(g, sm_scale)
        off += np.log(want[:, 0] / got[g, :, 0]).tolist()
        score += (-np.log(want[:, 0] / 2.0 ** 44)).tolist()           # (800 e^-30 beside 1: nothing)
    off, score = np.array(off), np.array(score)
    assert (np.abs(off) <= score * (2.0 ** -9 + 7.05e-4) + 2.0 ** -7 + 2.0 ** -12).all()
    # The mean of 320: roundings to nearest have none (a standard deviation of 0.0023 each for the weight and the output together, 1.3e-4
    # for the mean); what is cut off has, and not giving it back would show as 30 x 7.05e-4 = 0.021.  The mean of what is cut is taken
    # for spread mantissas, right to a seventh: 1e-4 of the score.
    assert abs(off.mean()) <= 30 * 1e-4 + 5 * 1.3e-4, off.mean()
