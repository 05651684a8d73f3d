"""Attention of beams over 8-bit pages whose V scales lie far apart: a page's scale is its own beams' affair.  The contexts are long
enough for several tiles a worker, and pages of the odd kind lie in every worker's stretch."""
import numpy as np
import pytest
import torch

from mepic_inputs import bf16_bits_to_f64, f32_to_bf16_bits
from oracle import mepic_oracle as O
from paper_2512_16822_b200 import runtime as RT
from beam_helpers import BeamCase
from test_attn_beam_gpu import _built      # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu
GROUPS, SLOTS = 4, 16000


def _case(seed, W, P=16, Hq=4):
    return BeamCase(seed, Hq=Hq, Hkv=2, D=128, P=P, width=W, specs=[(SLOTS, 0)] * GROUPS, theta=5e5, fp8=True, extra_pages=GROUPS * (SLOTS // P // 11 + 1))


def _run(case, sm_scale):
    case.batch()
    out = case.run(sm_scale)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    return out


def _follows_the_scale(case, out, sm_scale, rows):
    # sigma scales with V; the fp32 terms (2^-16 of the largest output) in place of an absolute 1e-4
    got = bf16_bits_to_f64(RT.bf16_bits(out))
    for r in rows:
        want, sigma = case.want(r, sm_scale)
        err, tol = np.abs(got[r] - want), 7 * sigma + 2.0 ** -16 * np.abs(want).max()
        assert (err <= tol).all(), (r, float((err / tol).max()))


@pytest.mark.parametrize("scale", [1e4, 1e10, 1e30, -1e10, 1e-10, 1e-30])
@pytest.mark.parametrize("W,P", [(2, 16), (8, 16), (3, 64)])
def test_one_beams_pages_with_a_scale_far_from_the_others(W, P, scale):
    # beam 1 holds a page of its own where the others share one, at every eleventh entry
    case = _case(W + P, W, P)
    spare = iter(sorted(set(range(case.num_pages)) - set(case.page_ids.reshape(-1).tolist())))
    own = []
    for g in range(GROUPS):
        for e in range(5, SLOTS // P, 11):
            own.append(next(spare))
            case.page_ids[g * W + 1, e] = own[-1]
    case.device()
    case.pools.v_scales[own] = scale
    out = _run(case, 0.09)
    case.check(out, 0.09, which=[g * W + w for g in (0, GROUPS - 1) for w in (0, W - 1) if w != 1])
    _follows_the_scale(case, out, 0.09, [1])                       # its own output has it


@pytest.mark.parametrize("scale", [1e6, 1e10, 1e30])
def test_pages_of_all_beams_that_have_next_to_no_weight(scale):
    # their keys point away from the query (scores of -115 or so): e^-115 of the largest scale there is here is still nothing
    W = 3
    case = _case(42, W, Hq=2)
    case.q[:] = np.repeat(case.q[::W], W, axis=0)
    odd = []
    for g in range(GROUPS):
        for e in range(5, SLOTS // 16, 11):
            odd.append(int(case.page_ids[g * W, e]))
            back = int(case.q_pos[g * W]) - (int(case.pos_base[g * W, e]) + np.arange(16))
            for h in range(2):
                q = bf16_bits_to_f64(case.q[g * W, h])
                case.kp[odd[-1], h] = f32_to_bf16_bits((-10 * O.rope_rotate(np.repeat(q[None], 16, 0), back, case.theta)).astype(np.float32))
    case.device()
    case.pools.v_scales[odd] = scale
    case.check(_run(case, 0.09), 0.09, which=[0, 2, GROUPS * W - 1])


def test_scales_that_change_at_every_page():
    # up and down by ten orders of magnitude, of either sign, pages that all beams hold and pages of their own in turn
    case = BeamCase(43, Hq=4, Hkv=2, D=128, P=16, width=4, specs=[(SLOTS, 200)] * GROUPS, theta=5e5, fp8=True)
    case.device()
    rng, shape = np.random.default_rng(43), tuple(case.pools.v_scales.shape)
    case.pools.v_scales.copy_(torch.from_numpy((10.0 ** rng.uniform(-5, 5, size=shape) * rng.choice([-1.0, 1.0], size=shape)).astype(np.float32)))
    _follows_the_scale(case, _run(case, 0.05), 0.05, [0, 1, 2, 3, GROUPS * 4 - 1])
