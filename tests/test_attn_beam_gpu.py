"""Attention of beams (mepic_beam_plan, mepic_attn_beam, mepic_attn_beam_fp8) against the fp64 oracle, row by row."""
import numpy as np
import pytest
import torch

import paper_2512_16822_b200 as M
from paper_2512_16822_b200 import runtime as RT
from paper_2512_16822_b200.build import build_library
from mepic_inputs import bf16_bits_to_f64
from beam_helpers import BeamCase, NAN_BITS, dev32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"


def _run(case, sm_scale=None, which=None):
    sm_scale = 1.0 / np.sqrt(case.D) if sm_scale is None else sm_scale
    case.device()
    case.batch()
    out = case.run(sm_scale)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    case.check(out, sm_scale, which)
    return out


EDGES = [(1, 0), (0, 1), (15, 1), (16, 1), (16, 0), (17, 15), (31, 33), (64, 0), (63, 2), (128, 130), (255, 1), (300, 40)]


@pytest.mark.parametrize("Hq,Hkv,D,P,W", [(8, 2, 128, 16, 4), (8, 2, 64, 16, 3), (1, 1, 128, 64, 1), (5, 1, 64, 32, 5), (8, 1, 128, 16, 4), (6, 2, 128, 32, 9),
                                          (7, 1, 64, 16, 2), (4, 2, 128, 128, 16), (2, 2, 128, 16, 32), (8, 1, 64, 64, 7), (4, 4, 64, 16, 20)])
def test_lengths_at_the_edges_of_pages_and_tiles(Hq, Hkv, D, P, W):
    case = BeamCase(Hq + D + P + W, Hq=Hq, Hkv=Hkv, D=D, P=P, width=W, specs=EDGES)
    case.poison()
    _run(case)


@pytest.mark.parametrize("Hq,Hkv,P,W", [(8, 2, 16, 4), (1, 1, 64, 1), (8, 1, 16, 5), (5, 1, 32, 6), (6, 2, 128, 3), (3, 1, 64, 32)])
def test_lengths_at_the_edges_over_8_bit_pages(Hq, Hkv, P, W):
    case = BeamCase(Hq + P + W, Hq=Hq, Hkv=Hkv, D=128, P=P, width=W, specs=EDGES, fp8=True)
    case.poison()
    _run(case)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("W", [3, 8])
def test_beams_of_a_group_may_have_lengths_of_their_own_and_none(W, fp8):
    rng = np.random.default_rng(3)
    specs = [(100, 90), (0, 40), (33, 0), (500, 200)]
    lens = np.concatenate([rng.integers(0, c + g + 1, size=W) for c, g in specs])
    lens[[0, W, 2 * W + 1]] = 0
    lens[2 * W] = 33
    _run(BeamCase(5 + W, Hq=8, Hkv=2, D=128, P=16, width=W, specs=specs, lens=lens, fp8=fp8))


def test_a_group_without_any_length_between_others():
    _run(BeamCase(6, Hq=4, Hkv=1, D=128, P=16, width=2, specs=[(0, 0), (40, 1), (0, 0), (0, 0), (5, 5), (0, 0)]))


@pytest.mark.parametrize("fp8", [False, True])
def test_any_tables_not_only_those_of_a_search(fp8):
    # pages held by any beams at any entries, the same page at several positions, lengths that end anywhere
    rng = np.random.default_rng(8)
    case = BeamCase(8, Hq=8, Hkv=2, D=128, P=16, width=6, specs=[(200, 0)] * 3, fp8=fp8)
    case.page_ids = rng.integers(0, 9, size=case.page_ids.shape).astype(np.int32)
    case.pos_base = (rng.integers(0, 3, size=case.pos_base.shape) * 40 + np.arange(case.pos_base.shape[1]) * 16).astype(np.int32)
    case.kv_len = rng.integers(1, 200, size=18).astype(np.int32)
    case.kv_len[3] = case.kv_len[4]
    case.finish()
    _run(case)


@pytest.mark.parametrize("D,fp8", [(64, False), (128, False), (128, True)])
def test_one_long_request_is_cut_along_its_keys(D, fp8):
    _run(BeamCase(11, Hq=4, Hkv=1, D=D, P=16, width=4, specs=[(5003, 60)], theta=5e5, fp8=fp8))


def test_many_groups():
    case = BeamCase(12, Hq=4, Hkv=2, D=128, P=16, width=3, specs=[(int(7 * i % 90), int(i % 23) + 1) for i in range(700)])
    _run(case, which=list(range(0, 2100, 37)) + [2099])


def test_rows_longer_than_a_segment_of_the_plan():
    # 256 table entries are a segment; the beams part in the second and in the third
    _run(BeamCase(13, Hq=8, Hkv=2, D=64, P=16, width=4, specs=[(4100, 3000), (10, 0), (8000, 500)], theta=5e5))


def test_more_groups_than_are_looked_through_in_two_rounds():
    # 32 column blocks are told apart at a time: 1,200 take three rounds; many of the groups have nothing
    rng = np.random.default_rng(28)
    specs = [(int(rng.integers(0, 40)) * int(rng.integers(0, 2)), int(rng.integers(0, 20)) * int(rng.integers(0, 2))) for _ in range(1200)]
    case = BeamCase(28, Hq=4, Hkv=2, D=64, P=16, width=2, specs=specs)
    _run(case, which=list(range(0, 2400, 41)) + [2398, 2399])


def test_a_row_of_more_segments_than_are_looked_through_at_a_time():
    # 33 stretches of 256 table entries and a part of one
    case = BeamCase(29, Hq=2, Hkv=1, D=64, P=16, width=2, specs=[(136_000, 40)], theta=5e5)
    case.pos_base = (case.pos_base // 8).astype(np.int32)             # (positions run into one another: the rope table need not reach as far)
    case.finish()
    _run(case)


@pytest.mark.parametrize("fp8", [False, True])
def test_large_pages(fp8):
    _run(BeamCase(30, Hq=4, Hkv=2, D=128, P=512, width=3, specs=[(1024, 700), (0, 1), (300, 212)], fp8=fp8))


@pytest.mark.parametrize("fp8", [False, True])
def test_what_a_beam_does_not_hold_has_no_influence(fp8):
    case = BeamCase(14, Hq=8, Hkv=2, D=128, P=16, width=4, specs=[(64, 20), (0, 9)], fp8=fp8)
    last = case.page_ids[1, (84 - 1) // 16]                     # beam 1's own page holds NaN, infinity and the largest numbers
    for pool in (case.kp, case.vp):
        pool[last, :, 0, :40] = NAN_BITS
        pool[last, :, 1, :40] = 0x7f80
        pool[last, :, 2, :40] = 0x7f7f
    sm_scale = 0.09
    case.device()
    case.batch()
    out = case.run(sm_scale)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    case.check(out, sm_scale, which=[0, 2, 3, 4, 5, 6, 7])
    got = bf16_bits_to_f64(RT.bf16_bits(out))[1]
    assert not np.isfinite(got[:, :40]).any()                   # ... and shows in its own output


def test_an_infinite_scale_of_one_beams_page():
    case = BeamCase(15, Hq=8, Hkv=2, D=128, P=16, width=4, specs=[(64, 20)], fp8=True)
    case.device()
    last = int(case.page_ids[2, (84 - 1) // 16])
    case.pools.k_scales[last] = float("inf")
    case.pools.v_scales[last] = float("inf")
    case.batch()
    out = case.run(0.09)
    torch.cuda.synchronize()
    case.check(out, 0.09, which=[0, 1, 3])
    assert not torch.isfinite(out[2].float()).any()


def test_scales_that_differ_by_orders_of_magnitude():
    # V scales from 1e-6 to 1e3 in one context, in an order of their own; K scales flat, so that every page has weight
    case = BeamCase(16, Hq=4, Hkv=1, D=128, P=16, width=3, specs=[(400, 50)], fp8=True)
    case.device()
    rng = np.random.default_rng(16)
    for lo, hi in ((-6, 3), (-3, -2.5)):
        case.pools.v_scales.copy_(torch.from_numpy(10.0 ** rng.uniform(lo, hi, size=tuple(case.pools.v_scales.shape)).astype(np.float32)))
        if hasattr(case, "_deq"):
            del case._deq
        case.batch()
        out = case.run(0.05)
        torch.cuda.synchronize()
        got = bf16_bits_to_f64(RT.bf16_bits(out))
        for r in range(3):
            want, sigma = case.want(r, 0.05)
            # sigma scales with V; the fp32 terms (2^-16 of the largest |V| are ample) in place of the absolute 1e-4
            assert (np.abs(got[r] - want) <= 7 * sigma + 2.0 ** -16 * np.abs(want).max()).all()


def test_8_bit_pages_whose_values_are_tiny():
    case = BeamCase(17, Hq=4, Hkv=1, D=128, P=16, width=2, specs=[(900, 30)], fp8=True)
    case.device()
    case.pools.v_scales.mul_(1e-12)
    case.batch()
    out = case.run(0.09)
    torch.cuda.synchronize()
    got = bf16_bits_to_f64(RT.bf16_bits(out))
    for r in range(2):
        want, sigma = case.want(r, 0.09)
        assert (np.abs(got[r] - want) <= 7 * sigma + 1e-16).all()


def test_scales_of_either_sign():
    # the oracle takes a page's values as code x scale, whatever its sign
    case = BeamCase(25, Hq=4, Hkv=2, D=128, P=16, width=3, specs=[(200, 30)], fp8=True)
    case.device()
    rng = np.random.default_rng(25)
    for scales in (case.pools.k_scales, case.pools.v_scales):
        scales.mul_(torch.from_numpy(rng.choice([-1.0, 1.0], size=tuple(scales.shape)).astype(np.float32)).cuda())
    case.pools.v_scales.neg_()
    case.pools.v_scales[int(case.page_ids[0, 0])].abs_().neg_()            # the first page met has a negative one
    case.batch()
    out = case.run(0.09)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    case.check(out, 0.09)


@pytest.mark.parametrize("D,fp8", [(64, False), (128, False), (128, True)])
def test_negative_positions_and_a_rope_table_shorter_than_the_context(D, fp8):
    # positions -176 .. 176, the query at 0: a key may be further from the first than the table reaches
    case = BeamCase(26, Hq=4, Hkv=2, D=D, P=16, width=2, specs=[(320, 30)], fp8=fp8)
    case.pos_base[:] = np.arange(case.pos_base.shape[1]) * 16 - 176
    case.q_pos[:] = 0
    case.max_position = 176
    case.cfg = M.Config(16, 4, 2, D, case.num_pages, 176, case.theta)
    case.device()
    case.batch()
    out = case.run(0.09)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    case.check(out, 0.09)


def test_what_a_dropped_call_holds_is_not_handed_out_while_it_runs():
    case = BeamCase(27, Hq=8, Hkv=2, D=128, P=16, width=4, specs=[(700, 100), (90, 33)])
    case.device()
    side = torch.cuda.Stream()
    case.batch()
    case.plan.run(side), case.attn.run(0.09, side)                  # what happens once is not waited for below
    torch.cuda.synchronize()
    case.batch()
    held = {t.data_ptr(): t.numel() for t in (case.plan.plan, case.attn.workspace)}
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(1_000_000_000)                            # half a second: the calls are still in the queue when their objects go
        case.plan.run()
        out = case.attn.run(0.09)
    del case.plan, case.attn
    early = not side.query()
    others = [torch.empty(n, dtype=torch.uint8, device="cuda:0") for n in held.values()]
    torch.cuda.synchronize()
    assert early, "the kernels were through before the memory was asked for"
    assert not {t.data_ptr() for t in others} & set(held)
    assert case.dev.read_status() == 0
    case.check(out, 0.09)


def test_scores_whose_exponentials_do_not_fit():
    # scores of some thousands: only differences from the largest count
    case = BeamCase(18, Hq=8, Hkv=2, D=128, P=16, width=4, specs=[(200, 30)])
    case.device()
    case.batch()
    out = case.run(40.0)
    torch.cuda.synchronize()
    got = bf16_bits_to_f64(RT.bf16_bits(out))
    assert np.isfinite(got).all()
    assert np.abs(got).max() <= float(np.abs(bf16_bits_to_f64(case.vp)).max())


def test_a_single_slot_gives_its_value_bit_for_bit():
    case = BeamCase(19, Hq=4, Hkv=2, D=128, P=16, width=3, specs=[(0, 1), (1, 0)])
    out = _run(case)
    got = RT.bf16_bits(out)
    for r in range(6):
        assert (got[r].reshape(2, 2, 128) == case.vp[case.page_ids[r, 0], :, 0][:, None]).all()


def test_same_input_same_bits_and_no_trace_of_the_last_call():
    case = BeamCase(20, Hq=8, Hkv=2, D=128, P=16, width=4, specs=[(700, 100), (31, 9)])
    first = _run(case).clone()
    for fill in (0, 255):
        case.attn.workspace.fill_(fill)
        case.plan.plan.fill_(fill)
        again = case.run(1.0 / np.sqrt(128))
        torch.cuda.synchronize()
        assert case.dev.read_status() == 0 and torch.equal(first.view(torch.int16), again.view(torch.int16))


def test_captured_and_replayed_with_other_lengths_and_tables():
    case = BeamCase(21, Hq=8, Hkv=2, D=128, P=16, width=4, specs=[(700, 100), (90, 33)])
    case.device()
    case.batch()
    case.run(0.09)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = case.run(0.09)
    rng = np.random.default_rng(21)
    for _ in range(3):
        case.kv_len = np.concatenate([rng.integers(0, 801, size=4), rng.integers(0, 124, size=4)]).astype(np.int32)
        swap = rng.permutation(4)
        case.page_ids[:4], case.pos_base[:4] = case.page_ids[swap], case.pos_base[swap]
        last = np.maximum(case.kv_len - 1, 0)
        case.q_pos = np.where(case.kv_len > 0, case.pos_base[np.arange(8), last // 16].astype(np.int64) + last % 16, 0)
        case.d_len.copy_(dev32(case.kv_len)), case.d_ids.copy_(dev32(case.page_ids)), case.d_qpos.copy_(dev32(case.q_pos))
        graph.replay()
        torch.cuda.synchronize()
        assert case.dev.read_status() == 0
        case.check(out, 0.09)


@pytest.mark.parametrize("captured", [False, True])
def test_queries_written_just_before_and_on_another_stream(captured):
    # the attention may be in place before what precedes it is done: the queries change on a side stream that is joined between
    # the plan and the attention, and in the launch right before it
    case = BeamCase(31, Hq=8, Hkv=2, D=128, P=16, width=4, specs=[(700, 100), (90, 33)])
    case.device()
    good = case.fused_q()
    q, half = torch.zeros_like(good), good.shape[0] // 2
    case.batch(q)
    side = torch.cuda.Stream()

    def step():
        main = torch.cuda.current_stream()
        q.zero_()
        case.plan.run()
        side.wait_stream(main)
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000)
            q[:half].copy_(good[:half])
        main.wait_stream(side)
        first = case.attn.run(0.09).clone()
        torch.cuda._sleep(100_000)
        q[half:].copy_(good[half:])
        return first, case.attn.run(0.09)

    if captured:
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            first, out = step()
        for _ in range(3):
            out.zero_()
            graph.replay()
    else:
        for _ in range(3):
            first, out = step()
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    case.check(first, 0.09, which=range(half))
    case.check(out, 0.09)


def test_layers_share_a_plan_and_run_on_two_streams():
    case = BeamCase(22, Hq=8, Hkv=2, D=128, P=16, width=4, specs=[(700, 100), (90, 33)])
    case.device()
    case.batch()
    other = RT.Device.over(case.cfg, case.dev.k_pool.flip(0).contiguous(), case.dev.v_pool.flip(0).contiguous(), rope=case.dev.rope)
    second = RT.BeamBatch(other, q=case.fused_q(), q_pos=case.d_qpos, plan=case.plan)
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    case.plan.run()
    for s in sides:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        a, b = case.attn.run(0.09, sides[0]), second.run(0.09, sides[1])
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0 and other.read_status() == 0
    case.check(a, 0.09)
    case.kp, case.vp = case.kp[::-1], case.vp[::-1]
    case.check(b, 0.09)


@pytest.mark.parametrize("how", ["never made", "another shape", "overwritten"])
def test_a_plan_that_does_not_fit_is_reported(how):
    case = BeamCase(23, Hq=8, Hkv=2, D=128, P=16, width=4, specs=[(70, 10), (90, 33)])
    case.device()
    case.batch()
    if how == "another shape":
        # the bytes of a plan made for two groups of two beams
        M.mepic_beam_plan(case.cfg, page_ids=case.d_ids, pos_base=case.d_base, kv_len=case.d_len, plan=case.plan.plan, plan_bytes=case.plan.plan.numel(),
                          status=case.dev.status, table_stride=case.plan.stride, groups=2, width=2)
    elif how == "overwritten":
        case.plan.run()
        case.plan.plan.view(torch.int32)[16:40] = 0x7fffffff
    out = case.attn.run(0.09)
    torch.cuda.synchronize()
    assert case.dev.read_status() == M.MEPIC_DEV_BAD_PLAN
    assert (out == 0).all()
    case.dev.status.zero_()
    out = case.run(0.09)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    case.check(out, 0.09)


def test_bad_lengths_pages_and_positions_are_reported_and_harmless():
    case = BeamCase(24, Hq=8, Hkv=2, D=128, P=16, width=4, specs=[(70, 10), (90, 33)])
    case.device()
    case.batch()
    stride = case.page_ids.shape[1]
    for name, at, value, bit, rows in (("d_len", 1, -5, M.MEPIC_DEV_BAD_SLOT, [0, 2, 3, 4, 5, 6, 7]), ("d_len", 6, stride * 16 + 1, M.MEPIC_DEV_BAD_SLOT, [0, 1, 2, 3, 4, 5, 7]),
                                       ("d_ids", (5, 2), case.num_pages, M.MEPIC_DEV_BAD_PAGE, [0, 1, 2, 3, 4, 6, 7]), ("d_ids", (5, 2), -1, M.MEPIC_DEV_BAD_PAGE, [0, 1, 2, 3, 4, 6, 7]),
                                       ("d_qpos", 2, case.max_position + 500, M.MEPIC_DEV_BAD_POSITION, [0, 1, 3, 4, 5, 6, 7])):
        t = getattr(case, name)
        keep = t.clone()
        t[at] = value
        out = case.run(0.09)
        torch.cuda.synchronize()
        # (a length past its own entries reads what the table holds there: pages and positions that are none)
        assert case.dev.read_status() & bit, name
        case.check(out, 0.09, rows)
        case.dev.status.zero_()
        t.copy_(keep)


def test_a_copy_that_never_comes():
    case = BeamCase(25, Hq=2, Hkv=1, D=128, P=16, width=3, specs=[(70000, 40)], theta=5e5)      # several tiles a worker
    case.device()
    case.batch()
    for tile in (0, 2):
        M.mepic_kernel_test_hooks(spin_limit=20000, skip_tile=tile)      # tens of milliseconds, then the wait gives up
        try:
            case.run(0.09)
            torch.cuda.synchronize()
        finally:
            M.mepic_kernel_test_hooks()
        assert case.dev.read_status() == M.MEPIC_DEV_WAIT_EXPIRED
        case.dev.status.zero_()
        out = case.run(0.09)
        torch.cuda.synchronize()
        assert case.dev.read_status() == 0
        case.check(out, 0.09)


@pytest.mark.parametrize("seed", range(12))
def test_random_shapes(seed):
    rng = np.random.default_rng(1000 + seed)
    Hkv = int(rng.integers(1, 5))
    G, D = int(rng.integers(1, 9)), int(rng.choice([64, 128]))
    W = int(rng.integers(1, 33))
    specs = [(int(rng.integers(0, 600)), int(rng.integers(1, 120))) for _ in range(int(rng.integers(1, 6)))]
    case = BeamCase(seed, Hq=G * Hkv, Hkv=Hkv, D=D, P=int(rng.choice([16, 32, 64, 128])), width=W, specs=specs, fp8=bool(D == 128 and rng.random() < 0.4), scale=float(rng.choice([0.5, 1, 3])))
    rows = sorted(set(rng.integers(0, len(specs) * W, size=10).tolist()))
    _run(case, which=rows)


def test_pages_past_32_bits_of_elements():
    # the pools hold more than 2^32 elements; the context lies at their end
    P, Hkv, D = 16, 8, 128
    pages = (1 << 32) // (Hkv * P * D) + 40
    case = BeamCase(26, Hq=16, Hkv=Hkv, D=D, P=P, width=2, specs=[(100, 20)])
    cfg = M.Config(P, 16, Hkv, D, pages, case.max_position, case.theta)
    first = pages - case.num_pages
    kp, vp = (torch.empty((pages, Hkv, P, D), dtype=torch.bfloat16, device="cuda:0") for _ in range(2))
    kp[first:], vp[first:] = RT.bf16_tensor(case.kp, "cuda:0"), RT.bf16_tensor(case.vp, "cuda:0")
    case.dev, case.pools = RT.Device.over(cfg, kp, vp), None
    case.d_ids, case.d_base, case.d_len, case.d_qpos = dev32(case.page_ids + first), dev32(case.pos_base), dev32(case.kv_len), dev32(case.q_pos)
    case.batch()
    out = case.run(0.09)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    case.check(out, 0.09)
