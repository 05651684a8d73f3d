"""Attention of drafted rows (mepic_attn_tree, mepic_attn_tree_fp8) against the fp64 oracle.

The tolerance is per element and follows from the roundings the call is allowed (TreeCase.check): it is tight enough that a
wrong mask bit, position, page or scale does not fit into it.
"""
import numpy as np
import pytest
import torch

import paper_2512_16822_b200 as M
from paper_2512_16822_b200 import runtime as RT
from paper_2512_16822_b200.build import build_library
from mepic_inputs import bf16_bits_to_f64
from oracle import mepic_oracle as O
from tree_helpers import TreeCase, dev32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"


def _run(case, sm_scale, **kw):
    case.device()
    batch = case.batch(**kw)
    out = batch.run(sm_scale)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    case.check(out, sm_scale)
    return batch


EDGES = [(0, 1), (0, 9), (1, 1), (1, 5), (15, 3), (16, 1), (17, 2), (127, 4), (128, 3), (129, 7), (300, 0), (255, 6), (257, 11)]


@pytest.mark.parametrize("Hq,Hkv,D,P", [(8, 2, 128, 16), (8, 2, 64, 16), (1, 1, 128, 64), (5, 1, 64, 32), (8, 1, 128, 16), (6, 2, 128, 32),
                                        (7, 1, 64, 16), (4, 2, 128, 128)])
def test_lengths_at_the_edges_of_pages_and_tiles(Hq, Hkv, D, P):
    _run(TreeCase(Hq * 10 + D + P, Hq=Hq, Hkv=Hkv, D=D, P=P, specs=EDGES), 1.0 / np.sqrt(D))


@pytest.mark.parametrize("Hq,Hkv,P", [(8, 2, 16), (1, 1, 64), (8, 1, 16), (5, 1, 32), (6, 2, 128)])
def test_lengths_at_the_edges_over_8_bit_pages(Hq, Hkv, P):
    _run(TreeCase(Hq + P, Hq=Hq, Hkv=Hkv, D=128, P=P, specs=EDGES, fp8=True), 1.0 / np.sqrt(128))


@pytest.mark.parametrize("kind", ["tree", "chain", "star"])
@pytest.mark.parametrize("fp8", [False, True])
def test_trees_larger_than_a_tile_of_keys_and_of_rows(kind, fp8):
    # 128-row query tiles and 128-key draft tiles are both passed: up to 300 rows x 4 heads = 10 query tiles, 3 draft tiles
    _run(TreeCase(7, Hq=8, Hkv=2, D=128, P=16, specs=[(70, 131), (0, 300), (500, 1), (129, 33)], kind=kind, fp8=fp8), 0.09)


@pytest.mark.parametrize("D", [64, 128])
def test_one_long_request_is_cut_along_its_keys(D):
    _run(TreeCase(11, Hq=4, Hkv=1, D=D, P=16, specs=[(5003, 6)], theta=5e5), 1.0 / np.sqrt(D))


def test_one_long_request_over_8_bit_pages():
    _run(TreeCase(12, Hq=4, Hkv=1, D=128, P=64, specs=[(5003, 6)], theta=5e5, fp8=True), 1.0 / np.sqrt(128))


def test_more_requests_than_multiprocessors():
    rng = np.random.default_rng(5)
    specs = [(int(rng.integers(0, 200)), int(rng.integers(0, 4))) for _ in range(333)]
    _run(TreeCase(13, Hq=4, Hkv=2, D=128, P=16, specs=specs), 1.0 / np.sqrt(128))


def test_ragged_rows_and_a_bound_above_them():
    # max_rows only bounds: a larger bound (another split of the work) gives the same result within the tolerance
    case = TreeCase(14, Hq=8, Hkv=1, D=128, P=16, specs=[(400, 2), (900, 60), (33, 17), (1200, 1)])
    case.words = 4
    _run(case, 0.09, max_rows=128)


@pytest.mark.parametrize("fp8", [False, True])
def test_loud_scores_move_the_running_maximum(fp8):
    # scores of standard deviation ~12 (base-2 units ~17): the reference rises again and again, most weights vanish
    case = TreeCase(15, Hq=4, Hkv=1, D=128, P=16, specs=[(1500, 9), (130, 40)], fp8=fp8, scale=12.0)
    case.device()
    out = case.batch().run(1.0 / np.sqrt(128))
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    # first-order propagation does not hold for score errors of order 1; what does: the weights are a distribution, so every
    # output lies between the smallest and the largest V the row sees (plus a rounding), and rows agree in the mean
    got = bf16_bits_to_f64(RT.bf16_bits(out))
    for b in range(2):
        want, _ = case.want(b, 1.0 / np.sqrt(128))
        g = got[case.off[b]:case.off[b + 1]]
        assert np.isfinite(g).all() and np.abs(g).max() <= 6.0
        # score errors: |ds| <= 2 * 2^-8 * sum |q k| sm ~ 0.7 at worst, 0.06 r.m.s.: a weight moves by a few per cent
        assert np.linalg.norm(g - want) <= 0.1 * np.linalg.norm(want)


def test_scores_rise_and_fall_by_hundreds():
    # keys whose scores grow tile by tile, then one dominant key, then small ones: the sum before a jump must be scaled away
    case = TreeCase(16, Hq=4, Hkv=1, D=64, P=16, specs=[(1024, 3)], jitter=False, theta=1e9)
    # only pairs that 1024 positions turn by less than 0.04 rad (theta = 1e9, i >= 16), so that scores go by the amplitudes:
    # 0.125 * |q|^2-like factors of ~5.6 times the amplitude, 420 for the dominant key against 252 for the next
    case.q[:] = case.q[0, 0]
    case.q[:, :, 0:16], case.q[:, :, 32:48] = 0, 0
    unit = bf16_bits_to_f64(case.q)[0, 0]
    unit = unit / np.linalg.norm(unit)
    from mepic_inputs import f32_to_bf16_bits
    amp = np.where(np.arange(1024) < 900, np.arange(1024) * 0.4, 1.0)
    amp[700] = 600.0
    for t in range(1024):
        case.kp[case.page_ids[0, t // 16], 0, t % 16] = f32_to_bf16_bits((amp[t] * unit).astype(np.float32))
    case.device()
    out = case.batch().run(0.125)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    got = bf16_bits_to_f64(RT.bf16_bits(out))
    want, _ = case.want(0, 0.125)
    assert np.isfinite(got).all()
    assert np.abs(got - want).max() <= 2 ** -7 * np.abs(want).max()     # one key carries the weight: V of it, rounded (P = 2^k exactly or rounded: two roundings)


@pytest.mark.parametrize("fp8", [False, True])
def test_what_a_mask_hides_has_no_influence(fp8):
    # NaN and infinities in rows somebody else may see, in pages past kv_len, and in the row arrays between requests
    case = TreeCase(17, Hq=4, Hkv=1, D=128, P=16, specs=[(37, 6), (200, 5), (0, 3)], kind="star", fp8=fp8)
    sees = case.sees[0]
    sees[:] = False
    sees[0, [0, 1]] = True
    sees[1, [1]] = True
    sees[2, [3]] = True
    case.sees[1][4, :] = False                                          # a row that does not even see itself
    case.sees[2][1, :] = False                                          # ... and has no context: nothing at all -> zeros
    if not fp8:
        last = case.page_ids[0, 2]
        case.kp[last, :, 5:], case.vp[last, :, 5:] = 0x7fc0, 0x7f80
    nan, inf = 0x7fc0, 0xff80
    for bad in (2, 4, 5):
        case.kn[bad], case.vn[bad] = nan, inf
        case.vn[bad, :, ::3] = nan
    clean_rows = [0, 1]
    case.device()
    out = case.batch().run(0.09)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    got = bf16_bits_to_f64(RT.bf16_bits(out))
    keep_k, keep_v = case.kn.copy(), case.vn.copy()
    for b in range(3):
        case_rows = slice(case.off[b], case.off[b + 1])
        n = int(case.rows[b])
        want, sigma = case.want(b, 0.09)
        for i in range(n):
            assert np.isfinite(want[i]).all()
            assert (np.abs(got[case.off[b] + i] - want[i]) <= 7 * sigma[i] + 1e-4).all(), (b, i)
    assert (got[case.off[2] + 1] == 0).all()


def test_a_visible_infinity_reaches_exactly_the_rows_that_see_it():
    case = TreeCase(18, Hq=4, Hkv=1, D=128, P=16, specs=[(150, 8)], kind="chain")
    case.vn[5, 0, 3], case.vn[5, 0, 64], case.vn[6, 0, 3] = 0x7f80, 0x7fc0, 0xff80      # +inf, NaN; -inf one row later
    case.device()
    out = case.batch().run(0.09)
    torch.cuda.synchronize()
    got = bf16_bits_to_f64(RT.bf16_bits(out))
    with np.errstate(invalid="ignore"):
        want, _ = case.want(0, 0.09)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isposinf(got), np.isposinf(want))
    fine = np.isfinite(want)
    case.vn[5, 0, [3, 64]], case.vn[6, 0, 3] = 0, 0
    clean, sigma = case.want(0, 0.09)
    assert (np.abs(got - clean)[fine] <= (7 * sigma + 1e-4)[fine]).all()


def test_packed_rows_strided_rows_and_rows_nobody_owns():
    case = TreeCase(19, Hq=8, Hkv=2, D=128, P=16, specs=[(90, 5), (260, 4)], stride_extra=24)
    case.device()
    strided = case.batch().run(0.09).clone()
    packed = case.batch(rows=tuple(RT.bf16_tensor(x, "cuda:0") for x in (case.q, case.kn, case.vn))).run(0.09).clone()
    torch.cuda.synchronize()
    assert torch.equal(strided, packed)
    case.check(strided, 0.09)
    # three rows behind the last request: their outputs stay as they were
    q, k, v = (torch.cat([RT.bf16_tensor(x, "cuda:0"), torch.full((3,) + x.shape[1:], float("nan"), dtype=torch.bfloat16, device="cuda:0")])
               for x in (case.q, case.kn, case.vn))
    total = int(case.off[-1])
    b = RT.TreeBatch(case.dev, q=q, k_new=k, v_new=v, row_offsets=dev32(case.off), row_pos=dev32(np.concatenate(case.row_pos + [[-5, -5, -5]])),
                     tree_mask=dev32(np.concatenate([case.mask(), np.full((3, case.words), -1)])), page_ids=dev32(case.page_ids),
                     pos_base=dev32(case.pos_base), kv_len=dev32(case.kv_len), max_rows=5)
    b.out.fill_(7.0)
    b.run(0.09)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    assert torch.equal(b.out[:total], packed) and (b.out[total:] == 7.0).all()


def test_same_call_gives_the_same_bits():
    case = TreeCase(20, Hq=8, Hkv=2, D=128, P=16, specs=[(1000, 9), (3, 2), (2000, 30)])
    batch = _run(case, 0.09)
    first = batch.out.clone()
    for _ in range(3):
        batch.workspace.fill_(255)
        batch.run(0.09)
    torch.cuda.synchronize()
    assert torch.equal(batch.out, first)


@pytest.mark.parametrize("fp8", [False, True])
def test_captured_call_replayed_with_other_lengths(fp8):
    case = TreeCase(21, Hq=4, Hkv=2, D=128, P=16, specs=[(700, 5), (300, 5)], jitter=False, fp8=fp8)
    case.device()
    batch = case.batch()
    batch.run(0.09)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        batch.run(0.09)
    for lens in ([700, 300], [1, 299], [513, 0], [640, 128]):
        case.kv_len[:] = lens
        case.d_kv.copy_(dev32(case.kv_len))
        batch.out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert case.dev.read_status() == 0
        case.check(batch.out, 0.09)


def test_two_streams_with_workspaces_of_their_own():
    a = TreeCase(22, Hq=8, Hkv=2, D=128, P=16, specs=[(3000, 7)] * 3)
    b = TreeCase(23, Hq=4, Hkv=1, D=64, P=32, specs=[(2000, 40)])
    a.device(), b.device()
    ba, bb = a.batch(), b.batch()
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        ba.run(0.09, s)
        bb.run(0.125, t)
    torch.cuda.synchronize()
    a.check(ba.out, 0.09), b.check(bb.out, 0.125)


def test_agrees_with_decode_on_a_committed_token():
    # the newest token as the only drafted row equals decode with the same token already in its page
    case = TreeCase(24, Hq=8, Hkv=2, D=128, P=16, specs=[(500, 1), (33, 1)], jitter=False)
    case.device()
    tree = bf16_bits_to_f64(RT.bf16_bits(case.batch().run(0.09)))
    for b in range(2):
        n = int(case.kv_len[b])
        for pool, new in ((case.dev.k_pool, case.kn), (case.dev.v_pool, case.vn)):
            pool[int(case.page_ids[b, n // 16]) if n % 16 else 0, :, n % 16] = RT.bf16_tensor(new[b], "cuda:0")
    d = RT.DecodeBatch(case.dev, np.maximum(case.page_ids, 0), np.where(case.pos_base < 1 << 30, case.pos_base, 0), case.kv_len + 1,
                       np.array([p[0] for p in case.row_pos], dtype=np.int32), case.q)
    got = bf16_bits_to_f64(RT.bf16_bits(d.run(0.09)))
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    assert np.abs(got - tree).max() <= 2e-2 and np.abs(got - tree).mean() <= 2e-3      # decode's stated tolerance


# ------------------------------------------------------------------------------------ malformed device data: reported, not faulted
def _status_of(case, **kw):
    case.device()
    batch = case.batch(**kw)
    batch.run(0.09)
    torch.cuda.synchronize()
    return case.dev.read_status(), batch


@pytest.mark.parametrize("fp8", [False, True])
def test_bad_page_position_and_length_are_reported(fp8):
    kw = dict(Hq=4, Hkv=1, D=128, P=16, specs=[(100, 3), (50, 2)], fp8=fp8)
    case = TreeCase(30, **kw)
    case.page_ids[0, 3] = case.num_pages + 4
    assert _status_of(case)[0] == M.MEPIC_DEV_BAD_PAGE
    case = TreeCase(30, **kw)
    case.page_ids[1, 0] = -2
    assert _status_of(case)[0] == M.MEPIC_DEV_BAD_PAGE
    case = TreeCase(30, **kw)
    case.pos_base[0, 2] = case.max_position + 100
    assert _status_of(case)[0] == M.MEPIC_DEV_BAD_POSITION
    case = TreeCase(30, **kw)
    case.row_pos[1][1] = -3
    assert _status_of(case)[0] == M.MEPIC_DEV_BAD_POSITION
    case = TreeCase(30, **kw)
    case.kv_len[0] = -4
    status, batch = _status_of(case)
    assert status == M.MEPIC_DEV_BAD_SLOT
    case.kv_len[0] = 0
    case.check(batch.out, 0.09)
    case = TreeCase(30, **kw)
    case.kv_len[0] = 10 ** 9
    assert _status_of(case)[0] & M.MEPIC_DEV_BAD_SLOT


def test_more_rows_than_announced_are_reported_and_left():
    case = TreeCase(31, Hq=4, Hkv=1, D=128, P=16, specs=[(100, 3), (50, 9), (20, 2)])
    case.device()
    batch = case.batch(max_rows=4)
    batch.out.fill_(7.0)
    batch.run(0.09)
    torch.cuda.synchronize()
    assert case.dev.read_status() == M.MEPIC_DEV_BAD_TREE
    lo = int(case.off[1])
    assert (batch.out[lo + 4:lo + 9] == 7.0).all() and (batch.out[:lo + 4] != 7.0).any(dim=-1).all()
    case.check(batch.out, 0.09, which=[0, 2])


@pytest.mark.parametrize("off", [[0, 5, 3], [0, 9, 2000], [-4, 3, 5], [7, 3, 5]])
def test_row_offsets_that_make_no_sense_are_reported(off):
    case = TreeCase(32, Hq=4, Hkv=1, D=128, P=16, specs=[(100, 3), (50, 2)])
    case.off[:] = off
    good = case.off
    case.device()
    total = 5
    b = RT.TreeBatch(case.dev, q=RT.bf16_tensor(case.q, "cuda:0"), k_new=RT.bf16_tensor(case.kn, "cuda:0"), v_new=RT.bf16_tensor(case.vn, "cuda:0"),
                     row_offsets=dev32(good), row_pos=dev32(np.concatenate(case.row_pos)),
                     tree_mask=dev32(np.concatenate([O.pack_mask(s, case.words) for s in case.sees])), page_ids=dev32(case.page_ids),
                     pos_base=dev32(case.pos_base), kv_len=dev32(case.kv_len), max_rows=5)
    b.run(0.09)
    torch.cuda.synchronize()
    assert case.dev.read_status() & M.MEPIC_DEV_BAD_TREE


def test_no_rows_launch_nothing():
    case = TreeCase(33, Hq=4, Hkv=1, D=128, P=16, specs=[(100, 0)])
    case.device()
    before = M.mepic_launch_count()
    q = torch.empty((0, 4, 128), dtype=torch.bfloat16, device="cuda:0")
    k = torch.empty((0, 1, 128), dtype=torch.bfloat16, device="cuda:0")
    RT.TreeBatch(case.dev, q=q, k_new=k, v_new=k, row_offsets=dev32([0, 0]), row_pos=dev32([]), tree_mask=torch.empty((0, 1), dtype=torch.int32, device="cuda:0"),
                 page_ids=dev32(case.page_ids), pos_base=dev32(case.pos_base), kv_len=dev32(case.kv_len), max_rows=0).run(0.1)
    assert M.mepic_launch_count() == before


@pytest.mark.parametrize("fp8", [False, True])
def test_pages_whose_elements_lie_past_32_bits(fp8):
    # pools of 2.6 G elements each; the case's pages are spread over them, the last page included, and the rest is never read.
    # Committed rows land there too.
    Hkv, P, D, pages = 8, 64, 128, 40000
    case = TreeCase(60, Hq=8, Hkv=Hkv, D=D, P=P, specs=[(700, 5), (130, 3)], jitter=False, fp8=fp8)
    case.device()
    small = case.dev
    where = np.linspace(1000, pages - 1, case.num_pages).astype(np.int64)
    cfg = M.Config(P, 8, Hkv, D, pages, case.max_position, case.theta)
    src = (small.k_pool, small.v_pool) if not fp8 else (case.pools.k_codes, case.pools.v_codes)
    big = [torch.empty((pages, Hkv, P, D), dtype=s.dtype, device="cuda:0") for s in src]
    for b, s in zip(big, src):
        b[torch.from_numpy(where).cuda()] = s
    pools = None
    if fp8:
        scales = []
        for s in (case.pools.k_scales, case.pools.v_scales):
            scales.append(torch.ones((pages, Hkv), dtype=torch.float32, device="cuda:0"))
            scales[-1][torch.from_numpy(where).cuda()] = s
    dev = RT.Device.over(cfg, None if fp8 else big[0], None if fp8 else big[1])
    if fp8:
        pools = RT.Fp8Pools.over(dev, *big, *scales)
    ids = np.where(case.page_ids >= 0, where[np.maximum(case.page_ids, 0)], -1)
    q, k, v = case.fused()
    out = RT.TreeBatch(dev, q=q, k_new=k, v_new=v, row_offsets=dev32(case.off), row_pos=dev32(np.concatenate(case.row_pos)),
                       tree_mask=dev32(case.mask()), page_ids=dev32(ids), pos_base=dev32(case.pos_base), kv_len=dev32(case.kv_len),
                       max_rows=5, pools=pools).run(0.09)
    torch.cuda.synchronize()
    assert dev.read_status() == 0
    case.check(out, 0.09)
    slots = torch.tensor([(pages - 1) * P + P - 8 + i for i in range(8)], dtype=torch.int64, device="cuda:0")
    if fp8:
        scales[0][-1], scales[1][-1] = 0.5, 0.25
    RT.RowsCommit(dev, k_new=k, v_new=v, row_offsets=dev32([0, 8]), slot_map=slots, pools=pools).run()
    torch.cuda.synchronize()
    assert dev.read_status() == 0
    for b, new, sc in ((big[0], case.kn, 0.5), (big[1], case.vn, 0.25)):
        got = b[-1, :, P - 8:].transpose(0, 1)
        if fp8:
            want = O.e4m3_encode((bf16_bits_to_f64(new).astype(np.float32) / np.float32(sc)))
            assert np.array_equal(got.cpu().numpy(), want)
        else:
            assert np.array_equal(RT.bf16_bits(got.contiguous()), new)


def test_use_on_another_stream_than_the_tensors_were_made_on():
    case = TreeCase(61, Hq=8, Hkv=2, D=128, P=16, specs=[(1500, 9), (40, 3)])
    case.device()
    batch = case.batch()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = batch.run(0.09)                       # no stream named: the current one, which is `side`
        done = out.clone()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    case.check(done, 0.09)


@pytest.mark.parametrize("seed", range(16))
def test_random_shapes(seed):
    rng = np.random.default_rng(1000 + seed)
    Hkv = int(rng.choice([1, 2, 3]))
    G = int(rng.integers(1, 9))
    fp8 = bool(rng.integers(0, 2))
    D = 128 if fp8 else int(rng.choice([64, 128]))
    P = int(rng.choice([16, 32, 64, 256]))
    specs = [(int(rng.choice([0, 1, 5, int(rng.integers(1, 1500))])), int(rng.choice([0, 1, int(rng.integers(1, 70))]))) for _ in range(int(rng.integers(1, 9)))]
    if not any(n for _, n in specs):
        specs[0] = (specs[0][0], 7)
    case = TreeCase(seed, Hq=Hkv * G, Hkv=Hkv, D=D, P=P, specs=specs, kind=str(rng.choice(["tree", "chain", "star"])), fp8=fp8, theta=float(rng.choice([1e4, 5e5])))
    for s in case.sees:                             # any relation, not only a tree's
        if rng.integers(0, 2):
            s ^= rng.random(s.shape) < 0.2
    _run(case, 1.0 / np.sqrt(D), max_rows=min(32 * case.words, int(case.rows.max()) + int(rng.integers(0, 5))))


@pytest.mark.parametrize("Hq,Hkv,n", [(8, 1, 1024), (1, 1, 1024), (7, 1, 700)])
def test_as_many_rows_as_a_request_may_have(Hq, Hkv, n):
    _run(TreeCase(70 + n, Hq=Hq, Hkv=Hkv, D=64, P=16, specs=[(200, n), (37, 2)]), 0.125)


def test_a_batch_of_more_requests_than_the_cut_looks_at_in_one_go():
    rng = np.random.default_rng(71)
    specs = [(int(rng.integers(0, 90)), int(rng.integers(0, 4))) for _ in range(1500)]
    specs[1400] = (700, 90)
    _run(TreeCase(71, Hq=2, Hkv=1, D=64, P=16, specs=specs), 0.125)
