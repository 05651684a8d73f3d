"""Which rows the commits of a step take, and steps without any."""
import numpy as np
import pytest
import torch

import paper_2512_16822_b200 as M
from paper_2512_16822_b200 import runtime as RT
from paper_2512_16822_b200.build import build_library
from mepic_inputs import f32_to_bf16_bits
from oracle import mepic_oracle as O
from tree_helpers import dev32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"


def _empty_pools(P, num_pages, fp8, Hkv=2, D=128):
    dev = RT.Device(M.Config(P, Hkv, Hkv, D, num_pages, 4 * P, 1e4))
    dev.k_pool.zero_(), dev.v_pool.zero_()
    pools = RT.Fp8Pools(dev) if fp8 else None
    return dev, pools


def _written(dev, pools, w):
    """[page, slot]: whether anything of the zeroed pool w (0: K, 1: V) was written."""
    pool = ((pools.k_codes, pools.v_codes) if pools else (dev.k_pool, dev.v_pool))[w]
    return pool.float().abs().amax(dim=(1, 3)).bool().nonzero().tolist()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("first,n", [(1, 1), (5, 4), (19, 30)])
def test_rows_before_the_first_request_are_not_committed(fp8, gather, first, n):
    # row_offsets start at `first`: the rows before it belong to nobody, whatever slots stand beside them (of the same page too)
    P = 16
    dev, pools = _empty_pools(P, 12, fp8)
    total = first + n
    rows = torch.ones((total, 2, 128), dtype=torch.bfloat16, device=DEV)
    rows[:first] = 100.0                                                 # would set a page's scale
    slots = torch.arange(3 * P, 3 * P + total, dtype=torch.int64, device=DEV)
    src = dev32(np.arange(first, total)[None]) if gather else None
    RT.RowsCommit(dev, k_new=rows, v_new=rows, row_offsets=dev32([first, total]), slot_map=slots, src_rows=src, pools=pools).run()
    torch.cuda.synchronize()
    assert dev.read_status() == 0
    want = [[(3 * P + r) // P, (3 * P + r) % P] for r in range(first, total)]
    assert _written(dev, pools, 0) == want and _written(dev, pools, 1) == want
    if fp8:
        for s in (pools.k_scales, pools.v_scales):
            for page in {p for p, _ in want}:
                started = [page, 0] in want
                # a run that writes slot 0 sets the scale from its own rows (1 / 448 of their 1.0), any other leaves it
                assert (s[page] == (float(np.float32(1) / np.float32(448)) if started else 1.0)).all()


@pytest.mark.parametrize("P", [16, 64])
def test_a_skipped_row_does_not_start_a_page(P):
    # the run's row for in-page slot 0 has no source: the run does not write slot 0, so it appends under the scale that stands
    dev, pools = _empty_pools(P, 4, True)
    for s in (pools.k_scales, pools.v_scales):
        s.fill_(0.5)
    rows = torch.full((4, 2, 128), 3.0, dtype=torch.bfloat16, device=DEV)
    slots = torch.tensor([P, P + 1, P + 2, 2 * P, 2 * P + 1, 3 * P, 3 * P + 1], dtype=torch.int64, device=DEV)
    src = dev32([[-1, 0, 9, 2, 1, -1, -1]])                              # page 1 appended to, page 2 started, page 3 left alone
    RT.RowsCommit(dev, k_new=rows, v_new=rows, row_offsets=dev32([0, 7]), slot_map=slots, src_rows=src, pools=pools).run()
    torch.cuda.synchronize()
    assert dev.read_status() == M.MEPIC_DEV_BAD_SLOT
    for w, (codes, scales) in enumerate(((pools.k_codes, pools.k_scales), (pools.v_codes, pools.v_scales))):
        assert _written(dev, pools, w) == [[1, 1], [2, 0], [2, 1]]
        assert (scales[[0, 1, 3]] == 0.5).all() and (scales[2] == float(np.float32(3) / np.float32(448))).all()
        value = codes.view(torch.float8_e4m3fn).float()
        assert (value[1, :, 1] == 6.0).all() and (value[2, :, :2] == 448.0).all()


@pytest.mark.parametrize("fp8", [False, True])
def test_a_step_in_which_nobody_drafts(fp8):
    # no rows at all in the row arrays: every call of the step is a call without work, and the lengths stay
    B, P = 3, 16
    dev, pools = _empty_pools(P, 6, fp8)
    none = dev32([])
    off, kv, ids, base = dev32([0] * (B + 1)), dev32([5, 0, 17]), dev32([[0, 1]] * B), dev32([[0, P]] * B)
    q, k = torch.empty((0, 2, 128), dtype=torch.bfloat16, device=DEV), torch.empty((0, 2, 128), dtype=torch.bfloat16, device=DEV)
    lay = RT.TreeLayout(dev, parent=none, row_offsets=off, kv_len=kv, pos_base=base, mask_words=1)
    att = RT.TreeBatch(dev, q=q, k_new=k, v_new=k, row_offsets=off, row_pos=lay.row_pos, tree_mask=lay.tree_mask, page_ids=ids, pos_base=base,
                       kv_len=kv, max_rows=4, pools=pools)
    acc = RT.TreeAccept(dev, parent=none, row_offsets=off, draft=none, target=none, root=dev32([7, 8, 9]), max_accept=4)
    tab = RT.StepTables(dev, kv_len=kv, n_new=acc.n_accept, page_ids=ids, pos_base=base, reserve=dev32([2]), reserve_used=dev32([0]), max_rows=4 * B)
    com = RT.RowsCommit(dev, k_new=k, v_new=k, row_offsets=tab.row_offsets, slot_map=tab.slot_map, src_rows=acc.accept_rows, pools=pools)
    for call in (lambda: lay.run(), lambda: att.run(0.1), lambda: acc.run(), lambda: tab.run(), lambda: com.run()):
        call()
    torch.cuda.synchronize()
    assert dev.read_status() == 0
    assert acc.n_accept.tolist() == [0] * B and acc.next_token.tolist() == [7, 8, 9] and (acc.accept_rows == -1).all()
    assert tab.kv_len_out.tolist() == [5, 0, 17] and tab.row_offsets.tolist() == [0] * (B + 1) and tab.reserve_used_out.item() == 0
    assert _written(dev, pools, 0) == [] and _written(dev, pools, 1) == []
    # rows that are asked for all the same have no source
    RT.RowsCommit(dev, k_new=k, v_new=k, row_offsets=dev32([0, 2]), slot_map=torch.tensor([3, 4], device=DEV), pools=pools).run()
    torch.cuda.synchronize()
    assert dev.read_status() == M.MEPIC_DEV_BAD_SLOT and _written(dev, pools, 0) == []


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("P,Hkv", [(128, 3), (512, 1)])
def test_commit_into_long_pages_in_any_order_of_slots(fp8, P, Hkv):
    # runs of hundreds of rows, whole pages among them, whose slots do not ascend; gathered from twice as many sources
    rng, D, pages = np.random.default_rng(P), 128, 6
    bits = lambda shape: f32_to_bf16_bits((rng.standard_normal(shape) * 2).astype(np.float32))
    kp, vp = bits((pages, Hkv, P, D)), bits((pages, Hkv, P, D))
    dev = RT.Device(M.Config(P, Hkv, Hkv, D, pages, P, 1e4), kp, vp)
    pools = RT.Fp8Pools(dev) if fp8 else None
    parts = [(4, rng.permutation(P)), (1, 1 + rng.permutation(P - 1)[:P // 2 + 5]), (5, rng.permutation(P // 2)), (0, np.array([P - 1]))]
    off = np.array([0, P, P + len(parts[1][1]), P + len(parts[1][1]) + len(parts[2][1]) + 1])       # the third request takes two pages
    slots = np.concatenate([page * P + t for page, t in parts])
    total = len(slots)
    k, v = bits((2 * total, Hkv, D)), bits((2 * total, Hkv, D))
    src = np.full((3, int(np.diff(off).max())), -1)
    for b in range(3):
        src[b, :off[b + 1] - off[b]] = rng.choice(np.arange(2 * total), size=off[b + 1] - off[b], replace=False)
    flat = np.concatenate([src[b, :off[b + 1] - off[b]] for b in range(3)])
    RT.RowsCommit(dev, k_new=RT.bf16_tensor(k, DEV), v_new=RT.bf16_tensor(v, DEV), row_offsets=dev32(off),
                  slot_map=torch.from_numpy(slots.astype(np.int64)).to(DEV), src_rows=dev32(src), pools=pools).run()
    torch.cuda.synchronize()
    assert dev.read_status() == 0
    if fp8:
        (kc, ks), (vc, vs) = O.quantize_pages(kp), O.quantize_pages(vp)
    at = 0
    for page, t in parts:
        rows = flat[at:at + len(t)]
        at += len(t)
        if fp8:
            O.commit_rows_fp8(kc, ks, vc, vs, [page], list(t), k[rows], v[rows])
        else:
            O.commit_rows(kp, vp, [page], list(t), k[rows], v[rows])
    if fp8:
        assert np.array_equal(pools.k_scales.cpu().numpy(), ks) and np.array_equal(pools.v_scales.cpu().numpy(), vs)
        assert np.array_equal(pools.k_codes.cpu().numpy(), kc) and np.array_equal(pools.v_codes.cpu().numpy(), vc)
    else:
        assert np.array_equal(RT.bf16_bits(dev.k_pool), kp) and np.array_equal(RT.bf16_bits(dev.v_pool), vp)
