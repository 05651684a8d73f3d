"""The integer calls of a step and the commits at the largest row counts their arguments can name: counters that step past an
int32 must not come round to the front of the arrays."""
import numpy as np
import pytest
import torch

import paper_2512_16822_b200 as M
from paper_2512_16822_b200.build import build_library
from tree_helpers import dev32

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 1
GUARD = 4096


@pytest.fixture(autouse=True)
def _built():
    build_library()
    yield
    torch.cuda.empty_cache()


def guarded(n, fill=77):
    """int32 [n] with GUARD elements before and behind it that nobody may write; -> (the array, a check of the guards)."""
    buf = torch.empty(n + 2 * GUARD, dtype=torch.int32, device="cuda:0")
    buf[:GUARD], buf[GUARD + n:] = fill, fill
    return buf[GUARD:GUARD + n], lambda: bool((buf[:GUARD] == fill).all() and (buf[GUARD + n:] == fill).all())


def all_are(t, value, step=1 << 28):
    return all(bool((t[i:i + step] == value).all()) for i in range(0, t.numel(), step))


def test_tables_with_the_largest_row_array():
    cfg = M.Config(16, 1, 1, 64, 100, 64, 1e4)
    slots, whole = guarded(MOST)
    status, ids, base = dev32([0]), dev32([[4, 0, 0]]), dev32([[0, 0, 0]])
    kv, new, off, kv_out, used, used_out = dev32([10]), dev32([30]), dev32([0, 0]), dev32([0]), dev32([0]), dev32([0])
    M.mepic_step_tables(cfg, kv_len=kv, n_new=new, page_ids=ids, pos_base=base, reserve=dev32([7, 9]), reserve_used=used, row_offsets=off,
                        kv_len_out=kv_out, reserve_used_out=used_out, status=status, table_stride=3, batch=1, max_rows=MOST, n_reserve=2,
                        row_slot=slots, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert status.item() == 0 and whole()
    assert slots[:30].tolist() == list(range(10, 40)) and all_are(slots[30:], -1) and ids.tolist() == [[4, 7, 9]]


def test_acceptance_with_the_longest_path_array():
    rows, whole = guarded(MOST)
    status, n, nxt = dev32([0]), dev32([0]), dev32([0])
    M.mepic_tree_accept(parent=dev32([-1, 0]), row_offsets=dev32([0, 2]), draft=dev32([5, 6]), target=dev32([6, 8]), root=dev32([5]), n_accept=n,
                        accept_rows=rows, next_token=nxt, status=status, batch=1, total_rows=2, max_accept=MOST, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert status.item() == 0 and whole() and n.item() == 2 and nxt.item() == 8
    assert rows[:2].tolist() == [0, 1] and all_are(rows[2:], -1)


def test_layout_of_the_most_rows_an_offset_can_name():
    # one request owns 2^31 - 1 rows: those the mask has no room for are reported and get the context's next position
    cfg = M.Config(16, 1, 1, 64, 100, 64, 1e4)
    parent = torch.zeros(MOST, dtype=torch.int32, device="cuda:0")
    parent[0] = -1
    pos, whole_pos = guarded(MOST)
    mask, whole_mask = guarded(MOST)
    status = dev32([0])
    M.mepic_tree_layout(cfg, parent=parent, row_offsets=dev32([0, MOST]), kv_len=dev32([3]), pos_base=dev32([[40]]), row_pos=pos, tree_mask=mask,
                        status=status, table_stride=1, batch=1, total_rows=MOST, mask_words=1, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert status.item() == M.MEPIC_DEV_BAD_TREE and whole_pos() and whole_mask()
    assert pos[:3].tolist() == [43, 44, 44] and all_are(pos[32:], 43)
    assert mask[:3].tolist() == [1, 3, 5] and all_are(mask[32:], 0)


@pytest.mark.parametrize("fp8", [False, True])
def test_commit_with_the_longest_slot_map(fp8):
    cfg = M.Config(16, 2, 2, 128, 6, 64, 1e4)
    slots = torch.empty(MOST, dtype=torch.int64, device="cuda:0")
    slots[:3] = torch.tensor([33, 34, 35], device="cuda:0")
    rows = torch.full((3, 2, 128), 2.0, dtype=torch.bfloat16, device="cuda:0")
    pools = [torch.zeros((6, 2, 16, 128), dtype=torch.uint8 if fp8 else torch.bfloat16, device="cuda:0") for _ in range(2)]
    status = dev32([0])
    a = dict(k_new=rows, v_new=rows, row_offsets=dev32([0, 3]), slot_map=slots, k_pool=pools[0], v_pool=pools[1], status=status, batch=1,
             max_rows=MOST, n_sources=3, stream=torch.cuda.current_stream())
    if fp8:
        scales = [torch.ones((6, 2), dtype=torch.float32, device="cuda:0") for _ in range(2)]
        M.mepic_rows_commit_fp8(cfg, k_scales=scales[0], v_scales=scales[1], **a)
    else:
        M.mepic_rows_commit(cfg, **a)
    torch.cuda.synchronize()
    assert status.item() == 0
    for p in pools:
        got = p.view(torch.float8_e4m3fn).float() if fp8 else p.float()
        want = torch.zeros((6, 2, 16, 128), device="cuda:0")
        want[2, :, 1:4] = 2.0
        assert torch.equal(got, want)
