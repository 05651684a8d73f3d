"""Argument checks of the drafted-token calls: all of them happen on the host before any launch, so no GPU is needed."""
import ctypes as C

import numpy as np
import pytest

import paper_2512_16822_b200 as M
from paper_2512_16822_b200.build import build_library
from oracle import mepic_oracle as O

PTR = 1 << 20                       # never dereferenced: every call below is refused (or has nothing to do)


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()


CFG = M.Config(page_size=16, n_q_heads=8, n_kv_heads=2, head_dim=128, num_pages=10, max_position=100, rope_theta=1e4)


def _attn(**over):
    a = dict(q=PTR, k_new=PTR, v_new=PTR, row_offsets=PTR, row_pos=PTR, tree_mask=PTR, k_pool=PTR, v_pool=PTR, page_ids=PTR, pos_base=PTR,
             kv_len=PTR, rope_table=PTR, out=PTR, workspace=PTR, workspace_bytes=0, status=PTR, table_stride=4, batch=1, total_rows=3,
             max_rows=3, mask_words=1, sm_scale=1.0)
    cfg = over.pop("cfg", CFG)
    a.update(over)
    M.mepic_attn_tree(cfg, **a)


ATTN = [dict(batch=0), dict(table_stride=0), dict(total_rows=-1), dict(max_rows=-1), dict(max_rows=1025), dict(mask_words=0),
        dict(max_rows=33), dict(q=None), dict(out=None), dict(status=None), dict(workspace=None), dict(tree_mask=None), dict(k_pool=PTR + 2),
        dict(q=PTR + 8), dict(out=PTR + 4), dict(q_stride=8), dict(q_stride=1028), dict(kv_stride=250), dict(kv_stride=260)]


@pytest.mark.parametrize("over", ATTN, ids=[",".join(f"{k}={v}" for k, v in d.items()) for d in ATTN])
def test_attention_refuses(over):
    with pytest.raises(M.MepicError) as e:
        _attn(**over)
    assert e.value.code == M.MEPIC_E_INVAL and "attn_tree" in str(e.value)


def test_attention_over_8_bit_pages_refuses():
    a = dict(q=PTR, k_new=PTR, v_new=PTR, row_offsets=PTR, row_pos=PTR, tree_mask=PTR, k_pool=PTR, v_pool=PTR, page_ids=PTR, pos_base=PTR,
             kv_len=PTR, rope_table=PTR, out=PTR, workspace=PTR, workspace_bytes=0, status=PTR, table_stride=4, batch=1, total_rows=3,
             max_rows=3, mask_words=1, sm_scale=1.0)
    small = M.Config(16, 8, 2, 64, 10, 100, 1e4)
    for cfg, ks, vs in ((small, PTR, PTR), (CFG, None, PTR), (CFG, PTR, None)):
        with pytest.raises(M.MepicError) as e:
            M.mepic_attn_tree_fp8(cfg, k_scales=ks, v_scales=vs, **a)
        assert e.value.code == M.MEPIC_E_INVAL


def test_attention_without_rows_needs_no_buffers():
    _attn(total_rows=0, q=None, out=None, workspace=None)
    _attn(max_rows=0, q=None, out=None, workspace=None)


def test_workspace_of_bad_arguments():
    for bad in (-1, 1025):
        with pytest.raises(M.MepicError):
            M.mepic_attn_tree_workspace(CFG, bad)
    with pytest.raises(M.MepicError):
        M.mepic_attn_tree_workspace(M.Config(15, 8, 2, 128, 10, 100, 1e4), 4)


@pytest.mark.parametrize("over", [dict(batch=0), dict(table_stride=0), dict(total_rows=-2), dict(mask_words=0), dict(mask_words=33),
                                  dict(parent=None), dict(row_pos=None), dict(status=None)])
def test_layout_refuses(over):
    a = dict(parent=PTR, row_offsets=PTR, kv_len=PTR, pos_base=PTR, row_pos=PTR, tree_mask=PTR, status=PTR, table_stride=4, batch=1,
             total_rows=3, mask_words=1)
    a.update(over)
    with pytest.raises(M.MepicError) as e:
        M.mepic_tree_layout(CFG, **a)
    assert e.value.code == M.MEPIC_E_INVAL


@pytest.mark.parametrize("over", [dict(batch=0), dict(total_rows=-2), dict(max_accept=0), dict(root=None), dict(draft=None), dict(next_token=None)])
def test_accept_refuses(over):
    a = dict(parent=PTR, row_offsets=PTR, draft=PTR, target=PTR, root=PTR, n_accept=PTR, accept_rows=PTR, next_token=PTR, status=PTR,
             batch=1, total_rows=3, max_accept=4)
    a.update(over)
    with pytest.raises(M.MepicError) as e:
        M.mepic_tree_accept(**a)
    assert e.value.code == M.MEPIC_E_INVAL


@pytest.mark.parametrize("over", [dict(batch=0), dict(batch=8193), dict(table_stride=0), dict(max_rows=-1), dict(n_reserve=-1), dict(kv_len=None),
                                  dict(reserve=None), dict(reserve_used_out=None), dict(kv_len_out=PTR), dict(reserve_used_out=PTR + 128),
                                  dict(slot_map=PTR + 4)])
def test_tables_refuse(over):
    a = dict(kv_len=PTR, n_new=PTR + 64, page_ids=PTR, pos_base=PTR, reserve=PTR, reserve_used=PTR + 128, row_offsets=PTR, kv_len_out=PTR + 256,
             reserve_used_out=PTR + 512, status=PTR, table_stride=4, batch=1, max_rows=3, n_reserve=2)
    a.update(over)
    with pytest.raises(M.MepicError) as e:
        M.mepic_step_tables(CFG, **a)
    assert e.value.code == M.MEPIC_E_INVAL


@pytest.mark.parametrize("over", [dict(batch=0), dict(max_rows=-1), dict(n_sources=-1), dict(k_new=None), dict(slot_map=None), dict(v_pool=None),
                                  dict(k_new=PTR + 2), dict(slot_map=PTR + 4), dict(kv_stride=8), dict(kv_stride=257), dict(src_rows=PTR, src_stride=0)])
def test_commit_refuses(over):
    a = dict(k_new=PTR, v_new=PTR, row_offsets=PTR, slot_map=PTR, k_pool=PTR, v_pool=PTR, status=PTR, batch=1, max_rows=3, n_sources=3)
    a.update(over)
    with pytest.raises(M.MepicError) as e:
        M.mepic_rows_commit(CFG, **a)
    assert e.value.code == M.MEPIC_E_INVAL


def test_commit_into_8_bit_pages_refuses():
    a = dict(k_new=PTR, v_new=PTR, row_offsets=PTR, slot_map=PTR, k_pool=PTR, v_pool=PTR, status=PTR, batch=1, max_rows=3, n_sources=3)
    for cfg, ks, vs in ((M.Config(16, 8, 2, 64, 10, 100, 1e4), PTR, PTR), (CFG, None, PTR), (CFG, PTR, None)):
        with pytest.raises(M.MepicError) as e:
            M.mepic_rows_commit_fp8(cfg, k_scales=ks, v_scales=vs, **a)
        assert e.value.code == M.MEPIC_E_INVAL


# ------------------------------------------------------------------------------------ the oracle, pinned by hand
def test_oracle_layout_by_hand():
    #        0
    #      /   \
    #     1     2      3 (root)
    #     |
    #     4
    pos, sees = O.tree_layout([-1, 0, 0, -1, 1], 10)
    assert pos.tolist() == [10, 11, 11, 10, 12]
    assert sees.astype(int).tolist() == [[1, 0, 0, 0, 0], [1, 1, 0, 0, 0], [1, 0, 1, 0, 0], [0, 0, 0, 1, 0], [1, 1, 0, 0, 1]]
    assert O.pack_mask(sees, 1)[:, 0].tolist() == [1, 3, 5, 8, 19]
    assert O.pack_mask(np.eye(40, dtype=bool), 2)[31].tolist() == [-2 ** 31, 0] and O.pack_mask(np.eye(40, dtype=bool), 2)[33].tolist() == [0, 2]


def test_oracle_accept_by_hand():
    parent, draft, target = [-1, 0, 0, -1, 1, 1], [5, 6, 6, 5, 7, 8], [6, 8, 9, 1, 2, 3]
    assert O.tree_accept(parent, draft, target, 5, 8) == ([0, 1, 5], 3)      # of two matching roots and children the first
    assert O.tree_accept(parent, draft, target, 5, 2) == ([0, 1], 8)
    assert O.tree_accept(parent, draft, target, 4, 8) == ([], 4)


def test_oracle_attention_reduces_to_decode():
    rng = np.random.default_rng(0)
    from mepic_inputs import f32_to_bf16_bits
    bits = lambda s: f32_to_bf16_bits(rng.standard_normal(s).astype(np.float32))
    kp, vp = bits((5, 2, 16, 64)), bits((5, 2, 16, 64))
    q, k, v = bits((1, 4, 64)), bits((1, 2, 64)), bits((1, 2, 64))
    out, _ = O.tree_attention_one(q, k, v, [37], np.ones((1, 1), bool), kp, vp, [3, 1, 4], [0, 16, 32], 37, 0.125, 1e4)
    kp[4, :, 5], vp[4, :, 5] = k[0], v[0]
    want = O.decode_attention_one(q[0], kp, vp, [3, 1, 4], [0, 16, 32], 38, 37, 0.125, 1e4)
    assert np.abs(out[0] - want).max() < 1e-12


def test_oracle_tables_by_hand():
    ids = np.array([[9, -1, -1], [4, 5, -1], [-1, -1, -1]])
    base = np.array([[100, 0, 0], [0, 16, 0], [0, 0, 0]])
    r = O.step_tables([15, 32, 0], [3, 1, 0], ids, base, [7, 2, 3], 1, 16, 6)
    assert r["page_ids"].tolist() == [[9, 2, -1], [4, 5, 3], [-1, -1, -1]]
    assert r["pos_base"].tolist() == [[100, 116, 0], [0, 16, 32], [0, 0, 0]]
    assert r["row_slot"].tolist() == [15, 16, 17, 32, -1, -1] and r["slot_map"].tolist() == [9 * 16 + 15, 32, 33, 48, -1, -1]
    assert r["kv_len"].tolist() == [18, 33, 0] and r["q_pos"].tolist() == [117, 32, -1] and r["reserve_used"] == 3
    r = O.step_tables([15, 32, 0], [3, 1, 1], ids, base, [7, 2, 3], 1, 16, 6)
    assert r["rejected"] and r["kv_len"].tolist() == [15, 32, 0] and r["reserve_used"] == 1
