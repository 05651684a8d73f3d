"""What the objects of a drafted-token step check before they bind a tensor: no GPU is needed to be refused."""
from types import SimpleNamespace

import pytest
import torch

import paper_2512_16822_b200 as M
from paper_2512_16822_b200 import runtime as RT

CPU = torch.device("cpu")
CFG = M.Config(page_size=16, n_q_heads=8, n_kv_heads=2, head_dim=128, num_pages=10, max_position=100, rope_theta=1e4)
ROWS = 5


def _dev(cfg=CFG):
    pool = torch.zeros((cfg.num_pages, cfg.n_kv_heads, cfg.page_size, cfg.head_dim), dtype=torch.bfloat16)
    return SimpleNamespace(cfg=cfg, device=CPU, k_pool=pool, v_pool=pool.clone(), rope=None, status=torch.zeros(1, dtype=torch.int32))


def _rows(heads, rows=ROWS):
    return torch.zeros((rows, heads, 128), dtype=torch.bfloat16)


def _broadcast(heads):
    return torch.zeros((1, heads, 128), dtype=torch.bfloat16).expand(ROWS, heads, 128)


def _overlapping(heads):
    return torch.zeros(64 * ROWS + heads * 128, dtype=torch.bfloat16).as_strided((ROWS, heads, 128), (64, 128, 1))


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def _tree(dev, **over):
    a = dict(q=_rows(8), k_new=_rows(2), v_new=_rows(2), row_offsets=_i32(2), row_pos=_i32(ROWS), tree_mask=_i32(ROWS, 1), page_ids=_i32(1, 4),
             pos_base=_i32(1, 4), kv_len=_i32(1), max_rows=ROWS)
    a.update(over)
    return RT.TreeBatch(dev, **a)


def _commit(dev, **over):
    a = dict(k_new=_rows(2), v_new=_rows(2), row_offsets=_i32(2), slot_map=torch.zeros(ROWS, dtype=torch.int64))
    a.update(over)
    return RT.RowsCommit(dev, **a)


@pytest.mark.parametrize("make", [_broadcast, _overlapping])
def test_rows_that_share_memory_are_refused(make):
    # a row stride of 0 is the call's word for "packed": a broadcast row bound as it is would be read as ROWS rows
    with pytest.raises(ValueError, match="q: .*stride"):
        _tree(_dev(), q=make(8))
    for name in ("k_new", "v_new"):
        with pytest.raises(ValueError, match=name + ": .*stride"):
            _tree(_dev(), **{name: make(2)})
        with pytest.raises(ValueError, match=name + ": .*stride"):
            _commit(_dev(), **{name: make(2)})
    both = make(2)
    with pytest.raises(ValueError, match="k_new: .*stride"):
        _commit(_dev(), k_new=both, v_new=both)


def test_row_strides_of_rows_that_lie_apart_or_alone():
    fused = torch.zeros((ROWS, 12 * 128), dtype=torch.bfloat16)
    q = fused[:, :8 * 128].unflatten(1, (8, 128))
    assert RT._row_stride(q, "q", 8, 128, CPU) == 12 * 128
    assert RT._row_stride(_rows(2), "k", 2, 128, CPU) == 2 * 128
    assert RT._row_stride(_broadcast(2)[:1], "k", 2, 128, CPU) == 2 * 128        # one row has no stride to speak of
    assert RT._row_stride(_rows(2, 0), "k", 2, 128, CPU) == 2 * 128


class _Elsewhere:
    """Stands in for a tensor on a GPU this machine does not have."""

    def __init__(self, like, device):
        self._like, self.device, self.dtype, self.shape = like, torch.device(device), like.dtype, like.shape

    def __getattr__(self, name):
        return getattr(self._like, name)


def test_tensors_of_another_gpu_are_refused():
    zero = torch.device("cuda:0")
    assert RT._row_stride(_Elsewhere(_rows(2), "cuda:0"), "k", 2, 128, zero) == 2 * 128
    for device in ("cuda:1", "cpu"):
        with pytest.raises(ValueError, match="on cuda:0"):
            RT._row_stride(_Elsewhere(_rows(2), device), "k", 2, 128, zero)
        with pytest.raises(ValueError, match="on cuda:0"):
            RT._expect(_Elsewhere(_i32(3), device), "kv_len", torch.int32, (3,), zero)


def test_a_device_without_an_index_is_the_current_one(monkeypatch):
    # ... at the time it is made: what is checked against it later may not lie on another GPU
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    assert RT._cuda_device("cuda") == torch.device("cuda:1")
    assert RT._cuda_device("cuda:0") == torch.device("cuda:0")
    assert RT._cuda_device(torch.device("cuda:2")) == torch.device("cuda:2")


def _pools(dev, num_pages=None, device=None):
    n = dev.cfg.num_pages if num_pages is None else num_pages
    codes, scales = torch.zeros((n, 2, 16, 128), dtype=torch.uint8), torch.ones((n, 2), dtype=torch.float32)
    if device is not None:
        codes, scales = _Elsewhere(codes, device), _Elsewhere(scales, device)
    return SimpleNamespace(dev=dev, k_codes=codes, v_codes=codes, k_scales=scales, v_scales=scales)


def test_pools_that_are_not_the_devices_are_refused():
    # a page id that is valid for the device's configuration must be valid for the pools it is looked up in
    dev = _dev()
    for build in (_tree, _commit):
        for pools in (_pools(dev, num_pages=9), _pools(dev, device="cuda:1")):
            with pytest.raises(ValueError, match="codes"):
                build(dev, pools=pools)
        short = _pools(dev)
        short.v_scales = short.v_scales[:9]
        with pytest.raises(ValueError, match="scales"):
            build(dev, pools=short)
        bare = _dev()
        bare.k_pool = bare.v_pool = None                             # a device whose only pools are 8-bit, and none are given
        with pytest.raises(ValueError, match="bf16 pools"):
            build(bare)
        small = _dev()
        small.v_pool = small.v_pool[:9]
        with pytest.raises(ValueError, match="pool"):
            build(small)


def test_counts_and_strides_that_32_bits_do_not_hold_are_refused():
    # (ctypes keeps the low 32 bits of a larger number: 2^32 + 3 rows were 3, a row stride of 2^32 was 0, "packed")
    ptr, big = 1 << 20, 2 ** 32
    calls = [
        lambda: M.mepic_step_tables(CFG, kv_len=ptr, n_new=ptr + 64, page_ids=ptr, pos_base=ptr, reserve=ptr, reserve_used=ptr + 128, row_offsets=ptr,
                                    kv_len_out=ptr + 256, reserve_used_out=ptr + 512, status=ptr, table_stride=4, batch=1, max_rows=big + 3, n_reserve=2),
        lambda: M.mepic_tree_layout(CFG, parent=ptr, row_offsets=ptr, kv_len=ptr, pos_base=ptr, row_pos=ptr, tree_mask=ptr, status=ptr, table_stride=4,
                                    batch=1, total_rows=big, mask_words=1),
        lambda: M.mepic_tree_accept(parent=ptr, row_offsets=ptr, draft=ptr, target=ptr, root=ptr, n_accept=ptr, accept_rows=ptr, next_token=ptr, status=ptr,
                                    batch=1, total_rows=3, max_accept=2 ** 31),
        lambda: M.mepic_rows_commit(CFG, k_new=ptr, v_new=ptr, row_offsets=ptr, slot_map=ptr, k_pool=ptr, v_pool=ptr, status=ptr, batch=1, max_rows=0,
                                    n_sources=3, kv_stride=big),
        lambda: M.mepic_attn_tree(CFG, q=ptr, k_new=ptr, v_new=ptr, row_offsets=ptr, row_pos=ptr, tree_mask=ptr, k_pool=ptr, v_pool=ptr, page_ids=ptr,
                                  pos_base=ptr, kv_len=ptr, rope_table=ptr, out=ptr, workspace=ptr, workspace_bytes=0, status=ptr, table_stride=4,
                                  batch=1, total_rows=0, max_rows=0, mask_words=1, sm_scale=1.0, q_stride=big),
    ]
    for call in calls:
        with pytest.raises(M.MepicError, match="32 bits") as e:
            call()
        assert e.value.code == M.MEPIC_E_INVAL
