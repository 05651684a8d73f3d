"""Argument checks of the beam calls and of their objects: all of them happen on the host before any launch, so no GPU is needed."""
from types import SimpleNamespace

import pytest
import torch

import paper_2512_16822_b200 as M
from paper_2512_16822_b200 import runtime as RT
from paper_2512_16822_b200.build import build_library

PTR = 1 << 20                       # never dereferenced: every call below is refused (or has nothing to do)
CPU = torch.device("cpu")
CFG = M.Config(page_size=16, n_q_heads=8, n_kv_heads=2, head_dim=128, num_pages=10, max_position=100, rope_theta=1e4)
SMALL = M.Config(16, 8, 2, 64, 10, 100, 1e4)
BIG = 1 << 40


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()


def _ids(cases):
    return [",".join(f"{k}={v}" for k, v in d.items()) for d in cases]


def _refused(call, what):
    with pytest.raises(M.MepicError) as e:
        call()
    assert e.value.code == M.MEPIC_E_INVAL and what in str(e.value), str(e.value)


SELECT = dict(logits=PTR, score=PTR, parent=2 * PTR, token=2 * PTR, score_out=2 * PTR, done_out=2 * PTR, n_new=2 * PTR, workspace=PTR, workspace_bytes=BIG,
              status=PTR, logits_type=0, groups=2, width=4, n_select=4, vocab=100, eos_token=1, pad_token=0)
BAD_SELECT = [dict(groups=0), dict(width=0), dict(width=33), dict(n_select=0), dict(n_select=65), dict(vocab=0), dict(vocab=(1 << 24) + 1),
              dict(groups=65536, width=1), dict(logits_type=3), dict(logits_type=-1), dict(logits=None), dict(score=None), dict(parent=None), dict(token=None),
              dict(score_out=None), dict(done_out=None), dict(n_new=None), dict(workspace=None), dict(status=None), dict(logits_stride=99),
              dict(logits_stride=-1), dict(eos_token=100), dict(eos_token=-2), dict(pad_token=-1), dict(pad_token=100), dict(logits=PTR + 1),
              dict(logits=PTR + 2, logits_type=2), dict(workspace=PTR + 8), dict(workspace_bytes=15), dict(score_out=PTR), dict(done=2 * PTR)]


@pytest.mark.parametrize("over", BAD_SELECT, ids=_ids(BAD_SELECT))
def test_select_refuses(over):
    _refused(lambda: M.mepic_beam_select(**{**SELECT, **over}), "beam_select")


FORK = dict(parent=PTR, kv_len=PTR, page_ids=PTR, pos_base=PTR, owned=PTR, reserve=PTR, reserve_used=PTR, page_ids_out=2 * PTR, pos_base_out=2 * PTR,
            kv_len_out=2 * PTR, copy_src=2 * PTR, copy_dst=2 * PTR, copy_slots=2 * PTR, n_copies=2 * PTR, reserve_used_out=2 * PTR, workspace=PTR,
            workspace_bytes=BIG, status=PTR, table_stride=8, groups=2, width_in=4, width_out=4, n_reserve=5)
BAD_FORK = [dict(groups=0), dict(groups=8193), dict(width_in=0), dict(width_in=33), dict(width_out=0), dict(width_out=33), dict(table_stride=0),
            dict(table_stride=(1 << 24) + 1), dict(groups=8192, table_stride=1 << 20), dict(n_reserve=-1)] + \
           [{k: None} for k, v in FORK.items() if v in (PTR, 2 * PTR)] + \
           [dict(page_ids_out=PTR), dict(pos_base_out=PTR), dict(kv_len_out=PTR), dict(reserve_used_out=PTR), dict(workspace=PTR + 4), dict(workspace_bytes=100)]


@pytest.mark.parametrize("over", BAD_FORK, ids=_ids(BAD_FORK))
def test_fork_refuses(over):
    _refused(lambda: M.mepic_beam_fork(CFG, **{**FORK, **over}), "beam_fork")


COPY = dict(src=PTR, dst=PTR, slots=PTR, n_copies=PTR, k_pool=PTR, v_pool=PTR, status=PTR, max_copies=3)
BAD_COPY = [dict(max_copies=-1), dict(src=None), dict(dst=None), dict(k_pool=None), dict(v_pool=None), dict(status=None), dict(k_pool=PTR + 8), dict(v_pool=PTR + 2)]


@pytest.mark.parametrize("over", BAD_COPY, ids=_ids(BAD_COPY))
def test_copy_refuses(over):
    _refused(lambda: M.mepic_pages_copy(CFG, **{**COPY, **over}), "pages_copy")
    _refused(lambda: M.mepic_pages_copy_fp8(CFG, k_scales=PTR, v_scales=PTR, **{**COPY, **over}), "pages_copy_fp8")


def test_copy_in_8_bit_pools_refuses():
    for cfg, ks, vs in ((SMALL, PTR, PTR), (CFG, None, PTR), (CFG, PTR, None)):
        _refused(lambda: M.mepic_pages_copy_fp8(cfg, k_scales=ks, v_scales=vs, **COPY), "pages_copy_fp8")


def test_no_copies_need_no_buffers():
    M.mepic_pages_copy(CFG, src=None, dst=None, k_pool=None, v_pool=None, status=None, max_copies=0)


PLAN = dict(page_ids=PTR, pos_base=PTR, kv_len=PTR, plan=PTR, plan_bytes=BIG, status=PTR, table_stride=8, groups=2, width=4)
BAD_PLAN = [dict(groups=0), dict(width=0), dict(width=33), dict(table_stride=0), dict(table_stride=1 << 30), dict(groups=1 << 20, width=32), dict(page_ids=None),
            dict(pos_base=None), dict(kv_len=None), dict(plan=None), dict(status=None), dict(plan=PTR + 8), dict(plan_bytes=64)]


@pytest.mark.parametrize("over", BAD_PLAN, ids=_ids(BAD_PLAN))
def test_plan_refuses(over):
    _refused(lambda: M.mepic_beam_plan(CFG, **{**PLAN, **over}), "beam_plan")


ATTN = dict(q=PTR, q_pos=PTR, plan=PTR, k_pool=PTR, v_pool=PTR, rope_table=PTR, out=PTR, workspace=PTR, workspace_bytes=0, status=PTR, table_stride=8,
            groups=2, width=4, sm_scale=1.0)
BAD_ATTN = [dict(groups=0), dict(width=0), dict(width=33), dict(table_stride=0)] + [{k: None} for k, v in ATTN.items() if v == PTR] + \
           [{k: PTR + 8} for k in ("q", "plan", "k_pool", "v_pool", "rope_table", "out", "workspace")] + [dict(q_stride=1016), dict(q_stride=1028), dict(q_stride=-8)]


@pytest.mark.parametrize("over", BAD_ATTN, ids=_ids(BAD_ATTN))
def test_attention_refuses(over):
    _refused(lambda: M.mepic_attn_beam(CFG, **{**ATTN, **over}), "attn_beam")
    _refused(lambda: M.mepic_attn_beam_fp8(CFG, k_scales=PTR, v_scales=PTR, **{**ATTN, **over}), "attn_beam_fp8")


def test_attention_over_8_bit_pages_refuses():
    for cfg, ks, vs in ((SMALL, PTR, PTR), (CFG, None, PTR), (CFG, PTR, None)):
        _refused(lambda: M.mepic_attn_beam_fp8(cfg, k_scales=ks, v_scales=vs, **ATTN), "attn_beam_fp8")


def test_sizes_of_bad_shapes():
    for f, good in ((M.mepic_beam_select_workspace, (2, 4, 4, 100)), (M.mepic_beam_fork_workspace, (2, 4, 4, 8))):
        assert f(*good) > 0
        for i in range(4):
            for bad in (0, -1):
                with pytest.raises(M.MepicError):
                    f(*(good[:i] + (bad,) + good[i + 1:]))
            with pytest.raises(M.MepicError, match="32 bits"):
                f(*(good[:i] + (1 << 32,) + good[i + 1:]))
    assert M.mepic_beam_plan_bytes(CFG, 2, 4, 8) > 0
    for bad in ((0, 4, 8), (2, 33, 8), (2, 4, 0), (1 << 32, 4, 8)):
        with pytest.raises(M.MepicError):
            M.mepic_beam_plan_bytes(CFG, *bad)
    with pytest.raises(M.MepicError):
        M.mepic_beam_plan_bytes(M.Config(15, 8, 2, 128, 10, 100, 1e4), 2, 4, 8)
    for bad in ((0, 4), (2, 0), (2, 33)):
        with pytest.raises(M.MepicError):
            M.mepic_attn_beam_workspace(CFG, *bad)


def test_a_plan_holds_every_entry_of_every_row():
    # one record for each table entry and beam is the most there can be
    for groups, width, stride in ((1, 1, 1), (3, 5, 257), (2, 32, 600)):
        assert M.mepic_beam_plan_bytes(CFG, groups, width, stride) >= 16 * groups * width * stride


# ------------------------------------------------------------------ objects
def _dev(cfg=CFG):
    pool = torch.zeros((cfg.num_pages, cfg.n_kv_heads, cfg.page_size, cfg.head_dim), dtype=torch.bfloat16)
    return SimpleNamespace(cfg=cfg, device=CPU, k_pool=pool, v_pool=pool.clone(), rope=None, status=torch.zeros(1, dtype=torch.int32))


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def _select(**over):
    a = dict(logits=torch.zeros((8, 100)), scores=torch.zeros((2, 4)), done=_i32(2, 4))
    a.update(over)
    return RT.BeamSelect(_dev(), **a)


@pytest.mark.parametrize("over,text", [(dict(logits=torch.zeros((7, 100))), "logits"), (dict(logits=torch.zeros((8, 100), dtype=torch.float64)), "logits"),
                                       (dict(logits=torch.zeros((8, 200))[:, ::2]), "packed"), (dict(logits=torch.zeros((1, 100)).expand(8, 100)), "share memory"),
                                       (dict(scores=torch.zeros(8)), "scores"), (dict(scores=torch.zeros((2, 4), dtype=torch.float64)), "scores"),
                                       (dict(done=_i32(2, 3)), "done"), (dict(done=torch.zeros((2, 4), dtype=torch.bool)), "done")])
def test_select_object_refuses(over, text):
    with pytest.raises(ValueError, match=text):
        _select(**over)


def test_select_object_passes_on_what_the_call_refuses():
    with pytest.raises(M.MepicError):
        _select(n_select=65)


def _fork(**over):
    a = dict(parent=_i32(2, 4), kv_len=_i32(8), page_ids=_i32(8, 5), pos_base=_i32(8, 5), page_ids_out=_i32(8, 5), pos_base_out=_i32(8, 5),
             owned=torch.zeros(10, dtype=torch.uint8), reserve=_i32(6), reserve_used=_i32(1))
    a.update(over)
    return RT.BeamFork(_dev(), **a)


@pytest.mark.parametrize("over,text", [(dict(kv_len=_i32(7)), "whole number"), (dict(kv_len=_i32(0)), "whole number"), (dict(page_ids=_i32(7, 5)), "page_ids"),
                                       (dict(pos_base=_i32(8, 6)), "pos_base"), (dict(page_ids_out=_i32(8, 6)), "page_ids_out"), (dict(pos_base_out=_i32(4, 5)), "pos_base_out"),
                                       (dict(owned=torch.zeros(9, dtype=torch.uint8)), "owned"), (dict(owned=_i32(10)), "owned"), (dict(parent=_i32(8)), "parent"),
                                       (dict(reserve_used=_i32(2)), "reserve_used"), (dict(reserve=torch.zeros(6)), "reserve")])
def test_fork_object_refuses(over, text):
    with pytest.raises(ValueError, match=text):
        _fork(**over)


def test_fork_object_refuses_tables_that_overlap():
    both = _i32(12, 5)
    with pytest.raises(ValueError, match="page_ids_out: must not overlap"):
        _fork(page_ids=both[:8], page_ids_out=both[4:])
    with pytest.raises(ValueError, match="pos_base_out: must not overlap"):
        _fork(page_ids=both[:8], pos_base_out=both[:8])


@pytest.mark.parametrize("over,text", [(dict(dst=_i32(4)), "dst"), (dict(slots=_i32(2)), "slots"), (dict(n_copies=_i32(2)), "n_copies"), (dict(src=torch.zeros(3)), "src")])
def test_copy_object_refuses(over, text):
    with pytest.raises(ValueError, match=text):
        RT.PagesCopy(_dev(), **{**dict(src=_i32(3), dst=_i32(3)), **over})


def test_plan_and_batch_objects_refuse():
    dev = _dev()
    plan = lambda **over: RT.BeamPlan(dev, **{**dict(page_ids=_i32(8, 5), pos_base=_i32(8, 5), kv_len=_i32(8), width=4), **over})
    for over in (dict(width=3), dict(width=0), dict(kv_len=_i32(7)), dict(pos_base=_i32(8, 4)), dict(page_ids=torch.zeros((8, 5))), dict(kv_len=_i32(0), page_ids=_i32(0, 5), pos_base=_i32(0, 5))):
        with pytest.raises(ValueError):
            plan(**over)
    p = SimpleNamespace(dev=dev, groups=2, width=4, stride=5, plan=torch.zeros(16, dtype=torch.uint8))
    q = torch.zeros((8, 8, 128), dtype=torch.bfloat16)
    for d, over in ((dev, dict(q=q[:7])), (dev, dict(q=q.float())), (dev, dict(q_pos=_i32(7))), (dev, dict(q=q[:1].expand(8, 8, 128))), (_dev(SMALL), dict())):
        with pytest.raises(ValueError):
            RT.BeamBatch(d, **{**dict(q=q, q_pos=_i32(8), plan=p), **over})
