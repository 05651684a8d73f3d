"""The tables a step builds on the device, handed to decode and to prefill: the calls they are made for, against the oracle."""
import numpy as np
import pytest
import torch

import paper_2512_16822_b200 as M
from paper_2512_16822_b200 import runtime as RT
from paper_2512_16822_b200.build import build_library
from mepic_inputs import bf16_bits_to_f64, f32_to_bf16_bits
from oracle import mepic_oracle as O
from tree_helpers import dev32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
Hq, Hkv, D, P, THETA = 8, 2, 128, 16, 1e4
SCALE = 1.0 / np.sqrt(D)


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"


def _close(got_bits, want):                          # the tolerance decode and prefill state
    err = np.abs(bf16_bits_to_f64(got_bits) - want)
    assert err.max() <= 2e-2 and err.mean() <= 2e-3, (err.max(), err.mean())


class Serving:
    """Three requests with some context, a reserve of pages, and the oracle's copy of everything."""

    def __init__(self, seed, fp8, kv=(0, 21, 40), stride=12):
        rng = self.rng = np.random.default_rng(seed)
        self.kv, self.fp8, self.used = np.array(kv, dtype=np.int64), fp8, 0
        B, pages = len(kv), 50
        perm = rng.permutation(pages)
        self.ids, self.base = np.zeros((B, stride), dtype=np.int32), np.zeros((B, stride), dtype=np.int32)
        at = 0
        for b in range(B):
            n = -(-int(self.kv[b]) // P)
            self.ids[b, :n], self.base[b, :n] = perm[at:at + n], 7 * b + np.arange(n) * P
            at += n
        self.reserve = perm[at:].astype(np.int32)
        self.kp, self.vp = self.bits((pages, Hkv, P, D)), self.bits((pages, Hkv, P, D))
        self.dev = RT.Device(M.Config(P, Hq, Hkv, D, pages, 400, THETA), self.kp, self.vp)
        self.pools = RT.Fp8Pools(self.dev) if fp8 else None
        if fp8:
            (self.kc, self.ks), (self.vc, self.vs) = O.quantize_pages(self.kp), O.quantize_pages(self.vp)

    def bits(self, shape):
        return f32_to_bf16_bits(self.rng.standard_normal(shape).astype(np.float32))

    def oracle_tables(self, new, max_rows):
        w = O.step_tables(list(self.kv), list(new), self.ids, self.base, list(self.reserve), self.used, P, max_rows)
        self.ids, self.base, self.used, self.kv = w["page_ids"], w["pos_base"], w["reserve_used"], w["kv_len"]
        return w

    def oracle_commit(self, b, slots, k, v):
        if self.fp8:
            O.commit_rows_fp8(self.kc, self.ks, self.vc, self.vs, list(self.ids[b]), list(slots), k, v)
        else:
            O.commit_rows(self.kp, self.vp, list(self.ids[b]), list(slots), k, v)

    def oracle_pools(self):
        return (O.dequantize_pages(self.kc, self.ks), O.dequantize_pages(self.vc, self.vs)) if self.fp8 else (self.kp, self.vp)

    def pools_agree(self):
        if self.fp8:
            pairs = ((self.pools.k_codes, self.kc), (self.pools.v_codes, self.vc), (self.pools.k_scales, self.ks), (self.pools.v_scales, self.vs))
            return all(np.array_equal(t.cpu().numpy(), a) for t, a in pairs)
        return np.array_equal(RT.bf16_bits(self.dev.k_pool), self.kp) and np.array_equal(RT.bf16_bits(self.dev.v_pool), self.vp)


@pytest.mark.parametrize("fp8", [False, True])
def test_prefill_takes_a_steps_tables(fp8):
    # the host chose n_new, so it knows the row offsets the prefill call wants on the host; all else stays on the device
    s, new = Serving(1, fp8), [50, 7, 33]
    B, rows = len(new), sum(new)
    ids, base = dev32(s.ids), dev32(s.base)
    tab = RT.StepTables(s.dev, kv_len=dev32(s.kv), n_new=dev32(new), page_ids=ids, pos_base=base, reserve=dev32(s.reserve),
                        reserve_used=dev32([0]), max_rows=rows)
    tab.run()
    q, k, v = s.bits((rows, Hq, D)), s.bits((rows, Hkv, D)), s.bits((rows, Hkv, D))
    off = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    cfg, out = s.dev.cfg, torch.empty((rows, Hq, D), dtype=torch.bfloat16, device=DEV)
    need = max(M.mepic_attn_prefill_workspace(cfg, B, off), 16)
    call = dict(q_new=RT.bf16_tensor(q, DEV), k_new=RT.bf16_tensor(k, DEV), v_new=RT.bf16_tensor(v, DEV), row_offsets=tab.row_offsets,
                q_slot=tab.row_slot, page_ids=ids, pos_base=base, kv_len=tab.kv_len_out, rope_table=s.dev.rope, out=out,
                workspace=torch.empty(need, dtype=torch.uint8, device=DEV), workspace_bytes=need, status=s.dev.status, row_offsets_host=off,
                table_stride=ids.shape[1], batch=B, sm_scale=SCALE, stream=torch.cuda.current_stream())
    if fp8:
        M.mepic_attn_prefill_fp8(cfg, k_pool=s.pools.k_codes, v_pool=s.pools.v_codes, k_scales=s.pools.k_scales, v_scales=s.pools.v_scales, **call)
    else:
        M.mepic_attn_prefill(cfg, k_pool=s.dev.k_pool, v_pool=s.dev.v_pool, **call)
    torch.cuda.synchronize()
    assert s.dev.read_status() == 0
    w = s.oracle_tables(new, rows)
    got = RT.bf16_bits(out)
    for b in range(B):
        r = slice(off[b], off[b + 1])
        slots = w["row_slot"][r]
        s.oracle_commit(b, slots, k[r], v[r])
        kp, vp = s.oracle_pools()
        _close(got[r], O.prefill_attention_one(q[r], k[r], v[r], list(slots), kp, vp, list(s.ids[b]), list(s.base[b]), int(s.kv[b]), SCALE, THETA))
    assert s.pools_agree()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("graph", [False, True])
def test_decode_loop_over_a_steps_tables(fp8, graph):
    # one token per request and step, from one page into the next: tables, commit and decode, nothing from the host in between
    s = Serving(2, fp8, kv=(1, 15, 30))
    B, ones = 3, dev32([1, 1, 1])
    dec = (RT.Fp8DecodeBatch(s.pools, s.ids, s.base, s.kv, np.zeros(B, np.int32)) if fp8
           else RT.DecodeBatch(s.dev, s.ids, s.base, s.kv, np.zeros(B, np.int32)))
    k, v = (torch.zeros((B, Hkv, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    used, kv = dev32([0]), dev32(s.kv)
    tab = RT.StepTables(s.dev, kv_len=kv, n_new=ones, page_ids=dec.page_ids, pos_base=dec.pos_base, reserve=dev32(s.reserve),
                        reserve_used=used, max_rows=B)
    com = RT.RowsCommit(s.dev, k_new=k, v_new=v, row_offsets=tab.row_offsets, slot_map=tab.slot_map, pools=s.pools)

    def step():
        tab.run(), com.run()
        tab.advance()
        dec.kv_len.copy_(tab.kv_len_out), dec.q_pos.copy_(tab.q_pos)
        dec.run(SCALE)

    if graph:
        live = [dec.page_ids, dec.pos_base, kv, used, *((s.pools.k_codes, s.pools.v_codes, s.pools.k_scales, s.pools.v_scales) if fp8 else (s.dev.k_pool, s.dev.v_pool))]
        saved = [t.clone() for t in live]
        step()
        side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=side):
            step()
        for t, x in zip(live, saved):
            t.copy_(x)
    for it in range(5):
        q_bits, k_bits, v_bits = s.bits((B, Hq, D)), s.bits((B, Hkv, D)), s.bits((B, Hkv, D))
        for t, x in ((dec.q, q_bits), (k, k_bits), (v, v_bits)):
            t.copy_(RT.bf16_tensor(x, DEV))
        g.replay() if graph else step()
        torch.cuda.synchronize()
        assert s.dev.read_status() == 0
        w = s.oracle_tables([1] * B, B)
        assert np.array_equal(dec.kv_len.cpu().numpy(), s.kv) and np.array_equal(dec.q_pos.cpu().numpy(), w["q_pos"])
        for b in range(B):
            s.oracle_commit(b, [int(s.kv[b]) - 1], k_bits[b:b + 1], v_bits[b:b + 1])
        assert s.pools_agree()
        kp, vp = s.oracle_pools()
        got = RT.bf16_bits(dec.out)
        for b in range(B):
            _close(got[b], O.decode_attention_one(q_bits[b], kp, vp, list(s.ids[b]), list(s.base[b]), int(s.kv[b]), int(w["q_pos"][b]), SCALE, THETA))
    assert s.used >= 2, "the loop is meant to pass page boundaries"
