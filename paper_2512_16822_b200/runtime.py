"""Device-side plumbing around the C ABI: torch tensors, streams, uploads.

Nothing here computes any part of the method; it allocates the buffers the ABI
asks the caller to own, moves host tables to the device and issues the calls.
"""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass
from typing import List, Optional, Sequence, Tuple

import numpy as np
import torch

from . import (Config, Segment, Store, MEPIC_SEG_CHUNK, MEPIC_SEG_PROMPT, mepic_attn_decode,
               mepic_decode_plan_build, mepic_decode_plan_patch, mepic_attn_decode_grouped, mepic_attn_decode_grouped_fp8, mepic_attn_decode_grouped_workspace,
               mepic_pages_quantize, mepic_attn_decode_fp8,
               mepic_attn_decode_workspace, mepic_attn_prefill, mepic_attn_prefill_fp8, mepic_attn_prefill_workspace,
               mepic_rope_table_fill, mepic_attn_tree_workspace, lib, _check, _AttnTreeArgsC, _TreeLayoutArgsC, _TreeAcceptArgsC,
               _StepTablesArgsC, _RowsCommitArgsC)


@dataclass
class Table:
    request_id: int
    page_ids: np.ndarray
    pos_base: np.ndarray
    kv_len: int
    recompute_slots: np.ndarray


def build_tables(store: Store, chunks: Sequence[np.ndarray], requests) -> List[Table]:
    """Register each request's chunks, then build its block table, in request order.

    ``requests`` are objects with ``request_id`` and ``segments`` = [(kind, value)] where a chunk
    segment's value indexes ``chunks``.
    """
    out = []
    for r in requests:
        segs = []
        for kind, val in r.segments:
            if kind == MEPIC_SEG_CHUNK:
                cid, _, _, _ = store.chunk_register(chunks[val])
                segs.append(Segment(MEPIC_SEG_CHUNK, cid))
            else:
                segs.append(Segment(MEPIC_SEG_PROMPT, int(val)))
        pages, base, kv_len, slots = store.build_block_table(r.request_id, segs)
        out.append(Table(r.request_id, pages, base, kv_len, slots))
    return out


def pack_tables(tables: Sequence[Table], page_size: int) -> Tuple[np.ndarray, np.ndarray, np.ndarray, np.ndarray]:
    """Host arrays page_ids[B, stride], pos_base[B, stride], kv_len[B], q_pos[B].

    q_pos is the position of the request's last slot: the decode query is the newest token, whose
    K/V is already in the cache.
    """
    stride = max(len(t.page_ids) for t in tables)
    B = len(tables)
    page_ids = np.zeros((B, stride), dtype=np.int32)
    pos_base = np.zeros((B, stride), dtype=np.int32)
    kv_len = np.zeros(B, dtype=np.int32)
    for i, t in enumerate(tables):
        page_ids[i, :len(t.page_ids)] = t.page_ids
        pos_base[i, :len(t.pos_base)] = t.pos_base
        kv_len[i] = t.kv_len
    last = kv_len - 1
    q_pos = pos_base[np.arange(B), last // page_size] + last % page_size
    return page_ids, pos_base, kv_len, q_pos.astype(np.int32)


def bf16_tensor(bits: np.ndarray, device) -> torch.Tensor:
    """uint16 bit patterns -> torch.bfloat16 tensor on ``device`` (no value conversion)."""
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16))
    return t.to(device).view(torch.bfloat16)


def bf16_bits(t: torch.Tensor) -> np.ndarray:
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


class Device:
    """The buffers one pool needs on a GPU: K/V pools, rope table, status word."""

    def __init__(self, cfg: Config, k_bits: Optional[np.ndarray] = None, v_bits: Optional[np.ndarray] = None,
                 device: str = "cuda:0", bf16_pools: bool = True):
        if not torch.cuda.is_available():
            raise RuntimeError("the MEPIC kernels need a CUDA device; there is no CPU path")
        self.cfg = cfg
        self.device = _cuda_device(device)
        shape = (cfg.num_pages, cfg.n_kv_heads, cfg.page_size, cfg.head_dim)
        if not bf16_pools:
            self.k_pool = self.v_pool = None           # a device whose only pools are 8-bit (see Fp8Pools)
        elif k_bits is not None:
            assert k_bits.shape == shape and v_bits.shape == shape
            self.k_pool = bf16_tensor(k_bits, self.device)
            self.v_pool = bf16_tensor(v_bits, self.device)
        else:
            self.k_pool = torch.empty(shape, dtype=torch.bfloat16, device=self.device)
            self.v_pool = torch.empty(shape, dtype=torch.bfloat16, device=self.device)
        self.rope = torch.from_numpy(mepic_rope_table_fill(cfg)).to(self.device)
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)

    @classmethod
    def over(cls, cfg: Config, k_pool: Optional[torch.Tensor] = None, v_pool: Optional[torch.Tensor] = None,
             rope: Optional[torch.Tensor] = None, device: str = "cuda:0") -> "Device":
        """A device whose pools (and rope table) the caller already holds on the GPU: nothing is copied.  Without a rope table
        the library's is built."""
        shape = (cfg.num_pages, cfg.n_kv_heads, cfg.page_size, cfg.head_dim)
        dev = cls.__new__(cls)
        dev.cfg, dev.device = cfg, _cuda_device(device)
        for pool in (k_pool, v_pool):
            if pool is not None:
                _expect(pool, "pool", torch.bfloat16, shape, dev.device)
        dev.k_pool, dev.v_pool = k_pool, v_pool
        if rope is None:
            rope = torch.from_numpy(mepic_rope_table_fill(cfg)).to(dev.device)
        dev.rope = _expect(rope, "rope", torch.float32, (cfg.max_position + 1, cfg.head_dim // 2, 2), dev.device)
        dev.status = torch.zeros(1, dtype=torch.int32, device=dev.device)
        return dev

    def read_status(self) -> int:
        return int(self.status.item())


def _cuda_device(device) -> torch.device:
    """``device`` with an index: "cuda" is the GPU that is current now."""
    d = torch.device(device)
    return torch.device("cuda", torch.cuda.current_device()) if d.type == "cuda" and d.index is None else d


def _lies_on(t: torch.Tensor, device: torch.device) -> bool:
    return t.device.type == device.type and (device.index is None or t.device.index == device.index)


def _expect(t: torch.Tensor, name: str, dtype: torch.dtype, shape, device: torch.device) -> torch.Tensor:
    """``t`` if it is a packed tensor of that type, shape and device (-1 in ``shape``: any size); raises ValueError otherwise."""
    if t.dtype != dtype or not _lies_on(t, device) or t.dim() != len(shape) or any(w >= 0 and g != w for g, w in zip(t.shape, shape)):
        raise ValueError(f"{name}: expected {dtype} {tuple(shape)} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    return t


def _row_stride(t: torch.Tensor, name: str, heads: int, head_dim: int, device: torch.device) -> int:
    """Row stride in elements of bf16 rows [rows, heads, head_dim] whose rows are packed but may lie apart."""
    if t.dtype != torch.bfloat16 or not _lies_on(t, device) or t.dim() != 3 or t.shape[1:] != (heads, head_dim):
        raise ValueError(f"{name}: expected bfloat16 [rows, {heads}, {head_dim}] on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    if t.stride(2) != 1 or (heads > 1 and t.stride(1) != head_dim):
        raise ValueError(f"{name}: the heads of a row must be packed")
    if t.shape[0] <= 1:
        return heads * head_dim
    if t.stride(0) < heads * head_dim:           # a broadcast row has stride 0, which the calls read as "packed"
        raise ValueError(f"{name}: rows must not share memory (row stride {t.stride(0)}, a row has {heads * head_dim} elements)")
    return t.stride(0)


def _pools_for(dev: Device, pools: Optional["Fp8Pools"]):
    """The K and V pools a call on ``dev`` uses: those of ``pools`` (8-bit) or the device's bf16 ones.  A page id that is valid
    for the device's configuration must be valid in them: ValueError otherwise."""
    cfg = dev.cfg
    shape = (cfg.num_pages, cfg.n_kv_heads, cfg.page_size, cfg.head_dim)
    if pools is None:
        if dev.k_pool is None or dev.v_pool is None:
            raise ValueError("the device has no bf16 pools: name the 8-bit pools to use")
        return tuple(_expect(t, "pool", torch.bfloat16, shape, dev.device) for t in (dev.k_pool, dev.v_pool))
    codes = tuple(_expect(t, "codes", torch.uint8, shape, dev.device) for t in (pools.k_codes, pools.v_codes))
    for t in (pools.k_scales, pools.v_scales):
        _expect(t, "scales", torch.float32, shape[:2], dev.device)
    return codes


class DecodeBatch:
    """Device copies of one decode batch's tables plus output and workspace."""

    def __init__(self, dev: Device, page_ids: np.ndarray, pos_base: np.ndarray, kv_len: np.ndarray,
                 q_pos: np.ndarray, q_bits: Optional[np.ndarray] = None):
        cfg = dev.cfg
        self.dev = dev
        self.batch, self.stride = page_ids.shape
        d = dev.device
        # The per-step inputs (q and the tables) are views of ONE device buffer, so that a serving loop can bring a
        # step's inputs over with a single host-to-device copy from a pinned mirror (see host_mirror / upload).
        qshape = (self.batch, cfg.n_q_heads, cfg.head_dim)
        parts = [("q", qshape, torch.bfloat16), ("page_ids", (self.batch, self.stride), torch.int32),
                 ("pos_base", (self.batch, self.stride), torch.int32), ("kv_len", (self.batch,), torch.int32),
                 ("q_pos", (self.batch,), torch.int32)]
        self._layout, at = [], 0
        for name, shape, dt in parts:
            n = int(np.prod(shape)) * torch.empty((), dtype=dt).element_size()
            self._layout.append((name, shape, dt, at, n))
            at += -(-n // 256) * 256                                   # every view starts 256-byte aligned
        self.step_inputs = torch.empty(at, dtype=torch.uint8, device=d)
        for name, shape, dt, off, n in self._layout:
            setattr(self, name, self.step_inputs[off:off + n].view(dt).view(shape))
        self.page_ids.copy_(torch.from_numpy(np.ascontiguousarray(page_ids, dtype=np.int32)))
        self.pos_base.copy_(torch.from_numpy(np.ascontiguousarray(pos_base, dtype=np.int32)))
        self.kv_len.copy_(torch.from_numpy(np.ascontiguousarray(kv_len, dtype=np.int32)))
        self.q_pos.copy_(torch.from_numpy(np.ascontiguousarray(q_pos, dtype=np.int32)))
        if q_bits is not None:
            self.q.view(torch.int16).copy_(torch.from_numpy(np.ascontiguousarray(q_bits).view(np.int16)))
        self.out = torch.empty(qshape, dtype=torch.bfloat16, device=d)
        self.ws_bytes = mepic_attn_decode_workspace(cfg, self.batch)
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=d)

    def run(self, sm_scale: float, stream=None) -> torch.Tensor:
        s = stream if stream is not None else torch.cuda.current_stream(self.dev.device)
        mepic_attn_decode(self.dev.cfg, q=self.q, k_pool=self.dev.k_pool, v_pool=self.dev.v_pool,
                          page_ids=self.page_ids, pos_base=self.pos_base, kv_len=self.kv_len, q_pos=self.q_pos,
                          rope_table=self.dev.rope, out=self.out, workspace=self.workspace,
                          workspace_bytes=self.ws_bytes, status=self.dev.status, table_stride=self.stride,
                          batch=self.batch, sm_scale=sm_scale, stream=s)
        return self.out

    def host_mirror(self):
        """Pinned host buffer with the layout of ``step_inputs`` and named views into it (q as int16 bit patterns)."""
        host = torch.empty(self.step_inputs.numel(), dtype=torch.uint8).pin_memory()
        views = {}
        for name, shape, dt, off, n in self._layout:
            hdt = torch.int16 if dt == torch.bfloat16 else dt
            views[name] = host[off:off + n].view(hdt).view(shape)
        return host, views

    def upload(self, host: torch.Tensor) -> None:
        """One asynchronous host-to-device copy of a whole step's inputs (on the current stream)."""
        self.step_inputs.copy_(host, non_blocking=True)


class Fp8Pools:
    """8-bit (e4m3) copies of a device's K/V pools with one scale per (page, kv head), made by the library's quantiser."""

    def __init__(self, dev: Device, pages: Optional[np.ndarray] = None):
        cfg = dev.cfg
        self.dev = dev
        d = dev.device
        shape = (cfg.num_pages, cfg.n_kv_heads, cfg.page_size, cfg.head_dim)
        self.k_codes = torch.zeros(shape, dtype=torch.uint8, device=d)
        self.v_codes = torch.zeros(shape, dtype=torch.uint8, device=d)
        self.k_scales = torch.ones((cfg.num_pages, cfg.n_kv_heads), dtype=torch.float32, device=d)
        self.v_scales = torch.ones((cfg.num_pages, cfg.n_kv_heads), dtype=torch.float32, device=d)
        if dev.k_pool is not None:                     # pools without a bf16 original start empty: prefill fills them
            self.quantize(np.arange(cfg.num_pages, dtype=np.int32) if pages is None else pages)

    @classmethod
    def over(cls, dev: Device, k_codes: torch.Tensor, v_codes: torch.Tensor, k_scales: torch.Tensor, v_scales: torch.Tensor) -> "Fp8Pools":
        """8-bit pools the caller already holds: nothing is copied or quantised."""
        pools = cls.__new__(cls)
        pools.dev = dev
        pools.k_codes, pools.v_codes, pools.k_scales, pools.v_scales = k_codes, v_codes, k_scales, v_scales
        _pools_for(dev, pools)
        return pools

    def quantize(self, pages: np.ndarray, stream=None) -> None:
        lst = torch.from_numpy(np.ascontiguousarray(pages, dtype=np.int32)).to(self.dev.device)
        s = stream if stream is not None else torch.cuda.current_stream(self.dev.device)
        for src, dst, sc in ((self.dev.k_pool, self.k_codes, self.k_scales), (self.dev.v_pool, self.v_codes, self.v_scales)):
            mepic_pages_quantize(self.dev.cfg, src_pool=src, dst_pool=dst, scales=sc, pages=lst, n_pages=int(lst.numel()),
                                 status=self.dev.status, stream=s)


class Fp8DecodeBatch(DecodeBatch):
    """A decode batch that reads the 8-bit pools."""

    def __init__(self, pools: Fp8Pools, page_ids, pos_base, kv_len, q_pos, q_bits=None):
        super().__init__(pools.dev, page_ids, pos_base, kv_len, q_pos, q_bits)
        self.pools = pools

    def run(self, sm_scale: float, stream=None) -> torch.Tensor:
        s = stream if stream is not None else torch.cuda.current_stream(self.dev.device)
        mepic_attn_decode_fp8(self.dev.cfg, q=self.q, k_pool=self.pools.k_codes, v_pool=self.pools.v_codes,
                              k_scales=self.pools.k_scales, v_scales=self.pools.v_scales, page_ids=self.page_ids,
                              pos_base=self.pos_base, kv_len=self.kv_len, q_pos=self.q_pos, rope_table=self.dev.rope,
                              out=self.out, workspace=self.workspace, workspace_bytes=self.ws_bytes,
                              status=self.dev.status, table_stride=self.stride, batch=self.batch, sm_scale=sm_scale,
                              stream=s)
        return self.out


class GroupedDecodeBatch:
    """One decode batch run through the sharing-aware path: host plan + its device copy, output, workspace."""

    def __init__(self, dev: Device, page_ids: np.ndarray, pos_base: np.ndarray, kv_len: np.ndarray,
                 q_pos: np.ndarray, q_bits: Optional[np.ndarray] = None, n_sms: int = 0):
        cfg = dev.cfg
        self.dev = dev
        self.batch = page_ids.shape[0]
        d = dev.device
        with torch.cuda.device(d):
            built = mepic_decode_plan_build(cfg, page_ids, pos_base, kv_len, n_sms)
        # the host copy lives in page-locked memory: a patch uploads stretches of it without a staging copy
        self._plan_pinned = torch.empty(len(built), dtype=torch.int32).pin_memory()
        self.plan_host = self._plan_pinned.numpy()
        self.plan_host[:] = built
        self.plan = torch.from_numpy(built).to(d)
        self._uploaded = None
        self.kv_len = torch.from_numpy(np.ascontiguousarray(kv_len, dtype=np.int32)).to(d)
        self.q_pos = torch.from_numpy(np.ascontiguousarray(q_pos, dtype=np.int32)).to(d)
        qshape = (self.batch, cfg.n_q_heads, cfg.head_dim)
        self.q = bf16_tensor(q_bits, d) if q_bits is not None else torch.empty(qshape, dtype=torch.bfloat16, device=d)
        self.out = torch.empty(qshape, dtype=torch.bfloat16, device=d)
        self.ws_bytes = mepic_attn_decode_grouped_workspace(cfg, self.plan_host)
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=d)

    def run(self, sm_scale: float, stream=None) -> torch.Tensor:
        s = stream if stream is not None else torch.cuda.current_stream(self.dev.device)
        mepic_attn_decode_grouped(self.dev.cfg, q=self.q, k_pool=self.dev.k_pool, v_pool=self.dev.v_pool,
                                  plan=self.plan, plan_host=self.plan_host, kv_len=self.kv_len, q_pos=self.q_pos,
                                  rope_table=self.dev.rope, out=self.out, workspace=self.workspace,
                                  workspace_bytes=self.ws_bytes, status=self.dev.status, batch=self.batch,
                                  sm_scale=sm_scale, stream=s)
        return self.out

    def patch(self, page_ids: np.ndarray, pos_base: np.ndarray, kv_len: np.ndarray) -> int:
        """Requests gained pages: patch the host plan in place and upload only what changed (on the current stream).
        Returns the bytes uploaded.  kv_len itself is the caller's per-step input and is not touched here."""
        if self._uploaded is not None:
            self._uploaded.synchronize()              # the previous patch's copies have read the host buffer
        ranges = mepic_decode_plan_patch(self.dev.cfg, self.plan_host, page_ids, pos_base, kv_len)
        sent = 0
        for lo, n in ranges:
            self.plan[lo:lo + n].copy_(self._plan_pinned[lo:lo + n], non_blocking=True)
            sent += 4 * n
        if ranges:
            self._uploaded = torch.cuda.Event(); self._uploaded.record()
            need = mepic_attn_decode_grouped_workspace(self.dev.cfg, self.plan_host)
            if need > self.ws_bytes:                  # more partial slots than before: a larger workspace (rare)
                self.ws_bytes = need + need // 8
                self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.dev.device)
        return sent


class PrefillBatch:
    """Device copies of one prefill batch: new rows, their slots, tables, output, workspace."""

    def __init__(self, dev: Device, page_ids: np.ndarray, pos_base: np.ndarray, kv_len: np.ndarray,
                 row_offsets: np.ndarray, q_slot: np.ndarray, q_bits: np.ndarray, k_bits: np.ndarray,
                 v_bits: np.ndarray):
        cfg = dev.cfg
        self.dev = dev
        self.batch, self.stride = page_ids.shape
        d = dev.device
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(d)
        self.page_ids, self.pos_base, self.kv_len = i32(page_ids), i32(pos_base), i32(kv_len)
        self.row_offsets_host = np.ascontiguousarray(row_offsets, dtype=np.int32)
        self.row_offsets, self.q_slot = i32(row_offsets), i32(q_slot)
        self.q_new, self.k_new, self.v_new = bf16_tensor(q_bits, d), bf16_tensor(k_bits, d), bf16_tensor(v_bits, d)
        self.out = torch.empty(self.q_new.shape, dtype=torch.bfloat16, device=d)
        self.ws_bytes = mepic_attn_prefill_workspace(cfg, self.batch, self.row_offsets_host)
        self.workspace = torch.empty(max(self.ws_bytes, 16), dtype=torch.uint8, device=d)

    def run(self, sm_scale: float, stream=None) -> torch.Tensor:
        s = stream if stream is not None else torch.cuda.current_stream(self.dev.device)
        mepic_attn_prefill(self.dev.cfg, q_new=self.q_new, k_new=self.k_new, v_new=self.v_new,
                           row_offsets=self.row_offsets, q_slot=self.q_slot, k_pool=self.dev.k_pool,
                           v_pool=self.dev.v_pool, page_ids=self.page_ids, pos_base=self.pos_base,
                           kv_len=self.kv_len, rope_table=self.dev.rope, out=self.out, workspace=self.workspace,
                           workspace_bytes=self.ws_bytes, status=self.dev.status,
                           row_offsets_host=self.row_offsets_host, table_stride=self.stride, batch=self.batch,
                           sm_scale=sm_scale, stream=s)
        return self.out

    def repeated(self) -> bool:
        """Whether the last call ran its repeat launch (first workspace word; synchronises the device)."""
        return int(self.workspace[:4].view(torch.int32).item()) != 0


class Fp8PrefillBatch(PrefillBatch):
    """A prefill batch that commits into, and attends over, the 8-bit pools."""

    def __init__(self, pools: Fp8Pools, page_ids, pos_base, kv_len, row_offsets, q_slot, q_bits, k_bits, v_bits):
        super().__init__(pools.dev, page_ids, pos_base, kv_len, row_offsets, q_slot, q_bits, k_bits, v_bits)
        self.pools = pools

    def run(self, sm_scale: float, stream=None) -> torch.Tensor:
        s = stream if stream is not None else torch.cuda.current_stream(self.dev.device)
        mepic_attn_prefill_fp8(self.dev.cfg, q_new=self.q_new, k_new=self.k_new, v_new=self.v_new,
                               row_offsets=self.row_offsets, q_slot=self.q_slot, k_pool=self.pools.k_codes,
                               v_pool=self.pools.v_codes, k_scales=self.pools.k_scales, v_scales=self.pools.v_scales,
                               page_ids=self.page_ids, pos_base=self.pos_base, kv_len=self.kv_len,
                               rope_table=self.dev.rope, out=self.out, workspace=self.workspace,
                               workspace_bytes=self.ws_bytes, status=self.dev.status,
                               row_offsets_host=self.row_offsets_host, table_stride=self.stride, batch=self.batch,
                               sm_scale=sm_scale, stream=s)
        return self.out


class Fp8GroupedDecodeBatch(GroupedDecodeBatch):
    """The sharing-aware decode path over the 8-bit pools."""

    def __init__(self, pools: Fp8Pools, page_ids, pos_base, kv_len, q_pos, q_bits=None, n_sms: int = 0):
        super().__init__(pools.dev, page_ids, pos_base, kv_len, q_pos, q_bits, n_sms)
        self.pools = pools

    def run(self, sm_scale: float, stream=None) -> torch.Tensor:
        s = stream if stream is not None else torch.cuda.current_stream(self.dev.device)
        mepic_attn_decode_grouped_fp8(self.dev.cfg, q=self.q, k_pool=self.pools.k_codes, v_pool=self.pools.v_codes,
                                      k_scales=self.pools.k_scales, v_scales=self.pools.v_scales, plan=self.plan,
                                      plan_host=self.plan_host, kv_len=self.kv_len, q_pos=self.q_pos,
                                      rope_table=self.dev.rope, out=self.out, workspace=self.workspace,
                                      workspace_bytes=self.ws_bytes, status=self.dev.status, batch=self.batch,
                                      sm_scale=sm_scale, stream=s)
        return self.out


class _StepCall:
    """One call of a step over buffers that stay in place: the argument struct is filled once, ``run`` only launches, so that a
    step costs the host a few microseconds and can be captured into a graph.  Inputs are read when the kernels run.  The results
    and the workspace are the object's own and the next ``run`` writes them again: runs that may overlap on the GPU need an
    object each.  An object may be dropped while its kernels still run on a torch stream; on a stream of the caller's own (a raw
    handle, an ExternalStream) it has to outlive them, and a graph that captured it always."""

    def _bind(self, dev: Device, name: str, args, *, with_cfg: bool = True, extra=(), keep=()):
        self.dev = dev
        self._index = _cuda_device(dev.device).index
        self._args, self._cfg, self._keep = args, dev.cfg.c(), keep            # the struct holds raw addresses: keep the tensors alive
        self._fn = getattr(lib(), name)
        self._argv = ((C.byref(self._cfg),) if with_cfg else ()) + (C.byref(args),) + tuple(extra)
        self._streams = set()                                                  # raw streams the bound tensors are recorded on

    def _record(self, stream, raw: int) -> None:
        """Tells the allocator that ``stream`` uses what is bound: memory of a dropped object is handed out again only when
        its kernels are through.  Not for a stream of the caller's own: the allocator comes back to the stream when the
        memory is freed, and such a stream may be gone by then."""
        if isinstance(stream, int):
            return
        if stream is None:
            stream = torch.cuda.current_stream(self._index)
        self._streams.add(raw)
        if stream.stream_id and stream.stream_id % 2 == 0:                     # a handle that torch did not make
            return
        held = list(vars(self).values()) + [self.dev.rope, self.dev.status]
        for t in self._keep:
            held += [t.k_codes, t.v_codes, t.k_scales, t.v_scales] if isinstance(t, Fp8Pools) else [t]
        for t in held:
            if isinstance(t, torch.Tensor) and t.numel():
                t.record_stream(stream)

    def _launch(self, stream=None) -> None:
        if torch._C._cuda_getDevice() != self._index:                # (the private forms of current_device and current_stream: the
            with torch.cuda.device(self._index):                     # public ones cost as much as the launch)
                return self._launch(stream)
        if stream is None:
            s = torch._C._cuda_getCurrentRawStream(self._index)
        else:
            s = stream if isinstance(stream, int) else stream.cuda_stream
        if s not in self._streams:
            self._record(stream, s)
        code = self._fn(*self._argv, s)
        if code:
            _check(code)

    def _i32(self, *shape):
        return torch.empty(shape, dtype=torch.int32, device=self.dev.device)


class TreeLayout(_StepCall):
    """Positions and ancestor masks of drafted rows: run() -> dict(row_pos [rows], tree_mask [rows, mask_words])."""

    def __init__(self, dev: Device, *, parent, row_offsets, kv_len, pos_base, mask_words: int):
        self.dev, d, i32 = dev, dev.device, torch.int32
        batch, rows = kv_len.numel(), parent.numel()
        _expect(parent, "parent", i32, (rows,), d), _expect(row_offsets, "row_offsets", i32, (batch + 1,), d)
        _expect(kv_len, "kv_len", i32, (batch,), d), _expect(pos_base, "pos_base", i32, (batch, -1), d)
        self.row_pos, self.tree_mask = self._i32(rows), self._i32(rows, mask_words)
        self._bind(dev, "mepic_tree_layout",
                   _TreeLayoutArgsC(parent.data_ptr(), row_offsets.data_ptr(), kv_len.data_ptr(), pos_base.data_ptr(), self.row_pos.data_ptr(),
                                    self.tree_mask.data_ptr(), dev.status.data_ptr(), pos_base.shape[1], batch, rows, mask_words),
                   keep=(parent, row_offsets, kv_len, pos_base))
        self._result = dict(row_pos=self.row_pos, tree_mask=self.tree_mask)

    def run(self, stream=None):
        self._launch(stream)
        return self._result


class TreeBatch(_StepCall):
    """Attention of drafted rows over the paged context and each other.  q / k_new / v_new are bf16 [rows, heads, head_dim];
    rows may lie apart (slices of one fused projection).  ``pools``: 8-bit pools to read instead of the device's bf16 ones."""

    def __init__(self, dev: Device, *, q, k_new, v_new, row_offsets, row_pos, tree_mask, page_ids, pos_base, kv_len, max_rows: int,
                 pools: Optional[Fp8Pools] = None):
        cfg, d, i32 = dev.cfg, dev.device, torch.int32
        rows, batch = q.shape[0], kv_len.numel()
        q_stride = _row_stride(q, "q", cfg.n_q_heads, cfg.head_dim, d)
        kv_stride = _row_stride(k_new, "k_new", cfg.n_kv_heads, cfg.head_dim, d)
        if _row_stride(v_new, "v_new", cfg.n_kv_heads, cfg.head_dim, d) != kv_stride or k_new.shape[0] != rows or v_new.shape[0] != rows:
            raise ValueError("k_new and v_new must have q's rows and one row stride")
        _expect(row_offsets, "row_offsets", i32, (batch + 1,), d), _expect(row_pos, "row_pos", i32, (rows,), d)
        _expect(tree_mask, "tree_mask", i32, (rows, -1), d), _expect(page_ids, "page_ids", i32, (batch, -1), d)
        _expect(pos_base, "pos_base", i32, tuple(page_ids.shape), d), _expect(kv_len, "kv_len", i32, (batch,), d)
        k_pool, v_pool = _pools_for(dev, pools)
        with torch.cuda.device(d):
            ws = mepic_attn_tree_workspace(cfg, max_rows)
        self.out = torch.empty((rows, cfg.n_q_heads, cfg.head_dim), dtype=torch.bfloat16, device=d)
        self.workspace = torch.empty(ws, dtype=torch.uint8, device=d)
        args = _AttnTreeArgsC(q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), row_offsets.data_ptr(), row_pos.data_ptr(),
                              tree_mask.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(), page_ids.data_ptr(), pos_base.data_ptr(),
                              kv_len.data_ptr(), dev.rope.data_ptr(), self.out.data_ptr(), self.workspace.data_ptr(), ws,
                              dev.status.data_ptr(), page_ids.shape[1], batch, rows, max_rows, tree_mask.shape[1], q_stride, kv_stride, 0.0)
        self._bind(dev, "mepic_attn_tree" if pools is None else "mepic_attn_tree_fp8", args,
                   extra=() if pools is None else (pools.k_scales.data_ptr(), pools.v_scales.data_ptr()),
                   keep=(q, k_new, v_new, row_offsets, row_pos, tree_mask, page_ids, pos_base, kv_len, k_pool, v_pool, pools))

    def run(self, sm_scale: float, stream=None) -> torch.Tensor:
        self._args.sm_scale = sm_scale
        self._launch(stream)
        return self.out


class TreeAccept(_StepCall):
    """The path the model agrees with: run() -> dict(n_accept [B], accept_rows [B, max_accept], next_token [B])."""

    def __init__(self, dev: Device, *, parent, row_offsets, draft, target, root, max_accept: int):
        self.dev, d, i32 = dev, dev.device, torch.int32
        batch, rows = root.numel(), parent.numel()
        for t, name in ((parent, "parent"), (draft, "draft"), (target, "target")):
            _expect(t, name, i32, (rows,), d)
        _expect(row_offsets, "row_offsets", i32, (batch + 1,), d), _expect(root, "root", i32, (batch,), d)
        self.n_accept, self.accept_rows, self.next_token = self._i32(batch), self._i32(batch, max_accept), self._i32(batch)
        self._bind(dev, "mepic_tree_accept",
                   _TreeAcceptArgsC(parent.data_ptr(), row_offsets.data_ptr(), draft.data_ptr(), target.data_ptr(), root.data_ptr(),
                                    self.n_accept.data_ptr(), self.accept_rows.data_ptr(), self.next_token.data_ptr(),
                                    dev.status.data_ptr(), batch, rows, max_accept),
                   with_cfg=False, keep=(parent, row_offsets, draft, target, root))
        self._result = dict(n_accept=self.n_accept, accept_rows=self.accept_rows, next_token=self.next_token)

    def run(self, stream=None):
        self._launch(stream)
        return self._result


class StepTables(_StepCall):
    """Block tables and slot maps from lengths: page_ids / pos_base grow in place out of ``reserve``;
    run() -> dict(row_offsets, row_slot, slot_map, kv_len, q_pos, reserve_used).  The tables may be a DecodeBatch's own
    (``batch.page_ids``, ``batch.pos_base``); its next run then needs ``kv_len`` and ``q_pos`` copied over."""

    def __init__(self, dev: Device, *, kv_len, n_new, page_ids, pos_base, reserve, reserve_used, max_rows: int):
        self.dev, d, i32 = dev, dev.device, torch.int32
        batch = kv_len.numel()
        _expect(kv_len, "kv_len", i32, (batch,), d), _expect(n_new, "n_new", i32, (batch,), d)
        _expect(page_ids, "page_ids", i32, (batch, -1), d), _expect(pos_base, "pos_base", i32, tuple(page_ids.shape), d)
        _expect(reserve, "reserve", i32, (-1,), d), _expect(reserve_used, "reserve_used", i32, (1,), d)
        self.kv_len, self.reserve_used = kv_len, reserve_used
        self.kv_len_out, self.q_pos, self.reserve_used_out, self.row_offsets = self._i32(batch), self._i32(batch), self._i32(1), self._i32(batch + 1)
        self.row_slot, self.slot_map = self._i32(max_rows), torch.empty(max_rows, dtype=torch.int64, device=d)
        self._bind(dev, "mepic_step_tables",
                   _StepTablesArgsC(kv_len.data_ptr(), n_new.data_ptr(), page_ids.data_ptr(), pos_base.data_ptr(), reserve.data_ptr() or None,
                                    reserve_used.data_ptr(), self.row_offsets.data_ptr(), self.row_slot.data_ptr() or None,
                                    self.slot_map.data_ptr() or None, self.kv_len_out.data_ptr(), self.q_pos.data_ptr(),
                                    self.reserve_used_out.data_ptr(), dev.status.data_ptr(), page_ids.shape[1], batch, max_rows, reserve.numel()),
                   keep=(kv_len, n_new, page_ids, pos_base, reserve, reserve_used))
        self._result = dict(row_offsets=self.row_offsets, row_slot=self.row_slot, slot_map=self.slot_map, kv_len=self.kv_len_out,
                            q_pos=self.q_pos, reserve_used=self.reserve_used_out)

    def run(self, stream=None):
        self._launch(stream)
        return self._result

    def advance(self) -> None:
        """The step's lengths and its use of the reserve become the next step's inputs (on the current stream)."""
        self.kv_len.copy_(self.kv_len_out)
        self.reserve_used.copy_(self.reserve_used_out)


class RowsCommit(_StepCall):
    """K/V rows into their physical slots.  ``src_rows`` (accept_rows of TreeAccept): which source row each appended row is."""

    def __init__(self, dev: Device, *, k_new, v_new, row_offsets, slot_map, src_rows=None, pools: Optional[Fp8Pools] = None):
        cfg, d = dev.cfg, dev.device
        batch, max_rows = row_offsets.numel() - 1, slot_map.numel()
        kv_stride = _row_stride(k_new, "k_new", cfg.n_kv_heads, cfg.head_dim, d)
        if _row_stride(v_new, "v_new", cfg.n_kv_heads, cfg.head_dim, d) != kv_stride or v_new.shape[0] != k_new.shape[0]:
            raise ValueError("k_new and v_new must have the same rows and row stride")
        _expect(row_offsets, "row_offsets", torch.int32, (batch + 1,), d), _expect(slot_map, "slot_map", torch.int64, (max_rows,), d)
        if src_rows is not None:
            _expect(src_rows, "src_rows", torch.int32, (batch, -1), d)
        k_pool, v_pool = _pools_for(dev, pools)
        self._bind(dev, "mepic_rows_commit" if pools is None else "mepic_rows_commit_fp8",
                   _RowsCommitArgsC(k_new.data_ptr(), v_new.data_ptr(), row_offsets.data_ptr(), slot_map.data_ptr(),
                                    None if src_rows is None else src_rows.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(),
                                    dev.status.data_ptr(), 0 if src_rows is None else src_rows.shape[1], batch, max_rows, k_new.shape[0], kv_stride),
                   extra=() if pools is None else (pools.k_scales.data_ptr(), pools.v_scales.data_ptr()),
                   keep=(k_new, v_new, row_offsets, slot_map, src_rows, k_pool, v_pool, pools))

    def run(self, stream=None) -> None:
        self._launch(stream)
