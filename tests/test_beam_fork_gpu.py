"""Block tables of forked beams (mepic_beam_fork) and page copies (mepic_pages_copy / _fp8), against plain statements of both."""
import numpy as np
import pytest
import torch

import paper_2512_16822_b200 as M
from paper_2512_16822_b200 import runtime as RT
from paper_2512_16822_b200.build import build_library
from beam_helpers import fork, dev32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"


class Tables:
    """Groups of beams over a context of the store's pages (not owned) and pages of the reserve, as a search leaves them."""

    def __init__(self, seed, *, G, W, P, context, grown, lens=None, spare=None, stride_extra=3, ragged=True):
        rng = self.rng = np.random.default_rng(seed)
        self.P, self.G, self.W = P, G, W
        self.kv = np.zeros((G, W), dtype=np.int64)
        ents = -(-(context + grown) // P) if context + grown else 0
        stride = max(1, ents + stride_extra)
        t = np.full((G, W, stride), -1, dtype=np.int64)
        used, own = 0, []
        for g in range(G):
            n = context + grown - (int(rng.integers(0, grown // 2 + 1)) if ragged else 0)
            self.kv[g] = n
            full, last = min(context, n) // P, -(-n // P)
            t[g, :, :full] = used + np.arange(full)
            used += full
            for e in range(full, last):
                t[g] = t[g, rng.integers(0, W, size=W)]
                t[g, :, e] = used + np.arange(W)
                own += list(range(used, used + W))
                used += W
        if lens is not None:
            self.kv = np.asarray(lens).reshape(G, W)
        spare = G * W + 7 if spare is None else spare
        self.num_pages = max(1, used + spare)
        perm = rng.permutation(self.num_pages)
        self.ids = np.where(t >= 0, perm[np.maximum(t, 0)], -1).reshape(G * W, stride)
        self.base = (np.arange(stride)[None] * P + rng.integers(0, 99, size=(G * W, 1)))
        held = {int(self.ids[r, e]) for r in range(G * W) for e in range(-(-int(self.kv.reshape(-1)[r]) // P))}
        out = [p for p in perm[own].tolist() if p in held] if own else []
        self.owned = np.zeros(self.num_pages, dtype=np.uint8)
        self.owned[out] = 1
        self.owned[perm[used:]] = 1
        self.reserve = np.array(rng.permutation(out).tolist() + perm[used:].tolist(), dtype=np.int64)
        self.used = len(out)

    def call(self, parent, **over):
        self.dev = RT.Device.over(M.Config(self.P, 8, 2, 128, self.num_pages, max(64, self.P), 1e4))
        stride = self.ids.shape[1]
        rows_out = parent.size
        self.d = dict(parent=dev32(parent), kv_len=dev32(self.kv.reshape(-1)), page_ids=dev32(self.ids), pos_base=dev32(self.base),
                      page_ids_out=dev32(np.full((rows_out, stride), -9)), pos_base_out=dev32(np.full((rows_out, stride), -9)),
                      owned=torch.from_numpy(self.owned).cuda(), reserve=dev32(self.reserve), reserve_used=dev32([self.used]))
        self.d.update(over)
        op = RT.BeamFork(self.dev, **self.d)
        op.workspace.fill_(255)
        return op

    def check(self, parent, op, got, status=0):
        torch.cuda.synchronize()
        got = {k: v.cpu().numpy() for k, v in got.items()}
        ids, base = self.d["page_ids_out"].cpu().numpy(), self.d["pos_base_out"].cpu().numpy()
        ok = np.where((parent >= 0) & (parent < self.W), parent, -1)
        want = fork(ok, self.kv.reshape(-1), self.ids, self.base, self.owned, self.reserve.tolist(), self.used, self.P)
        assert self.dev.read_status() == want["status"] | status
        rows = parent.size
        if want["status"]:
            assert (got["kv_len"] == 0).all() and got["n_copies"][0] == 0 and got["reserve_used"][0] == self.used
            assert (got["copy_src"] == -1).all() and (got["copy_dst"] == -1).all() and (got["copy_slots"] == -1).all()
            assert (self.d["reserve"].cpu().numpy() == self.reserve).all()
            return want
        for r, (p, b, n) in enumerate(want["rows"]):
            assert got["kv_len"][r] == n
            assert ids[r, :len(p)].tolist() == p and (ids[r, len(p):] == -9).all(), r
            assert base[r, :len(b)].tolist() == b and (base[r, len(b):] == -9).all(), r
        c = want["copies"]
        assert got["n_copies"][0] == len(c) and got["reserve_used"][0] == want["used"]
        for name, i in (("copy_src", 0), ("copy_dst", 1), ("copy_slots", 2)):
            assert got[name].tolist() == [x[i] for x in c] + [-1] * (rows - len(c)), name
        assert self.d["reserve"].cpu().numpy().tolist() == want["reserve"]
        return want


def _run(t, parent, status=0):
    op = t.call(parent)
    want = t.check(parent, op, op.run(), status)
    op.run()                                                      # the call reads what it read before: the same again
    return t.check(parent, op, op._result, status), want


@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("W", [1, 2, 5, 8, 32])
@pytest.mark.parametrize("context,grown", [(0, 1), (16, 0), (100, 0), (100, 45), (128, 64), (0, 300)])
def test_forks_of_a_search(P, W, context, grown):
    t = Tables(W + P + grown, G=4, W=W, P=P, context=context, grown=grown)
    for _ in range(2):
        _run(t, t.rng.integers(-1, W, size=(4, W)))
    _run(t, np.tile(np.arange(W), (4, 1)))                         # nothing changes
    _run(t, np.zeros((4, W), dtype=np.int64))                      # one beam takes all
    _run(t, np.full((4, W), -1))                                   # every request ends


@pytest.mark.parametrize("wi,wo", [(1, 4), (1, 32), (4, 1), (3, 7), (32, 2)])
def test_widths_that_change(wi, wo):
    t = Tables(wi + wo, G=3, W=wi, P=16, context=75, grown=40, spare=3 * 40)
    _run(t, t.rng.integers(0, wi, size=(3, wo)))


def test_a_prompts_last_page_is_never_written():
    # the prompt's pages are the store's: its partly filled last page is copied for every beam, the first among them
    t = Tables(3, G=2, W=1, P=16, context=90, grown=0, spare=20)
    full = 90 // 16
    t.owned[t.ids[:, full]] = 0
    keep = np.isin(t.reserve, t.ids[:, full])
    t.reserve, t.used = t.reserve[~keep], 0
    want, _ = _run(t, np.zeros((2, 4), dtype=np.int64))
    assert len(want["copies"]) == 8 and want["used"] == 8


def test_lengths_of_their_own_and_shared_last_pages():
    rng = np.random.default_rng(5)
    for seed in range(6):
        t = Tables(seed, G=3, W=6, P=16, context=64, grown=60, lens=rng.integers(0, 110, size=18), spare=60, ragged=False)
        _run(t, rng.integers(-1, 6, size=(3, 6)))
    t = Tables(9, G=1, W=4, P=16, context=0, grown=40, spare=20, lens=[20, 20, 32, 9], ragged=False)
    t.ids[:] = t.ids[0]                                            # one page in four lengths: full, partly filled, not reached
    held = set(t.ids[0, :2].tolist())
    t.owned[:] = 0
    t.owned[list(held)] = 1
    t.owned[t.reserve[-20:]] = 1
    t.reserve, t.used = np.array(sorted(held) + t.reserve[-20:].tolist()), 2
    for parent in ([0, 1, 2, 3], [2, 2, 0, 1], [3, 3, 3, -1], [0, 0, 1, 1]):
        _run(t, np.array([parent]))


def test_long_tables_and_many_groups():
    t = Tables(11, G=2, W=8, P=16, context=40000, grown=3000)       # several stretches of entries a group
    _run(t, t.rng.integers(0, 8, size=(2, 8)))
    t = Tables(12, G=900, W=3, P=16, context=20, grown=50)
    _run(t, t.rng.integers(-1, 3, size=(900, 3)))


def test_the_most_groups_there_may_be():
    t = Tables(21, G=M.MEPIC_STEP_MAX_BATCH, W=2, P=16, context=20, grown=20)
    _run(t, t.rng.integers(-1, 2, size=(M.MEPIC_STEP_MAX_BATCH, 2)))


def test_a_reserve_that_cannot_supply_the_copies():
    t = Tables(13, G=2, W=1, P=16, context=0, grown=40, spare=5, ragged=False)
    parent = np.zeros((2, 4), dtype=np.int64)
    want, _ = _run(t, parent)                                       # six copies, five pages
    assert want["status"] == M.MEPIC_DEV_NO_PAGES
    t = Tables(13, G=2, W=1, P=16, context=0, grown=40, spare=6, ragged=False)
    want, _ = _run(t, parent)
    assert want["used"] == len(t.reserve)


def test_no_reserve_at_all():
    t = Tables(22, G=2, W=2, P=16, context=64, grown=0, spare=0)       # whole pages of the store's: nothing to copy, nothing to give back
    assert t.reserve.size == 0
    _run(t, np.array([[1, 0], [0, 0]]))
    t.kv[:] = 60
    want, _ = _run(t, np.array([[1, 0], [0, 0]]))                      # a copy each
    assert want["status"] == M.MEPIC_DEV_NO_PAGES


def test_a_reserve_that_would_get_back_more_than_it_gave():
    t = Tables(14, G=2, W=4, P=16, context=30, grown=90)
    t.used = 1
    want, _ = _run(t, np.zeros((2, 4), dtype=np.int64))
    assert want["status"] == M.MEPIC_DEV_BAD_BEAM
    for used in (-1, len(t.reserve) + 1):
        t.used = used
        want, _ = _run(t, np.tile(np.arange(4), (2, 1)))
        assert want["status"] == M.MEPIC_DEV_BAD_BEAM


def test_parents_lengths_and_pages_that_are_none():
    t = Tables(15, G=2, W=4, P=16, context=30, grown=90)
    _run(t, np.array([[0, 4, -2, 1], [1 << 30, 2, 2, -1]]), M.MEPIC_DEV_BAD_BEAM)
    t.kv[0, 1], t.kv[1, 2] = -3, t.ids.shape[1] * 16 + 1
    op = t.call(np.array([[1, 0, 0, 2], [0, 1, 3, 3]]))
    got = op.run()
    torch.cuda.synchronize()
    assert t.dev.read_status() & M.MEPIC_DEV_BAD_SLOT and got["kv_len"][0].item() == 0
    t = Tables(16, G=2, W=4, P=16, context=30, grown=90)
    for bad in (-1, t.num_pages, 1 << 30):
        keep = t.ids[1, 1]
        t.ids[1, 1] = bad                                           # in a beam that is dropped, and in one that goes on
        for parent in ([[0, 2, 2, 3], [0, 1, 2, 3]], [[1, 1, 2, 3], [0, 1, 2, 3]]):
            op = t.call(np.array(parent))
            got = op.run()
            torch.cuda.synchronize()
            assert t.dev.read_status() & ~M.MEPIC_DEV_BAD_PAGE == 0
        t.ids[1, 1] = keep


def test_captured_and_replayed():
    t = Tables(17, G=3, W=4, P=16, context=30, grown=90)
    first = np.tile(np.arange(4), (3, 1))
    op = t.call(first)
    op.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = op.run()
    for _ in range(4):
        parent = t.rng.integers(-1, 4, size=(3, 4))
        t.d["parent"].copy_(dev32(parent)), t.d["page_ids_out"].fill_(-9), t.d["pos_base_out"].fill_(-9)
        t.d["reserve"].copy_(dev32(t.reserve))
        graph.replay()
        t.check(parent, op, got)


# ------------------------------------------------------------------ page copies
def _pools(cfg, seed, fp8):
    rng = np.random.default_rng(seed)
    shape = (cfg.num_pages, cfg.n_kv_heads, cfg.page_size, cfg.head_dim)
    if not fp8:
        dev = RT.Device(cfg, *(rng.integers(0, 1 << 16, size=shape).astype(np.uint16) for _ in range(2)))
        return dev, None, [dev.k_pool.view(torch.int16), dev.v_pool.view(torch.int16)]
    dev = RT.Device(cfg, bf16_pools=False)
    pools = RT.Fp8Pools(dev)
    for t in (pools.k_codes, pools.v_codes):
        t.copy_(torch.from_numpy(rng.integers(0, 256, size=shape).astype(np.uint8)))
    for t in (pools.k_scales, pools.v_scales):
        t.copy_(torch.from_numpy(rng.random(tuple(t.shape)).astype(np.float32)))
    return dev, pools, [pools.k_codes, pools.v_codes, pools.k_scales, pools.v_scales]


def _copied(tensors, src, dst, slots, n, num_pages):
    want = [t.clone() for t in tensors]
    for i in range(n):
        if not (0 <= src[i] < num_pages and 0 <= dst[i] < num_pages):
            continue
        for k, t in enumerate(tensors):
            if k < 2:
                want[k][dst[i], :, :slots[i]] = t[src[i], :, :slots[i]]
            else:
                want[k][dst[i]] = t[src[i]]
    return want


@pytest.mark.parametrize("Hkv,D,P,fp8", [(2, 128, 16, False), (8, 128, 64, False), (1, 64, 16, False), (3, 64, 128, False), (5, 128, 32, False),
                                         (2, 128, 16, True), (8, 128, 64, True), (1, 128, 128, True)])
def test_copies(Hkv, D, P, fp8):
    cfg = M.Config(P, Hkv, Hkv, D, 120, P, 1e4)
    rng = np.random.default_rng(Hkv + D + P)
    dev, pools, t = _pools(cfg, P, fp8)
    perm = rng.permutation(120)
    n = 50
    src, dst = perm[:20][rng.integers(0, 20, size=n)], perm[20:20 + n]
    slots = np.array([0, P, 1, P - 1, P + 7, -3] + rng.integers(0, P + 1, size=n - 6).tolist())
    for live, with_slots in ((n, True), (n - 9, True), (n, False), (0, True)):
        want = _copied(t, src, dst, np.clip(slots, 0, P) if with_slots else np.full(n, P), live, 120)
        op = RT.PagesCopy(dev, src=dev32(src), dst=dev32(dst), slots=dev32(slots) if with_slots else None, n_copies=None if live == n else dev32([live]), pools=pools)
        op.run()
        torch.cuda.synchronize()
        assert dev.read_status() == 0
        assert all(torch.equal(a, b) for a, b in zip(t, want))


@pytest.mark.parametrize("fp8", [False, True])
def test_copies_from_and_to_pages_that_are_none(fp8):
    cfg = M.Config(16, 2, 2, 128, 30, 16, 1e4)
    dev, pools, t = _pools(cfg, 1, fp8)
    src, dst = np.array([1, -1, 30, 2, 3, 1 << 30]), np.array([11, 12, 13, -5, 30, 14])
    want = _copied(t, src, dst, np.full(6, 16), 6, 30)
    RT.PagesCopy(dev, src=dev32(src), dst=dev32(dst), pools=pools).run()
    torch.cuda.synchronize()
    assert dev.read_status() == M.MEPIC_DEV_BAD_PAGE and all(torch.equal(a, b) for a, b in zip(t, want))
    for n in (7, -1):
        dev.status.zero_()
        want = _copied(t, src[:1], dst[:1], [16], 1 if n > 0 else 0, 30)
        RT.PagesCopy(dev, src=dev32(src[:1]), dst=dev32(dst[:1]), n_copies=dev32([n]), pools=pools).run()
        torch.cuda.synchronize()
        assert dev.read_status() == M.MEPIC_DEV_BAD_SLOT and all(torch.equal(a, b) for a, b in zip(t, want))


def test_no_copies_at_all():
    dev, pools, t = _pools(M.Config(16, 2, 2, 128, 30, 16, 1e4), 2, False)
    RT.PagesCopy(dev, src=dev32([]), dst=dev32([])).run()
    torch.cuda.synchronize()
    assert dev.read_status() == 0


def test_copies_past_32_bits_of_elements():
    pages = (1 << 32) // (8 * 16 * 128) + 40
    cfg = M.Config(16, 8, 8, 128, pages, 16, 1e4)
    dev = RT.Device(cfg)
    src, dst = [pages - 1, 3, pages - 2], [5, pages - 7, pages - 8]
    for p in src:
        dev.k_pool[p].normal_(), dev.v_pool[p].normal_()
    RT.PagesCopy(dev, src=dev32(src), dst=dev32(dst)).run()
    torch.cuda.synchronize()
    assert dev.read_status() == 0
    for s, d in zip(src, dst):
        assert torch.equal(dev.k_pool[s], dev.k_pool[d]) and torch.equal(dev.v_pool[s], dev.v_pool[d])
