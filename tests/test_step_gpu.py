"""The integer calls of a step with drafted tokens, the commit of rows, and a whole step in a run, against the oracle."""
import numpy as np
import pytest
import torch

import paper_2512_16822_b200 as M
from paper_2512_16822_b200 import runtime as RT
from paper_2512_16822_b200.build import build_library
from mepic_inputs import bf16_bits_to_f64, f32_to_bf16_bits
from oracle import mepic_oracle as O
from tree_helpers import TreeCase, dev32, random_parents

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"


def _dev(P=16, num_pages=4000, D=128, Hkv=2, pools=False):
    cfg = M.Config(P, Hkv, Hkv, D, num_pages, 4 * P, 1e4)
    return RT.Device.over(cfg) if not pools else RT.Device(cfg)


def _host(t):
    return t.cpu().numpy()


# ------------------------------------------------------------------------------------ layout
@pytest.mark.parametrize("kind", ["tree", "chain", "star"])
@pytest.mark.parametrize("counts,words", [([1], 1), ([8, 0, 31], 1), ([32, 33, 64, 65, 1], 3), ([1024, 1000, 0, 3], 32), ([0, 0, 2], 2)])
def test_layout(kind, counts, words):
    rng = np.random.default_rng(sum(counts) + words)
    P, stride = 32, 9
    parents = [random_parents(rng, n, kind) for n in counts]
    kv = rng.integers(0, P * stride + 1, size=len(counts))
    kv[0] = P * stride
    base = rng.integers(0, 10000, size=(len(counts), stride))
    off = np.concatenate([[0], np.cumsum(counts)])
    dev = _dev(P)
    lay = RT.TreeLayout(dev, parent=dev32(np.concatenate(parents)), row_offsets=dev32(off), kv_len=dev32(kv), pos_base=dev32(base), mask_words=words)
    lay.row_pos.fill_(-99), lay.tree_mask.fill_(-99)
    r = lay.run()
    torch.cuda.synchronize()
    assert dev.read_status() == 0
    for b, p in enumerate(parents):
        nxt = int(base[b, (kv[b] - 1) // P]) + (kv[b] - 1) % P + 1 if kv[b] else 0
        pos, sees = O.tree_layout(p, nxt)
        assert np.array_equal(_host(r["row_pos"])[off[b]:off[b + 1]], pos), b
        assert np.array_equal(_host(r["tree_mask"])[off[b]:off[b + 1]], O.pack_mask(sees, words)), b


def test_layout_of_the_largest_tree_captured_and_replayed():
    n, dev = 1024, _dev()
    parents, lens = dev32(np.full(n, -1)), dev32([7])
    lay = RT.TreeLayout(dev, parent=parents, row_offsets=dev32([0, n]), kv_len=lens, pos_base=dev32([[100]]), mask_words=32)
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        lay.run()
    for p, kv in ((np.arange(n) - 1, 9), (np.full(n, -1), 0), (random_parents(np.random.default_rng(2), n), 16)):
        parents.copy_(dev32(p)), lens.fill_(kv)
        g.replay()
        torch.cuda.synchronize()
        pos, sees = O.tree_layout(p, 100 + kv if kv else 0)
        assert dev.read_status() == 0
        assert lay.row_pos.tolist() == list(pos) and np.array_equal(_host(lay.tree_mask), O.pack_mask(sees, 32))


def test_layout_reports_what_makes_no_sense():
    base = dev32(np.zeros((1, 4)))
    def status(parent, off, kv=5, words=1):
        dev = _dev()
        lay = RT.TreeLayout(dev, parent=dev32(parent), row_offsets=dev32(off), kv_len=dev32([kv]), pos_base=base, mask_words=words)
        lay.row_pos.fill_(-99), lay.tree_mask.fill_(-99)
        r = lay.run()
        torch.cuda.synchronize()
        return dev.read_status(), _host(r["row_pos"]).tolist(), _host(r["tree_mask"]).tolist()
    assert status([-1, 1, 0], [0, 3]) == (M.MEPIC_DEV_BAD_TREE, [5, 5, 6], [[1], [2], [5]])
    assert status([-1, 2, -2], [0, 3])[0] == M.MEPIC_DEV_BAD_TREE
    assert status([-1, 0], [0, 7])[0] == M.MEPIC_DEV_BAD_TREE
    assert status([-1, 0], [1, 0])[0] == M.MEPIC_DEV_BAD_TREE
    assert status([-1, 0], [0, 2], kv=65)[0] == M.MEPIC_DEV_BAD_SLOT
    assert status([-1, 0], [0, 2], kv=-1) == (M.MEPIC_DEV_BAD_SLOT, [0, 1], [[1], [3]])
    code, pos, mask = status(list(range(-1, 33)), [0, 34])
    assert code == M.MEPIC_DEV_BAD_TREE and pos[31:] == [36, 5, 5] and mask[31:] == [[-1], [0], [0]]
    assert status([-1, 0, 0], [0, 2])[1:] == ([5, 6, -99], [[1], [3], [-99]])       # a row nobody owns stays as it was


# ------------------------------------------------------------------------------------ acceptance
@pytest.mark.parametrize("counts,max_accept", [([1], 1), ([8, 0, 31], 4), ([200, 33, 64, 1024], 16), ([60], 1), ([1024], 1024), ([5, 5], 2000)])
@pytest.mark.parametrize("kind", ["tree", "chain"])
def test_accept(counts, max_accept, kind):
    rng = np.random.default_rng(sum(counts) + max_accept)
    off = np.concatenate([[0], np.cumsum(counts)])
    parents = [random_parents(rng, n, kind) for n in counts]
    vocab = 3 if kind == "tree" else 1                              # few tokens: many siblings fit, long paths
    target, draft = rng.integers(0, vocab, size=off[-1]), rng.integers(0, vocab, size=off[-1])
    root = rng.integers(0, vocab, size=len(counts))
    dev = _dev()
    acc = RT.TreeAccept(dev, parent=dev32(np.concatenate(parents)), row_offsets=dev32(off), draft=dev32(draft), target=dev32(target),
                        root=dev32(root), max_accept=max_accept)
    r = {k: _host(v) for k, v in acc.run().items()}
    assert dev.read_status() == 0
    for b, p in enumerate(parents):
        s = slice(off[b], off[b + 1])
        path, nxt = O.tree_accept(p, draft[s], target[s], root[b], max_accept)
        assert r["n_accept"][b] == len(path) and r["next_token"][b] == nxt
        assert r["accept_rows"][b].tolist() == [off[b] + i for i in path] + [-1] * (max_accept - len(path))


def test_accept_reports_what_makes_no_sense():
    dev = _dev()
    acc = RT.TreeAccept(dev, parent=dev32([-1, 1, 0]), row_offsets=dev32([0, 3]), draft=dev32([4, 4, 4]), target=dev32([4, 4, 9]), root=dev32([4]), max_accept=5)
    r = acc.run()
    torch.cuda.synchronize()
    assert dev.read_status() == M.MEPIC_DEV_BAD_TREE
    assert _host(r["accept_rows"]).tolist() == [[0, 2, -1, -1, -1]] and r["next_token"].item() == 9
    n = 1030
    dev = _dev()
    acc = RT.TreeAccept(dev, parent=dev32(np.arange(n) - 1), row_offsets=dev32([0, n]), draft=dev32(np.zeros(n)), target=dev32(np.zeros(n)), root=dev32([0]), max_accept=2000)
    assert acc.run()["n_accept"].item() == 1024 and dev.read_status() == M.MEPIC_DEV_BAD_TREE


# ------------------------------------------------------------------------------------ tables
def _tables(dev, kv, new, ids, base, reserve, used, max_rows, check=True):
    P = dev.cfg.page_size
    d_ids, d_base = dev32(ids), dev32(base)
    st = RT.StepTables(dev, kv_len=dev32(kv), n_new=dev32(new), page_ids=d_ids, pos_base=d_base, reserve=dev32(reserve), reserve_used=dev32([used]), max_rows=max_rows)
    r = {k: _host(v) for k, v in st.run().items()}
    r["page_ids"], r["pos_base"] = _host(d_ids), _host(d_base)
    if check:
        want = O.step_tables(list(kv), list(new), np.asarray(ids), np.asarray(base), list(reserve), used, P, max_rows)
        for k, v in r.items():
            assert np.array_equal(v.reshape(-1), np.asarray(want[k]).reshape(-1)), k
    return r


@pytest.mark.parametrize("B,P,longest,most", [(1, 16, 40, 1), (3, 16, 100, 70), (32, 64, 900, 5), (33, 16, 900, 300), (513, 32, 200, 3), (8192, 16, 60, 2), (7, 16, 3, 2000)])
def test_tables(B, P, longest, most):
    rng = np.random.default_rng(B + P)
    kv, new = rng.integers(0, longest + 1, size=B), rng.integers(0, most + 1, size=B)
    stride = -(-(longest + most) // P) + 1
    ids, base = rng.integers(0, 4000, size=(B, stride)), rng.integers(0, 1000, size=(B, stride))
    grow = int((-(-(kv + new) // P) - -(-kv // P)).sum())
    dev = _dev(P, 4000)
    _tables(dev, kv, new, ids, base, rng.integers(0, 4000, size=grow + 3), 3, int(new.sum()) + int(rng.integers(0, 20)))
    assert dev.read_status() == 0


def test_tables_hand_out_all_or_nothing():
    ids, base = np.zeros((2, 4), dtype=int), np.zeros((2, 4), dtype=int)
    for kv, new, reserve, used, max_rows in (([10, 16], [7, 1], [5, 6], 1, 8), ([10, 16], [7, 1], [5, 6], 0, 7), ([10, 64], [7, 1], [5, 6], 0, 8),
                                             ([10, 16], [-1, 1], [5, 6], 0, 8), ([-1, 16], [0, 1], [5, 6], 0, 8), ([10, 16], [7, 1], [5, 6], -1, 8),
                                             ([10, 16], [2 ** 31 - 1, 2 ** 31 - 1], [5, 6], 0, 8)):
        dev = _dev()
        r = _tables(dev, kv, new, ids, base, reserve, used, max_rows, check=False)
        assert dev.read_status() == M.MEPIC_DEV_NO_PAGES
        assert r["row_offsets"].tolist() == [0, 0, 0] and r["kv_len"].tolist() == list(kv) and r["reserve_used"].item() == used
        assert (r["row_slot"] == -1).all() and (r["slot_map"] == -1).all() and not r["page_ids"].any() and not r["pos_base"].any()
    dev = _dev(num_pages=6)
    r = _tables(dev, [10, 16], [7, 1], ids, base, [5, 6], 0, 8, check=False)
    assert dev.read_status() == M.MEPIC_DEV_BAD_PAGE
    assert r["slot_map"].tolist() == [10, 11, 12, 13, 14, 15, 80, -1]


def test_tables_of_a_wide_pool_pass_32_bits():
    # physical slots beyond 2^31: page ids near 2^31 / 16 and above
    dev = RT.Device.over(M.Config(64, 1, 1, 64, 2 ** 31 - 1, 64, 1e4))
    r = _tables(dev, [60], [8], np.array([[2 ** 30, 0]]), np.array([[0, 0]]), [2 ** 31 - 2], 0, 8, check=False)
    assert dev.read_status() == 0
    assert r["slot_map"].tolist() == [2 ** 36 + 60 + i for i in range(4)] + [(2 ** 31 - 2) * 64 + i for i in range(4)]


# ------------------------------------------------------------------------------------ commit
def test_tables_of_lengths_at_the_end_of_32_bits():
    # table rows longer than an int32 length can name: what ends beyond 2^31 - 1 is refused, what ends there is not
    P, stride = 1 << 16, 32769
    dev = RT.Device.over(M.Config(P, 1, 1, 64, 4, P - 1, 1e4))
    top = 2 ** 31 - 1
    for kv, new, fits in ((top - 300, 1000, False), (top, 1, False), (top - 5, 5, True), (top, 0, True), (top - P, 3, True)):
        ids, base = np.zeros((1, stride), dtype=int), np.zeros((1, stride), dtype=int)
        r = _tables(dev, [kv], [new], ids, base, [1, 2], 0, 1000, check=False)
        assert dev.read_status() == (0 if fits else M.MEPIC_DEV_NO_PAGES)
        dev.status.zero_()
        assert r["kv_len"].item() == kv + (new if fits else 0) and r["row_offsets"].tolist() == [0, new if fits else 0]
        old, all_ = -(-kv // P), -(-(kv + new) // P)
        assert r["reserve_used"].item() == (all_ - old if fits else 0)
        if fits:
            assert r["row_slot"][:new].tolist() == list(range(kv, kv + new))
            page = [int(r["page_ids"][0, s // P]) for s in range(kv, kv + new)]
            assert r["slot_map"][:new].tolist() == [g * P + s % P for g, s in zip(page, range(kv, kv + new))]


def test_layouts_and_tables_of_two_sizes_at_once():
    # two host threads whose calls need different amounts of shared memory
    import threading
    rng, dev, failed = np.random.default_rng(9), _dev(16, 64), []

    def work(words, batch):
        try:
            n = 32 * words
            parents = np.arange(n, dtype=np.int32) - 1
            lay = RT.TreeLayout(dev, parent=dev32(parents), row_offsets=dev32([0, n]), kv_len=dev32([3]), pos_base=dev32([[0]]), mask_words=words)
            tab = RT.StepTables(dev, kv_len=dev32(np.full(batch, 3)), n_new=dev32(np.ones(batch)), page_ids=dev32(np.ones((batch, 1))),
                                pos_base=dev32(np.zeros((batch, 1))), reserve=dev32([0]), reserve_used=dev32([0]), max_rows=batch)
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.default_stream())
            for _ in range(200):
                lay.run(s)
                tab.run(s)
            s.synchronize()
            assert lay.row_pos.tolist() == list(range(3, 3 + n)) and tab.slot_map.tolist() == [19] * batch
        except Exception as e:                       # shown by the test's thread
            failed.append(e)

    threads = [threading.Thread(target=work, args=w) for w in ((32, 8192), (20, 5500), (1, 7))]
    [t.start() for t in threads], [t.join() for t in threads]
    assert not failed and dev.read_status() == 0


@pytest.mark.parametrize("D,P,Hkv", [(128, 16, 8), (64, 16, 1), (128, 64, 3)])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("fp8", [False, True])
def test_commit(D, P, Hkv, gather, fp8):
    if fp8 and D != 128:
        pytest.skip("8-bit pages have head_dim 128")
    rng = np.random.default_rng(D + P + Hkv)
    counts = [5, 0, 3 * P + 2, 1, P, 40, 0]
    B, off = len(counts), np.concatenate([[0], np.cumsum(counts)])
    total, num_pages = int(off[-1]), 60
    kp, vp = (f32_to_bf16_bits(rng.standard_normal((num_pages, Hkv, P, D)).astype(np.float32)) for _ in range(2))
    perm, at = rng.permutation(num_pages), 0
    slots, tables = [], []
    for b, n in enumerate(counts):
        start = 0 if b in (4, 3) else int(rng.integers(0, P))
        pages = perm[at:at + -(-(start + n) // P) + 1]
        at += len(pages)
        tables.append((pages, start + np.arange(n)))
        slots += [int(pages[t // P]) * P + int(t) % P for t in range(start, start + n)]
    sources = total if not gather else 3 * total
    k, v = (f32_to_bf16_bits((rng.standard_normal((sources, Hkv, D)) * 3).astype(np.float32)) for _ in range(2))
    k[0, 0, 0], v[0, 0, 1] = 0x7fc0, 0x8000
    src = [np.sort(rng.choice(np.arange(3 * off[b], 3 * off[b + 1]), size=n, replace=False)) if gather else np.arange(off[b], off[b + 1]) for b, n in enumerate(counts)]
    dev = RT.Device(M.Config(P, Hkv, Hkv, D, num_pages, P, 1e4), kp, vp)
    pools = RT.Fp8Pools(dev) if fp8 else None
    buf = torch.full((sources, 2 * Hkv * D + 8), float("nan"), dtype=torch.bfloat16, device=DEV)
    buf[:, :Hkv * D], buf[:, Hkv * D:2 * Hkv * D] = RT.bf16_tensor(k, DEV).view(sources, -1), RT.bf16_tensor(v, DEV).view(sources, -1)
    d_src = None
    if gather:
        d_src = np.full((B, max(counts) + 1), -1)
        for b, s in enumerate(src):
            d_src[b, :len(s)] = s
        d_src = dev32(d_src)
    slot_map = torch.tensor(slots + [-1] * 4, dtype=torch.int64, device=DEV)
    if fp8:
        codes = [O.quantize_pages(x) for x in (kp, vp)]
        (kc, ks), (vc, vs) = codes
        assert np.array_equal(_host(pools.k_codes), kc) and np.array_equal(_host(pools.v_scales), vs)
    RT.RowsCommit(dev, k_new=buf[:, :Hkv * D].unflatten(1, (Hkv, D)), v_new=buf[:, Hkv * D:2 * Hkv * D].unflatten(1, (Hkv, D)),
                  row_offsets=dev32(off), slot_map=slot_map, src_rows=d_src, pools=pools).run()
    torch.cuda.synchronize()
    assert dev.read_status() == 0
    for b, (pages, t) in enumerate(tables):
        if not len(t):
            continue
        if fp8:
            O.commit_rows_fp8(kc, ks, vc, vs, list(pages), list(t), k[src[b]], v[src[b]])
        else:
            O.commit_rows(kp, vp, list(pages), list(t), k[src[b]], v[src[b]])
    if fp8:
        assert np.array_equal(_host(pools.k_scales), ks) and np.array_equal(_host(pools.v_scales), vs)
        assert np.array_equal(_host(pools.k_codes), kc) and np.array_equal(_host(pools.v_codes), vc)
    else:
        assert np.array_equal(RT.bf16_bits(dev.k_pool), kp) and np.array_equal(RT.bf16_bits(dev.v_pool), vp)


@pytest.mark.parametrize("P", [16, 32])
def test_commit_of_extreme_values_into_8_bit_pages(P):
    # a page per magnitude, started (its scale from its rows) or appended to under a scale that stands, from subnormal to infinite
    rng, Hkv, D = np.random.default_rng(P), 2, 128
    exps = [-132, -120, -100, -88, -80, -72, -71, -40, 0, 40, 88, 89, 90, 110, 119]
    standing = np.array([0.0, 1e-44, 2.0 ** -127, 2.0 ** -100, 2.0 ** -81, 2.0 ** -80, 2.0 ** -79, 2.0 ** -3, 2.0 ** 79, 2.0 ** 80, 2.0 ** 81, 2.0 ** 120, 3e38, np.inf, 0.37],
                        dtype=np.float32)
    n_pages = 2 * len(exps) + 3
    rows, slots, off, src = [], [], [0], []
    def add(page, first, x):
        rows.append(x), slots.extend(page * P + first + i for i in range(len(x))), off.append(off[-1] + len(x))
        src.append((page, first))
    normal = lambda n: rng.standard_normal((n, 2, Hkv, D)).astype(np.float32)
    with np.errstate(over="ignore", under="ignore"):
        for i, e in enumerate(exps):
            add(i, 0, (normal(P).astype(np.float64) * 2.0 ** e).astype(np.float32))
            x = normal(7)
            x[..., ::2] *= np.float32(standing[i]) if np.isfinite(standing[i]) else np.float32(1)       # in the scale's range, and far from it
            x[0, :, :, :4] = [np.inf, -np.inf, np.nan, -0.0]
            add(len(exps) + i, 5, x)
    at = 2 * len(exps)
    x = normal(P); x[3, 0, 0, 5] = np.inf; x[4, 1, 1, 7] = -np.inf
    add(at, 0, x)
    x = normal(P); x[:, :, 1] = -0.0; x[2, 0, 0, 0] = np.nan; x[:, 1, 0] = np.nan
    add(at + 1, 0, x)
    add(at + 2, 0, np.full((1, 2, Hkv, D), 3.3895e38, dtype=np.float32))
    kv = f32_to_bf16_bits(np.concatenate(rows))
    kv[0, 0, 0, :3] = 0x0001, 0x8001, 0x7f
    dev = RT.Device(M.Config(P, Hkv, Hkv, D, n_pages, P, 1e4))
    dev.k_pool.zero_(), dev.v_pool.zero_()
    pools = RT.Fp8Pools(dev)
    for s in (pools.k_scales, pools.v_scales):
        s[len(exps):2 * len(exps)] = torch.from_numpy(standing).cuda()[:, None]
    kc, vc, ks, vs = (_host(t).copy() for t in (pools.k_codes, pools.v_codes, pools.k_scales, pools.v_scales))
    k, v = (RT.bf16_tensor(np.ascontiguousarray(kv[:, w]), DEV) for w in range(2))
    RT.RowsCommit(dev, k_new=k, v_new=v, row_offsets=dev32(off), slot_map=torch.tensor(slots, dtype=torch.int64, device=DEV), pools=pools).run()
    torch.cuda.synchronize()
    assert dev.read_status() == 0
    with np.errstate(all="ignore"):
        for i, (page, first) in enumerate(src):
            part = kv[off[i]:off[i + 1]]
            O.commit_rows_fp8(kc, ks, vc, vs, [page], list(first + np.arange(len(part))), part[:, 0], part[:, 1])
    assert np.array_equal(_host(pools.k_scales), ks, equal_nan=True) and np.array_equal(_host(pools.v_scales), vs, equal_nan=True)
    assert np.array_equal(_host(pools.k_codes), kc) and np.array_equal(_host(pools.v_codes), vc)


@pytest.mark.parametrize("fp8", [False, True])
def test_commit_reports_and_skips(fp8):
    dev = _dev(num_pages=4, pools=True)
    dev.k_pool.zero_(), dev.v_pool.zero_()
    pools = RT.Fp8Pools(dev) if fp8 else None
    rows = torch.ones((4, 2, 128), dtype=torch.bfloat16, device=DEV)
    def status(off, slots, src=None):
        dev.status.zero_()
        RT.RowsCommit(dev, k_new=rows, v_new=rows, row_offsets=dev32(off), slot_map=torch.tensor(slots, dtype=torch.int64, device=DEV),
                      src_rows=None if src is None else dev32(src), pools=pools).run()
        torch.cuda.synchronize()
        return dev.read_status()
    pool = lambda: (pools.k_codes if fp8 else dev.k_pool).float().abs().amax(dim=(1, 3)).bool()           # [page, slot]
    assert status([0, 3], [3, 64, -1]) == M.MEPIC_DEV_BAD_PAGE
    assert pool().nonzero().tolist() == [[0, 3]]
    assert status([0, 2], [17, 18], [[4, 1]]) == M.MEPIC_DEV_BAD_SLOT
    assert pool().nonzero().tolist() == [[0, 3], [1, 2]]
    assert status([0, 2], [19, 20], [[0]]) == M.MEPIC_DEV_BAD_SLOT
    assert status([0, 3], [35, 36]) == M.MEPIC_DEV_BAD_SLOT
    assert status([0, 2], [50, 51], [[-1, 0]]) == M.MEPIC_DEV_BAD_SLOT
    assert pool().nonzero().tolist() == [[0, 3], [1, 2], [1, 3], [2, 3], [2, 4], [3, 3]]
    assert status([0, 0], [50, 51]) == 0


# ------------------------------------------------------------------------------------ a whole step, in a run
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("graph", [False, True])
def test_steps_in_a_run(fp8, graph):
    """layout -> attention -> acceptance -> tables -> commit, three steps over the same buffers: the pools, lengths and outputs
    of every step against the oracle stepping alongside.  Tables start from the store's; captured: one graph, replayed."""
    Hq, Hkv, D, P, B, T, A = 8, 2, 128, 16, 3, 11, 4
    rng = np.random.default_rng(50)
    cfg = M.Config(P, Hq, Hkv, D, 64, 400, 1e4)
    with M.Store(cfg) as st:
        chunk = st.chunk_register(rng.integers(1, 1000, size=48))[0]
        tabs = []
        for b, tail in enumerate((30, 1, 64)):
            tabs.append(st.build_block_table(b, [M.Segment(M.MEPIC_SEG_CHUNK, chunk), M.Segment(M.MEPIC_SEG_PROMPT, tail)]))
        reserve = st.build_block_table(99, [M.Segment(M.MEPIC_SEG_PROMPT, 10 * P)])[0]
    stride = 12
    ids, base = np.full((B, stride), -1, dtype=np.int32), np.zeros((B, stride), dtype=np.int32)
    kv = np.array([t[2] for t in tabs], dtype=np.int64)
    for b, t in enumerate(tabs):
        ids[b, :len(t[0])], base[b, :len(t[1])] = t[0], t[1]
    bits = lambda shape: f32_to_bf16_bits(rng.standard_normal(shape).astype(np.float32))
    kp, vp = bits((64, Hkv, P, D)), bits((64, Hkv, P, D))
    dev = RT.Device(cfg, kp, vp)
    pools = RT.Fp8Pools(dev) if fp8 else None
    counts = [T, 6, 1]
    off = np.concatenate([[0], np.cumsum(counts)])
    total = int(off[-1])
    # the step's buffers
    d = dict(parent=dev32(np.full(total, -1)), draft=dev32(np.zeros(total)), target=dev32(np.zeros(total)), root=dev32(np.zeros(B)), off=dev32(off),
             kv=dev32(kv), ids=dev32(ids), base=dev32(base), used=dev32([0]), reserve=dev32(reserve))
    q, k, v = (torch.zeros((total, h, D), dtype=torch.bfloat16, device=DEV) for h in (Hq, Hkv, Hkv))
    lay = RT.TreeLayout(dev, parent=d["parent"], row_offsets=d["off"], kv_len=d["kv"], pos_base=d["base"], mask_words=1)
    att = RT.TreeBatch(dev, q=q, k_new=k, v_new=v, row_offsets=d["off"], row_pos=lay.row_pos, tree_mask=lay.tree_mask, page_ids=d["ids"],
                       pos_base=d["base"], kv_len=d["kv"], max_rows=T, pools=pools)
    acc = RT.TreeAccept(dev, parent=d["parent"], row_offsets=d["off"], draft=d["draft"], target=d["target"], root=d["root"], max_accept=A)
    tab = RT.StepTables(dev, kv_len=d["kv"], n_new=acc.n_accept, page_ids=d["ids"], pos_base=d["base"], reserve=d["reserve"], reserve_used=d["used"], max_rows=B * A)
    com = RT.RowsCommit(dev, k_new=k, v_new=v, row_offsets=tab.row_offsets, slot_map=tab.slot_map, src_rows=acc.accept_rows, pools=pools)

    def step():
        lay.run(), att.run(0.09), acc.run(), tab.run(), com.run()
        tab.advance()
        d["root"].copy_(acc.next_token)

    if fp8:
        (kc, ks), (vc, vs) = O.quantize_pages(kp), O.quantize_pages(vp)
    saved = [t.clone() for t in d.values()] + ([t.clone() for t in (pools.k_codes, pools.v_codes, pools.k_scales, pools.v_scales)] if fp8 else [dev.k_pool.clone(), dev.v_pool.clone()])
    live = list(d.values()) + ([pools.k_codes, pools.v_codes, pools.k_scales, pools.v_scales] if fp8 else [dev.k_pool, dev.v_pool])
    if graph:
        step()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step()
        for t, s in zip(live, saved):
            t.copy_(s)
    used, root = 0, np.zeros(B, dtype=np.int64)
    grew = 0
    for it in range(3):
        parents = [random_parents(rng, n) for n in counts]
        draft, target = rng.integers(0, 2, size=total), rng.integers(0, 2, size=total)
        qn, kn, vn = bits((total, Hq, D)), bits((total, Hkv, D)), bits((total, Hkv, D))
        for t, a in ((d["parent"], np.concatenate(parents)), (d["draft"], draft), (d["target"], target)):
            t.copy_(dev32(a))
        for t, a in ((q, qn), (k, kn), (v, vn)):
            t.copy_(RT.bf16_tensor(a, DEV))
        g.replay() if graph else step()
        torch.cuda.synchronize()
        assert dev.read_status() == 0
        got = bf16_bits_to_f64(RT.bf16_bits(att.out))
        dk, dv = (kp, vp) if not fp8 else (O.dequantize_pages(kc, ks), O.dequantize_pages(vc, vs))
        paths = []
        for b in range(B):
            r = slice(off[b], off[b + 1])
            n = int(kv[b])
            pos, sees = O.tree_layout(parents[b], int(base[b, (n - 1) // P]) + (n - 1) % P + 1)
            want, sigma = O.tree_attention_one(qn[r], kn[r], vn[r], pos, sees, dk, dv, ids[b], base[b], n, 0.09, 1e4)
            assert (np.abs(got[r] - want) <= 7 * sigma + 1e-4).all(), (it, b)
            path, nxt = O.tree_accept(parents[b], draft[r], target[r], root[b], A)
            paths.append([int(off[b]) + i for i in path])
            root[b] = nxt
        w = O.step_tables(list(kv), [len(p) for p in paths], ids, base, list(reserve), used, P, B * A)
        grew += w["reserve_used"] - used
        ids, base, used = w["page_ids"], w["pos_base"], w["reserve_used"]
        for b, path in enumerate(paths):
            t = list(range(int(kv[b]), int(kv[b]) + len(path)))
            if not path:
                continue
            if fp8:
                O.commit_rows_fp8(kc, ks, vc, vs, list(ids[b]), t, kn[path], vn[path])
            else:
                O.commit_rows(kp, vp, list(ids[b]), t, kn[path], vn[path])
        kv = w["kv_len"]
        assert np.array_equal(_host(d["kv"]), kv) and np.array_equal(_host(d["root"]), root) and np.array_equal(_host(d["ids"]), ids)
        if fp8:
            assert np.array_equal(_host(pools.k_codes), kc) and np.array_equal(_host(pools.v_codes), vc)
            assert np.array_equal(_host(pools.k_scales), ks) and np.array_equal(_host(pools.v_scales), vs)
        else:
            assert np.array_equal(RT.bf16_bits(dev.k_pool), kp) and np.array_equal(RT.bf16_bits(dev.v_pool), vp)
    assert grew >= 1, "the run is meant to pass a page boundary"
