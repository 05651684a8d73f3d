"""A search run as it would be: tables, commit, plan, attention, selection, fork and page copies step after step, all on the device,
against a host that keeps every beam's whole past as a list of rows."""
import numpy as np
import pytest
import torch

import paper_2512_16822_b200 as M
from paper_2512_16822_b200 import runtime as RT
from paper_2512_16822_b200.build import build_library
from mepic_inputs import f32_to_bf16_bits, bf16_bits_to_f64
from oracle import mepic_oracle as O
from beam_helpers import dev32, select_group

pytestmark = pytest.mark.gpu

Hq, Hkv, D, P, V = 8, 2, 128, 16, 500
EOS, PAD, SM = 3, 0, 0.09


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"


def _bits(rng, *shape):
    return f32_to_bf16_bits(rng.standard_normal(shape).astype(np.float32))


class Search:
    """Two layers (pools of their own) under one set of tables; tables go to and fro between two buffers."""

    def __init__(self, seed, prompts, width, fp8=False, spare=None, layers=2):
        rng = self.rng = np.random.default_rng(seed)
        self.G, self.W, self.R, self.fp8 = len(prompts), width, len(prompts) * width, fp8
        ents = [-(-n // P) for n in prompts]
        spare = 6 * self.R if spare is None else spare
        stride = max(ents) + 8
        self.num_pages = sum(ents) + spare
        perm = rng.permutation(self.num_pages)
        cfg = M.Config(P, Hq, Hkv, D, self.num_pages, 4096, 1e4)
        self.devs = [RT.Device(cfg, _bits(rng, self.num_pages, Hkv, P, D), _bits(rng, self.num_pages, Hkv, P, D)) for _ in range(layers)]
        self.dev = self.devs[0]
        self.pools = [RT.Fp8Pools(d) for d in self.devs] if fp8 else [None] * layers
        self.reserve0 = perm[sum(ents):]
        self.owned = np.zeros(self.num_pages, dtype=np.uint8)
        self.owned[self.reserve0] = 1
        first = np.full((self.G, stride), -1, dtype=np.int64)
        at = 0
        for g, n in enumerate(ents):
            first[g, :n] = perm[at:at + n]
            at += n
        base = np.tile(np.arange(stride) * P, (self.G, 1))
        # state of the search
        self.n_new, self.kv, self.used, self.reserve = dev32(np.ones(self.R)), dev32(np.zeros(self.R)), dev32([0]), dev32(self.reserve0)
        self.scores, self.done = torch.zeros((self.G, width), device="cuda:0"), dev32(np.zeros((self.G, width)))
        self.ids, self.base = ([dev32(np.full((self.R, stride), -1)) for _ in range(2)] for _ in range(2))
        d_owned = torch.from_numpy(self.owned).cuda()
        # the prompt's one row becomes `width` beams
        start = RT.BeamFork(self.dev, parent=dev32(np.zeros((self.G, width))), kv_len=dev32(prompts), page_ids=dev32(first), pos_base=dev32(base),
                            page_ids_out=self.ids[0], pos_base_out=self.base[0], owned=d_owned, reserve=self.reserve, reserve_used=self.used)
        r = start.run()
        self._copies(r)
        for c in self.copies[-1]:
            c.run()
        self.kv.copy_(r["kv_len"]), self.used.copy_(r["reserve_used"])
        torch.cuda.synchronize()
        # the calls of a step, for either direction of the tables
        self.kn, self.vn = ([torch.empty((self.R, Hkv, D), dtype=torch.bfloat16, device="cuda:0") for _ in range(layers)] for _ in range(2))
        self.q = torch.empty((self.R, Hq, D), dtype=torch.bfloat16, device="cuda:0")
        self.logits = torch.empty((self.R, V), dtype=torch.float32, device="cuda:0")
        self.q_pos, self.lens = dev32(np.zeros(self.R)), dev32(np.zeros(self.R))
        rows = dev32(np.arange(self.R)[:, None])
        self.calls = []
        for i in (0, 1):
            tables = RT.StepTables(self.dev, kv_len=self.kv, n_new=self.n_new, page_ids=self.ids[i], pos_base=self.base[i], reserve=self.reserve, reserve_used=self.used, max_rows=self.R)
            commits = [RT.RowsCommit(d, k_new=k, v_new=v, row_offsets=tables.row_offsets, slot_map=tables.slot_map, src_rows=rows, pools=p)
                       for d, k, v, p in zip(self.devs, self.kn, self.vn, self.pools)]
            plan = RT.BeamPlan(self.dev, page_ids=self.ids[i], pos_base=self.base[i], kv_len=tables.kv_len_out, width=width)
            attn = [RT.BeamBatch(d, q=self.q, q_pos=tables.q_pos, plan=plan, pools=p) for d, p in zip(self.devs, self.pools)]
            select = RT.BeamSelect(self.dev, logits=self.logits, scores=self.scores, done=self.done, eos_token=EOS, pad_token=PAD)
            fork = RT.BeamFork(self.dev, parent=select.parent, kv_len=tables.kv_len_out, page_ids=self.ids[i], pos_base=self.base[i], page_ids_out=self.ids[1 - i],
                               pos_base_out=self.base[1 - i], owned=d_owned, reserve=self.reserve, reserve_used=tables.reserve_used_out)
            self._copies(fork._result)
            self.calls.append((tables, commits, plan, attn, select, fork, self.copies[-1]))
        self.at = 0

    def _copies(self, r):
        if not hasattr(self, "copies"):
            self.copies = []
        self.copies.append([RT.PagesCopy(d, src=r["copy_src"], dst=r["copy_dst"], slots=r["copy_slots"], n_copies=r["n_copies"], pools=p)
                            for d, p in zip(self.devs, self.pools)])

    def feed(self, seed):
        """The step's inputs: rows of the newest tokens, queries, logits."""
        g = torch.Generator(device="cuda:0").manual_seed(seed)
        for t in self.kn + self.vn + [self.q]:
            t.copy_(torch.randn(t.shape, generator=g, device="cuda:0"))
        self.logits.copy_(torch.randn(self.logits.shape, generator=g, device="cuda:0") * 2)
        self.logits[:, EOS] += 4.0                                   # beams end now and then

    def first_half(self, i):
        tables, commits, plan, attn, select, fork, copies = self.calls[i]
        tables.run()
        for c in commits:
            c.run()
        plan.run()
        return [a.run(SM) for a in attn]

    def second_half(self, i):
        tables, commits, plan, attn, select, fork, copies = self.calls[i]
        r = select.run()
        f = fork.run()
        for c in copies:
            c.run()
        self.scores.copy_(r["score"]), self.done.copy_(r["done"]), self.n_new.copy_(r["n_new"].view(-1))
        self.kv.copy_(f["kv_len"]), self.used.copy_(f["reserve_used"])

    def state(self):
        return [t.clone() for t in (self.kv, self.used, self.reserve, self.scores, self.done, self.n_new, *self.ids, *self.base)] + \
               [t.clone() for d in self.devs for t in (d.k_pool, d.v_pool)]

    def rows_of(self, i, layer):
        """Every row's K and V out of the pages (bits, or codes and scales), by the tables of direction i and the present lengths."""
        ids, kv = self.ids[i].cpu().numpy(), self.kv.cpu().numpy()
        p = self.pools[layer]
        src = (self.devs[layer].k_pool.view(torch.int16), self.devs[layer].v_pool.view(torch.int16)) if p is None else (p.k_codes, p.v_codes)
        src = [t.cpu().numpy() for t in src]
        scales = [] if p is None else [p.k_scales.cpu().numpy(), p.v_scales.cpu().numpy()]
        out = []
        for r, n in enumerate(kv):
            page = ids[r, :-(-n // P)]
            take = [t[page].transpose(0, 2, 1, 3).reshape(-1, *t.shape[1:2], D)[:n] for t in src]
            out.append(take + [s[page] for s in scales])
        return out

    def check_pages(self, i):
        """Every page of the reserve is held by beams of one request or free, never both; a partly filled last page has one holder."""
        ids, kv = self.ids[i].cpu().numpy(), self.kv.cpu().numpy()
        free = self.reserve.cpu().numpy()[int(self.used):].tolist()
        held = [set() for _ in range(self.G)]
        last = []
        for r, n in enumerate(kv):
            pages = ids[r, :-(-n // P)].tolist()
            held[r // self.W] |= {p for p in pages if self.owned[p]}
            if n % P:
                last.append(pages[-1])
        everything = free + [p for h in held for p in h]
        assert sorted(everything) == sorted(self.reserve0.tolist())
        assert len(set(last)) == len(last) and all(self.owned[p] for p in last)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("prompts,width", [([37, 16, 1, 95], 4), ([70], 1), ([33, 64], 7)])
def test_a_search_step_by_step(prompts, width, fp8):
    s = Search(len(prompts) + width, prompts, width, fp8)
    assert s.dev.read_status() == 0
    s.check_pages(0)
    past = [s.rows_of(0, layer) for layer in range(2)]
    kv, done, scores = np.repeat(prompts, width), np.zeros((s.G, width), dtype=np.int64), np.zeros((s.G, width))
    n_new = np.ones(s.R, dtype=np.int64)
    for step in range(22):
        i = step % 2
        s.feed(1000 + step)
        outs = s.first_half(i)
        torch.cuda.synchronize()
        # lengths, and what the pages hold: the past of the beam and the row just committed
        kv = kv + n_new
        assert (s.calls[i][0].kv_len_out.cpu().numpy() == kv).all()
        s.kv.copy_(s.calls[i][0].kv_len_out)
        now = [s.rows_of(i, layer) for layer in range(2)]
        for layer in range(2):
            kn = s.kn[layer].view(torch.int16).cpu().numpy()
            for r in range(s.R):
                old = past[layer][r]
                if not fp8:
                    assert (now[layer][r][0][:len(old[0])] == old[0]).all() and (now[layer][r][1][:len(old[1])] == old[1]).all(), (step, r)
                    if n_new[r]:
                        assert (now[layer][r][0][-1] == kn[r]).all()
                elif len(old[0]) % P:
                    assert (now[layer][r][0][:len(old[0])] == old[0]).all()
        # attention of some rows
        got = [bf16_bits_to_f64(RT.bf16_bits(o)) for o in outs]
        q = RT.bf16_bits(s.q)
        none = np.zeros((1, Hkv, D))
        for r in sorted({0, s.R - 1, (step * 7) % s.R}):
            for layer in range(2):
                K, Vv = now[layer][r][:2]
                if fp8:
                    n = len(K)
                    ent = np.arange(n) // P
                    K, Vv = (O.e4m3_values()[c] * sc[ent][:, :, None] for c, sc in zip((K, Vv), now[layer][r][2:]))
                else:
                    K, Vv = bf16_bits_to_f64(K.view(np.uint16)), bf16_bits_to_f64(Vv.view(np.uint16))
                n = len(K)
                pool = lambda x: np.concatenate([x, np.zeros((-n % P,) + x.shape[1:])]).reshape(-1, P, Hkv, D).transpose(0, 2, 1, 3)
                ents = -(-n // P)
                want, sigma = O.tree_attention_one(q[r:r + 1], none, none, [n - 1], np.zeros((1, 1), dtype=bool), pool(K), pool(Vv), np.arange(ents), np.arange(ents) * P, n, SM, 1e4)
                assert (np.abs(got[layer][r] - want[0]) <= 7 * sigma[0] + 1e-4).all(), (step, r, layer)
        # selection
        s.second_half(i)
        torch.cuda.synchronize()
        assert s.dev.read_status() == 0 and s.devs[1].read_status() == 0
        x = s.logits.double().cpu().numpy().reshape(s.G, width, V)
        parent, token = s.calls[i][4].parent.cpu().numpy(), s.calls[i][4].token.cpu().numpy()
        new_scores = s.scores.double().cpu().numpy()
        for g in range(s.G):
            want, _ = select_group(x[g], scores[g], done[g], width, EOS, PAD)
            for k in range(min(len(want), width)):
                assert abs(new_scores[g, k] - want[k][0]) <= 5e-6 + abs(want[k][0]) * 2.0 ** -23
                if all(abs(want[k][0] - want[j][0]) > 2e-5 for j in (k - 1, k + 1) if 0 <= j < len(want)):
                    assert (parent[g, k], token[g, k]) == want[k][1:3]
        # the new beams' past is their parents'
        s.check_pages(1 - i)
        flat = (np.arange(s.G)[:, None] * width + parent).reshape(-1)
        after = [s.rows_of(1 - i, layer) for layer in range(2)]
        for layer in range(2):
            for r in range(s.R):
                if parent.reshape(-1)[r] < 0:
                    assert len(after[layer][r][0]) == 0
                    continue
                assert all((a == b).all() for a, b in zip(after[layer][r], now[layer][flat[r]])), (step, r)
        past = after
        kv, n_new = s.kv.cpu().numpy().astype(np.int64), s.n_new.cpu().numpy().astype(np.int64)
        done, scores = s.done.cpu().numpy(), new_scores
        assert (kv == np.where(parent.reshape(-1) >= 0, np.array([len(now[0][f][0]) for f in np.maximum(flat, 0)]), 0)).all()


def test_the_steps_captured_give_the_same_bits():
    eager, graph = Search(5, [37, 16, 95], 4), Search(5, [37, 16, 95], 4)
    for step in range(2):                                            # kernels loaded, and past the first step
        for s in (eager, graph):
            s.feed(step)
            s.first_half(step), s.second_half(step)
    torch.cuda.synchronize()
    captured = torch.cuda.CUDAGraph()
    kept = graph.state()
    with torch.cuda.graph(captured):
        graph.first_half(0), graph.second_half(0), graph.first_half(1), graph.second_half(1)
    assert all(torch.equal(a, b) for a, b in zip(graph.state(), kept))
    for rounds in range(8):
        # the same inputs in both steps of a replay
        for s in (eager, graph):
            s.feed(50 + rounds)
        for i in (0, 1):
            eager.first_half(i), eager.second_half(i)
        captured.replay()
        torch.cuda.synchronize()
        assert eager.dev.read_status() == 0 and graph.dev.read_status() == 0
        assert all(torch.equal(a, b) for a, b in zip(eager.state(), graph.state())), rounds
    eager.check_pages(0)


def test_a_search_that_runs_out_of_pages_stops_without_harm():
    s = Search(9, [33, 64], 4, spare=8 + 3)
    for step in range(40):
        s.feed(step)
        s.logits[:, EOS] -= 40.0
        s.first_half(step % 2)
        s.second_half(step % 2)
        torch.cuda.synchronize()
        if s.dev.read_status():
            break
    assert s.dev.read_status() == M.MEPIC_DEV_NO_PAGES
