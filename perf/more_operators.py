"""Measured cases of the beam-search operators: one step of a decode with beams over the page pool.

A request is decoded by a few beams that share its context's pages and, beyond it, the pages of the ancestors they have in
common.  The operators, in the order a step uses them:

* attn_beam   - attention of every beam's newest token over its un-rotated paged context, bf16 or 8-bit (e4m3) pages: the plan of
                which beams share which page (made from the block tables) and the attention that reads each page once,
* beam_select - the model's logits and the beams' scores -> the best continuations over beams and vocabulary,
* beam_fork   - parents -> block tables of the new beams, pages to copy on write, pages returned to the reserve,
* pages_copy  - those copies, bf16 or 8-bit pages.

``run`` computes the plain form (torch) unless ``own`` is set, and then makes the calls of the package.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
E4M3_MAX = 448.0


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one user's request, early in its answer: only latency counts
        dict(name="attn one request", op="attn_beam", fp8=False, groups=1, width=4, context=203, grown=21, q_heads=8, kv_heads=2,
             head_dim=64, page=16),
        # a full serving batch of RAG prompts (16 chunks of 512 tokens and a question), four beams each
        dict(name="attn serving batch", op="attn_beam", fp8=False, groups=32, width=4, context=8256, grown=75, q_heads=32, kv_heads=8,
             head_dim=128, page=16),
        # eight beams over long prompts, with long answers behind them: many pages that only some of the beams share
        dict(name="attn wide beams", op="attn_beam", fp8=False, groups=8, width=8, context=16640, grown=700, q_heads=32, kv_heads=8,
             head_dim=128, page=16),
        # five query heads a kv head and five beams: ragged columns, odd lengths
        dict(name="attn odd heads", op="attn_beam", fp8=False, groups=7, width=5, context=2049, grown=130, q_heads=40, kv_heads=8,
             head_dim=128, page=32),
        # very long prompts in 8-bit pages, 64-token pages
        dict(name="attn long fp8", op="attn_beam", fp8=True, groups=8, width=4, context=32768, grown=200, q_heads=32, kv_heads=8,
             head_dim=128, page=64),
        # the choice of one request's beams, and of a full batch with twice as many candidates as beams over a large vocabulary
        dict(name="select one request", op="beam_select", groups=1, width=4, select=4, vocab=32000, dtype="bf16"),
        dict(name="select batch", op="beam_select", groups=64, width=8, select=16, vocab=100003, dtype="fp32"),
        # the tables of one request, and of a full batch over long prompts
        dict(name="fork one request", op="beam_fork", groups=1, width=4, context=203, grown=21, page=16),
        dict(name="fork batch", op="beam_fork", groups=64, width=8, context=16640, grown=300, page=16),
        # the copies of one request's fork, of a batch's, and of a batch over large 8-bit pages
        dict(name="copy one request", op="pages_copy", fp8=False, copies=3, kv_heads=8, head_dim=128, page=16),
        dict(name="copy batch", op="pages_copy", fp8=False, copies=448, kv_heads=8, head_dim=128, page=64),
        dict(name="copy batch fp8", op="pages_copy", fp8=True, copies=448, kv_heads=8, head_dim=128, page=64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng: random.Random):
    op = rng.choice(["attn_beam", "attn_beam", "beam_select", "beam_fork", "pages_copy"])
    if op == "attn_beam":
        q_heads, kv_heads, head_dim = rng.choice([(8, 2, 64), (32, 8, 128), (40, 8, 128), (8, 1, 128), (4, 4, 128), (6, 2, 64), (28, 4, 128)])
        groups, width = _log_int(rng, 1, 48), rng.choice([1, 2, 3, 4, 5, 6, 8, 11, 16])
        most = 1_000_000 // (groups * width) * 8 // kv_heads             # bounds the plain form's gathered pages
        return dict(op=op, fp8=head_dim == 128 and rng.random() < 0.4, groups=groups, width=width, context=_log_int(rng, 1, min(32768, most)),
                    grown=_log_int(rng, 1, 400), q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, page=rng.choice([16, 16, 32, 64]))
    if op == "beam_select":
        groups, width = _log_int(rng, 1, 64), rng.choice([1, 2, 3, 4, 5, 6, 8])
        return dict(op=op, groups=groups, width=width, select=width * rng.choice([1, 1, 2]), vocab=_log_int(rng, 50, 100003),
                    dtype=rng.choice(["bf16", "fp16", "fp32"]))
    if op == "beam_fork":
        return dict(op=op, groups=_log_int(rng, 1, 64), width=rng.choice([1, 2, 3, 4, 5, 6, 8]), context=_log_int(rng, 1, 16640),
                    grown=_log_int(rng, 1, 300), page=rng.choice([16, 16, 32, 64]))
    return dict(op=op, fp8=rng.random() < 0.5, copies=_log_int(rng, 1, 448), kv_heads=rng.choice([1, 2, 8]), head_dim=128, page=rng.choice([16, 32, 64]))


# ------------------------------------------------------------------------------------------------ shapes that follow from the case
def _ragged(n, most, least):
    """n whole numbers between least and most, uneven, the largest among them; a function of the arguments alone."""
    span = most - least + 1
    return np.array([most - (b * 7919 + (b * b) % 13) % span for b in range(n)], dtype=np.int64)


def _beams(case):
    """Lengths [groups, width] and block tables [groups, width, entries] of a decode with beams, the pages numbered as they came
    to be used: a request's context is shared, and from there on the beams are re-drawn from one another at every page, so that
    old pages are common to all or some and young ones a beam's own.  A function of the case alone."""
    P, n, W = case["page"], case["groups"], case["width"]
    rng = np.random.default_rng(17)
    prompt = _ragged(n, case["context"], max(1, (3 * case["context"]) // 4))
    kv = np.repeat((prompt + _ragged(n, case["grown"], max(1, case["grown"] // 2)))[:, None], W, axis=1)
    fixed, ents = prompt // P, -(-kv[:, 0] // P)                       # full pages of the prompt; entries in all
    stride = int(ents.max()) + 1
    tables = np.zeros((n, W, stride), dtype=np.int64)
    used = 0
    for g in range(n):
        f, last = int(fixed[g]), int(ents[g])
        tables[g, :, :f] = used + np.arange(f)
        used += f
        for e in range(f, last):
            tables[g] = tables[g, rng.integers(0, W, size=W)]
            tables[g, :, e] = used + np.arange(W)
            used += W
        if W > 1 and g % 3 == 0:                                         # a beam that has ended, some tokens ago, inside its last page
            kv[g, W - 1] -= int(rng.integers(0, (kv[g, 0] - 1) % P + 1))
    return kv, tables, fixed, used


def _distinct_slots(case, kv, tables):
    """Slots of all distinct pages: what an attention that reads each page once has to read."""
    P, total = case["page"], 0
    for g in range(case["groups"]):
        fill = np.clip(kv[g][:, None] - np.arange(tables.shape[2])[None, :] * P, 0, P)
        page, first = np.unique(np.where(fill > 0, tables[g], -1), return_inverse=True)
        most = np.zeros(len(page), dtype=np.int64)
        np.maximum.at(most, first.reshape(-1), fill.reshape(-1))
        total += int(most[page >= 0].sum())
    return total


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(shape, g, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * std).to(torch.bfloat16)


def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(dtype)


def _rope_table(max_position, head_dim, theta):
    i = torch.arange(head_dim // 2, device=DEV, dtype=torch.float64)
    a = torch.arange(max_position + 1, device=DEV, dtype=torch.float64)[:, None] * torch.pow(torch.tensor(float(theta), device=DEV, dtype=torch.float64), -2 * i / head_dim)
    return torch.stack([torch.cos(a), torch.sin(a)], dim=-1).float().contiguous()


def _quantised(pool):
    """bf16 [pages, heads, page, D] -> e4m3 codes (as bytes) and one scale per (page, head)."""
    x = pool.float()
    scale = x.abs().amax(dim=(2, 3)) / E4M3_MAX
    scale = torch.where(scale > 0, scale, torch.ones_like(scale))
    return (x / scale[:, :, None, None]).to(torch.float8_e4m3fn).view(torch.uint8), scale.contiguous()


def _add_pools(s, shape, g):
    k_pool, v_pool = _normal(shape, g), _normal(shape, g)
    if s["case"]["fp8"]:
        s["k_pool"], s["k_scales"] = _quantised(k_pool)
        s["v_pool"], s["v_scales"] = _quantised(v_pool)
    else:
        s["k_pool"], s["v_pool"] = k_pool, v_pool
    return s


def _prepare_attn(case, seed):
    g, rng = _gen(seed), np.random.default_rng(seed)
    P, D, Hq, Hkv = case["page"], case["head_dim"], case["q_heads"], case["kv_heads"]
    kv, tables, _, used = _beams(case)
    rows, stride = kv.size, tables.shape[2]
    num_pages = used + 3
    perm = rng.permutation(num_pages)                                       # where the pages lie in the pool
    s = dict(case=case, page_ids=_dev(perm[tables].reshape(rows, stride)), pos_base=_dev(np.tile(np.arange(stride) * P, (rows, 1))),
             kv_len=_dev(kv.reshape(-1)), q_pos=_dev(kv.reshape(-1) - 1), rope=_rope_table(int(kv.max()) + P + 64, D, 5e5),
             sm_scale=1.0 / math.sqrt(D), num_pages=num_pages, longest=int(kv.max()))
    qkv = _normal((rows, (Hq + 2 * Hkv) * D), g)                           # one fused projection of the newest tokens
    s["q"] = qkv[:, :Hq * D].view(rows, Hq, D)
    return _add_pools(s, (num_pages, Hkv, P, D), g)


_DTYPES = dict(bf16=torch.bfloat16, fp16=torch.float16, fp32=torch.float32)


def _prepare_select(case, seed):
    g, rng = _gen(seed), np.random.default_rng(seed)
    n, W, V = case["groups"], case["width"], case["vocab"]
    logits = torch.randn((n * W, V), generator=g, device=DEV) * 2.5         # a model's logits: a broad bulk and a few that stand out
    strong = torch.randint(0, V, (n * W, 6), generator=g, device=DEV)
    logits.scatter_(1, strong, torch.rand((n * W, 6), generator=g, device=DEV) * 4 + 11)
    scores = -rng.uniform(0.0, 1.0, size=(n, W)).cumsum(axis=1) - 20 * rng.random((n, 1))
    done = (rng.random((n, W)) < 0.1).astype(np.int64)
    return dict(case=case, logits=logits.to(_DTYPES[case["dtype"]]), scores=_dev(scores, torch.float32), done=_dev(done), eos=2, pad=0)


def _prepare_fork(case, seed):
    rng = np.random.default_rng(seed)
    P, n, W = case["page"], case["groups"], case["width"]
    kv, tables, fixed, used = _beams(case)
    spare = n * W + 40
    perm = rng.permutation(used + spare)
    ents = -(-kv // P)
    mine = np.arange(tables.shape[2])[None, None, :] < ents[..., None]
    grown = mine & (np.arange(tables.shape[2])[None, None, :] >= fixed[:, None, None])      # entries that came out of the reserve
    taken = np.unique(tables[grown])
    owned = np.zeros(used + spare, dtype=np.int64)
    owned[perm[taken]] = 1
    owned[perm[used:]] = 1
    parent = np.where(rng.random((n, W)) < 0.03, -1, rng.integers(0, W, size=(n, W)))
    rows, stride = n * W, tables.shape[2]
    page_ids = np.where(mine, perm[tables], -1).reshape(rows, stride)
    pos_base = np.where(mine, np.arange(stride)[None, None, :] * P + rng.integers(0, 50, size=(n, 1, 1)), 0).reshape(rows, stride)
    reserve = np.concatenate([perm[taken], perm[used:]])                    # what is handed out, then what is free
    return dict(case=case, parent=_dev(parent), kv_len=_dev(kv.reshape(-1)), page_ids=_dev(page_ids), pos_base=_dev(pos_base),
                page_ids_out=_dev(np.full((rows, stride), -1)), pos_base_out=_dev(np.zeros((rows, stride))), owned=_dev(owned, torch.uint8),
                reserve=_dev(reserve), reserve_used=_dev(np.array([len(taken)])), num_pages=used + spare, page=P)


def _prepare_copy(case, seed):
    g, rng = _gen(seed), np.random.default_rng(seed)
    n, P = case["copies"], case["page"]
    num_pages = 2 * n + 5
    perm = rng.permutation(num_pages)
    # a parent's page may go to several beams; a quarter of the list is unused, as after most steps
    src = np.sort(perm[:n])[rng.integers(0, n, size=n)]
    live = max(1, (3 * n) // 4)
    slots = 1 + (np.arange(n) * 7 + 3) % P                                  # how far the pages are filled
    s = dict(case=case, src=_dev(src), dst=_dev(perm[n:2 * n]), slots=_dev(slots), n_copies=_dev(np.array([live])), num_pages=num_pages, page=P)
    return _add_pools(s, (num_pages, case["kv_heads"], P, case["head_dim"]), g)


_PREPARE = dict(attn_beam=_prepare_attn, beam_select=_prepare_select, beam_fork=_prepare_fork, pages_copy=_prepare_copy)


def prepare(case, seed):
    s = _PREPARE[case["op"]](case, seed)
    if own:
        s["call"] = _handle(s)
    return s


# ------------------------------------------------------------------------------------------------ the package's calls
def _device(s, head_dim=128, q_heads=8, kv_heads=8, rope=None):
    import paper_2512_16822_b200 as M
    from paper_2512_16822_b200 import runtime as RT
    max_position = 64 if rope is None else rope.shape[0] - 1
    cfg = M.Config(s["case"].get("page", 16), q_heads, kv_heads, head_dim, s.get("num_pages", 1), max_position, 5e5)
    if "k_scales" in s:
        dev = RT.Device.over(cfg, rope=rope, device=DEV)
        return RT, dev, RT.Fp8Pools.over(dev, s["k_pool"], s["v_pool"], s["k_scales"], s["v_scales"])
    return RT, RT.Device.over(cfg, s.get("k_pool"), s.get("v_pool"), rope=rope, device=DEV), None


def _handle(s):
    """The objects a serving program keeps for the call: they bind the step's buffers and own the outputs and the workspace."""
    case = s["case"]
    if case["op"] == "attn_beam":
        RT, dev, pools = _device(s, case["head_dim"], case["q_heads"], case["kv_heads"], s["rope"])
        plan = RT.BeamPlan(dev, page_ids=s["page_ids"], pos_base=s["pos_base"], kv_len=s["kv_len"], width=case["width"])
        return plan, RT.BeamBatch(dev, q=s["q"], q_pos=s["q_pos"], plan=plan, pools=pools)
    if case["op"] == "beam_select":
        RT, dev, _ = _device(s)
        return RT.BeamSelect(dev, logits=s["logits"], scores=s["scores"], done=s["done"], n_select=case["select"], eos_token=s["eos"], pad_token=s["pad"])
    if case["op"] == "beam_fork":
        RT, dev, _ = _device(s)
        return RT.BeamFork(dev, parent=s["parent"], kv_len=s["kv_len"], page_ids=s["page_ids"], pos_base=s["pos_base"], page_ids_out=s["page_ids_out"],
                           pos_base_out=s["pos_base_out"], owned=s["owned"], reserve=s["reserve"], reserve_used=s["reserve_used"])
    RT, dev, pools = _device(s, case["head_dim"], case["kv_heads"], case["kv_heads"])
    return RT.PagesCopy(dev, src=s["src"], dst=s["dst"], slots=s["slots"], n_copies=s["n_copies"], pools=pools)


def run(state):
    op = state["case"]["op"]
    if own:
        if op == "attn_beam":
            plan, batch = state["call"]
            plan.run()
            return batch.run(state["sm_scale"])
        r = state["call"].run()
        if op == "pages_copy":
            return _pools_of(state)
        if op == "beam_fork":
            return dict(page_ids=state["page_ids_out"], pos_base=state["pos_base_out"], reserve=state["reserve"], **r)
        return r
    return _PLAIN[op](state)


def _pools_of(s):
    if s["case"]["fp8"]:
        return dict(k=s["k_pool"].view(torch.float8_e4m3fn), v=s["v_pool"].view(torch.float8_e4m3fn), k_scales=s["k_scales"], v_scales=s["v_scales"])
    return dict(k=s["k_pool"], v=s["v_pool"])


# ------------------------------------------------------------------------------------------------ plain forms
def _rotate(x, cs):
    """x [..., heads, D] fp32 by the table rows cs [..., D/2, 2] of its positions."""
    c, n = cs[..., None, :, 0], cs[..., None, :, 1]
    lo, hi = x.chunk(2, dim=-1)
    return torch.cat([lo * c - hi * n, lo * n + hi * c], dim=-1)


def _plain_attn(s):
    case = s["case"]
    P, D, Hq, Hkv = case["page"], case["head_dim"], case["q_heads"], case["kv_heads"]
    R, L = s["kv_len"].numel(), s["longest"]
    t = torch.arange(L, device=DEV)
    have = t[None, :] < s["kv_len"][:, None]                                # [R, L]
    ent = (t // P).expand(R, L)
    page = torch.where(have, s["page_ids"].gather(1, ent), 0).long()
    pos = torch.where(have, s["pos_base"].gather(1, ent) + t % P, 0).long()

    def fetch(pool, scales):
        x = pool[page, :, (t % P).expand(R, L)]                             # [R, L, Hkv, D]
        if scales is None:
            return x.float()
        return x.view(torch.float8_e4m3fn).float() * scales[page][..., None]

    K = _rotate(fetch(s["k_pool"], s.get("k_scales")), s["rope"][pos])
    q = (_rotate(s["q"].float(), s["rope"][s["q_pos"].long()]) * s["sm_scale"]).view(R, Hkv, Hq // Hkv, D)
    score = torch.matmul(q, K.permute(0, 2, 3, 1))                          # [R, Hkv, G, L]
    score.masked_fill_(~have[:, None, None], -math.inf)
    w = (score - score.amax(dim=-1, keepdim=True)).exp_()
    V = fetch(s["v_pool"], s.get("v_scales")) * have[..., None, None]
    return (torch.matmul(w, V.transpose(1, 2)) / w.sum(dim=-1, keepdim=True)).reshape(R, Hq, D).to(torch.bfloat16)


def _plain_select(s):
    case = s["case"]
    n, W, V, K = case["groups"], case["width"], case["vocab"], case["select"]
    x = s["logits"].double().view(n, W, V)                                  # 64 bits: continuations of two beams may be neighbours
    done = s["done"].bool()
    top = x.amax(dim=2, keepdim=True)
    cand = s["scores"].double()[..., None] + (x - (top + (x - top).exp().sum(dim=2, keepdim=True).log()))
    stay = torch.where(torch.arange(V, device=DEV) == s["pad"], s["scores"].double()[..., None], -math.inf)
    best, place = torch.where(done[..., None], stay, cand).view(n, W * V).sort(dim=1, descending=True, stable=True)
    best, place = best[:, :K], place[:, :K]
    parent, token = place // V, place % V
    ended = done.gather(1, parent) | (token == s["eos"])
    none = best == -math.inf
    return dict(parent=torch.where(none, -1, parent).int(), token=torch.where(none, -1, token).int(), score=best.float(),
                done=(ended & ~none).int(), n_new=(~ended & ~none).int())


def _plain_fork(s):
    P, n, W = s["page"], s["case"]["groups"], s["case"]["width"]
    stride = s["page_ids"].shape[1]
    e = torch.arange(stride, device=DEV)
    kv, owned = s["kv_len"].long().view(n, W), s["owned"].bool()
    ids, base = s["page_ids"].long().view(n, W, stride), s["pos_base"].long().view(n, W, stride)
    held = e < ((kv + P - 1) // P)[..., None]                                # [n, W, stride]
    parent = s["parent"].long()
    p = parent.clamp(min=0)
    kv2 = torch.where(parent >= 0, kv.gather(1, p), 0)
    wide = p[..., None].expand(n, W, stride)
    held2 = held.gather(1, wide) & (parent >= 0)[..., None]
    ids2, base2 = ids.gather(1, wide), base.gather(1, wide)
    mine = torch.where(held, ids, -1)
    theirs = torch.where(held2, ids2, -2)
    # a page goes back if it is the reserve's and no new beam holds it: once, by the first beam that held it
    kept = (mine[:, :, None] == theirs[:, None]).any(dim=2)
    earlier = torch.arange(W, device=DEV)
    again = ((mine[:, :, None] == mine[:, None]) & (earlier[:, None] > earlier[None])[None, :, :, None]).any(dim=2)
    back = held & owned[ids.clamp(min=0)] & ~kept & ~again
    freed = ids.transpose(1, 2)[back.transpose(1, 2)]                         # by request, entry, beam
    # the partly filled last page is a beam's own: the first that holds it keeps it, if it is the reserve's and nobody's full page
    last = ((kv2 - 1).clamp(min=0) // P)[..., None]
    partial = kv2 % P != 0
    page = theirs.gather(2, last)[..., 0]
    at = theirs.gather(2, last.transpose(1, 2).expand(n, W, W))               # [n, j, k]: what beam j holds where k's last page is
    same = at == page[:, None, :]
    full = kv2[:, :, None] >= (last.transpose(1, 2) + 1) * P
    before = ((same & ~full) & (earlier[:, None] < earlier[None])).any(dim=1)
    copy = partial & ~(owned[page.clamp(min=0)] & ~before & ~(same & full).any(dim=1))
    rank = torch.cumsum(copy.view(-1).long(), 0) - 1
    used = s["reserve_used"].long()
    i = torch.arange(s["reserve"].numel(), device=DEV)
    start = used - freed.numel()
    pad = torch.cat([freed, freed.new_zeros(1)])
    reserve = torch.where((i >= start) & (i < used), pad[(i - start).clamp(0, freed.numel())], s["reserve"].long())
    fresh = reserve[(start + rank).clamp(0, reserve.numel() - 1)].view(n, W)
    swap = copy[..., None] & (e == last)
    ids3 = torch.where(swap, fresh[..., None], ids2)
    out_ids = torch.where(held2, ids3, s["page_ids_out"].long().view(n, W, stride))
    out_base = torch.where(held2, base2, s["pos_base_out"].long().view(n, W, stride))
    total = copy.sum()
    place = torch.where(copy.view(-1), rank, n * W)
    lists = [torch.full((n * W + 1,), -1, device=DEV, dtype=torch.long).scatter(0, place, v.reshape(-1))[:-1].int() for v in (page, fresh, kv2 % P)]
    s["reserve"].copy_(reserve)
    s["page_ids_out"].copy_(out_ids.view(n * W, stride))
    s["pos_base_out"].copy_(out_base.view(n * W, stride))
    return dict(page_ids=s["page_ids_out"], pos_base=s["pos_base_out"], reserve=s["reserve"], kv_len=kv2.view(-1).int(), copy_src=lists[0],
                copy_dst=lists[1], copy_slots=lists[2], n_copies=total.view(1).int(), reserve_used=(start + total).int())


def _plain_copy(s):
    n, P = s["case"]["copies"], s["page"]
    t = torch.arange(P, device=DEV)
    live = (torch.arange(n, device=DEV)[:, None] < s["n_copies"]) & (t[None, :] < s["slots"][:, None])
    i, t = live.nonzero(as_tuple=True)
    src, dst = s["src"].long()[i], s["dst"].long()[i]
    for name in ("k", "v"):
        pool = s[name + "_pool"]
        pool[dst, :, t] = pool[src, :, t]
        if s["case"]["fp8"]:
            scales = s[name + "_scales"]
            scales[dst] = scales[src]
    return _pools_of(s)


_PLAIN = dict(attn_beam=_plain_attn, beam_select=_plain_select, beam_fork=_plain_fork, pages_copy=_plain_copy)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    op = case["op"]
    if op == "attn_beam":
        kv, tables, _, _ = _beams(case)
        P, D, Hq, Hkv = case["page"], case["head_dim"], case["q_heads"], case["kv_heads"]
        slots = _distinct_slots(case, kv, tables)
        nbytes = 2 * slots * Hkv * D * (1 if case["fp8"] else 2) + (8 * Hkv * (slots // P) if case["fp8"] else 0)
        return dict(bytes=nbytes + kv.size * Hq * D * 4 + int((-(-kv // P)).sum()) * 8, flops=4.0 * int(kv.sum()) * Hq * D)
    if op == "beam_select":
        rows = case["groups"] * case["width"]
        size = 4 if case["dtype"] == "fp32" else 2
        return dict(bytes=rows * case["vocab"] * size + 8 * rows + 20 * case["groups"] * case["select"], flops=4.0 * rows * case["vocab"])
    if op == "beam_fork":
        kv, _, _, _ = _beams(case)
        return dict(bytes=int((-(-kv // case["page"])).sum()) * 16 + kv.size * 24, flops=0)
    n, P = case["copies"], case["page"]
    slots = int((1 + (np.arange(max(1, (3 * n) // 4)) * 7 + 3) % P).sum())
    return dict(bytes=4 * slots * case["kv_heads"] * case["head_dim"] * (1 if case["fp8"] else 2) + 12 * n, flops=0)


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def _exact_attn(case, s):
    P, D, Hq, Hkv = case["page"], case["head_dim"], case["q_heads"], case["kv_heads"]
    G = Hq // Hkv
    inv = torch.pow(torch.tensor(5e5, device=DEV, dtype=torch.float64), -2 * torch.arange(D // 2, device=DEV, dtype=torch.float64) / D)

    def turned(x, pos):                                                     # x [n, D] by its positions, as complex numbers
        z = torch.complex(x[:, :D // 2].contiguous(), x[:, D // 2:].contiguous()) * torch.exp(1j * (pos.double()[:, None] * inv))
        return torch.cat([z.real, z.imag], dim=1)

    kv = s["kv_len"].tolist()
    out = torch.zeros(len(kv), Hq, D, device=DEV, dtype=torch.float64)
    for r, n in enumerate(kv):
        ents = -(-n // P)
        ids = s["page_ids"][r, :ents].long()
        pos = (s["pos_base"][r, :ents, None] + torch.arange(P, device=DEV)).reshape(-1)[:n]
        for h in range(Hkv):
            kp, vp = s["k_pool"][ids, h], s["v_pool"][ids, h]
            if case["fp8"]:
                kp = kp.view(torch.float8_e4m3fn).double() * s["k_scales"][ids, h].double()[:, None, None]
                vp = vp.view(torch.float8_e4m3fn).double() * s["v_scales"][ids, h].double()[:, None, None]
            q = turned(s["q"][r, h * G:(h + 1) * G].double(), s["q_pos"][r].expand(G))
            w = torch.softmax(q @ turned(kp.double().reshape(-1, D)[:n], pos).T / math.sqrt(D), dim=1)
            out[r, h * G:(h + 1) * G] = w @ vp.double().reshape(-1, D)[:n]
    return out


def _exact_select(case, s):
    n, W, K = case["groups"], case["width"], case["select"]
    scores, done = s["scores"].tolist(), s["done"].tolist()
    found = torch.full((n, K), -math.inf, device=DEV, dtype=torch.float64)
    for g in range(n):
        lists = []
        for w in range(W):
            if done[g][w]:
                lists.append(torch.tensor([scores[g][w]], device=DEV, dtype=torch.float64))
            else:
                lists.append(scores[g][w] + torch.log_softmax(s["logits"][g * W + w].double(), dim=0).topk(min(K, case["vocab"])).values)
        best = torch.cat(lists).sort(descending=True).values[:K]
        found[g, :best.numel()] = best
    return dict(parent=None, token=None, score=found, done=None, n_new=None)


def _exact_copy(case, s):
    src, dst, slots = s["src"].tolist(), s["dst"].tolist(), s["slots"].tolist()
    found = {}
    for name in ("k", "v"):
        pool = s[name + "_pool"]
        pool = (pool.view(torch.float8_e4m3fn) if case["fp8"] else pool).double()
        for i in range(int(s["n_copies"])):
            pool[dst[i], :, :slots[i]] = pool[src[i], :, :slots[i]]
        found[name] = pool
        if case["fp8"]:
            scales = s[name + "_scales"].double()
            for i in range(int(s["n_copies"])):
                scales[dst[i]] = scales[src[i]]
            found[name + "_scales"] = scales
    return found


def exact(case, seed):
    if case["op"] == "beam_fork":
        return None                                                         # whole numbers only
    s = _PREPARE[case["op"]](case, seed)
    return dict(attn_beam=_exact_attn, beam_select=_exact_select, pages_copy=_exact_copy)[case["op"]](case, s)
