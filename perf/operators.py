"""Measured cases of the drafted-token operators: one speculative serving step over the page pool.

A step drafts a tree of tokens per request, attends every drafted row to the request's paged context and to its own
ancestors, keeps the path the model agrees with, hands out the slots and pages of the kept tokens and writes their K/V
rows into the pages.  The operators, in the order a step uses them:

* tree_layout  - parents -> position and ancestor mask of every drafted row,
* attn_tree    - attention of the drafted rows over the un-rotated paged context plus the drafted rows they may see,
                 over bf16 pages or 8-bit (e4m3) pages,
* tree_accept  - parents, drafted tokens and the model's choices -> the accepted path of every request,
* step_tables  - lengths and new-row counts -> block tables, logical slots and physical slots, pages taken from a reserve,
* rows_commit  - K/V rows into their physical slots, bf16 or 8-bit pages.

``run`` computes the plain form (fp32 torch) unless ``own`` is set, and then makes the calls of the package.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
VOCAB = 32000
E4M3_MAX = 448.0


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one user's request at the start of a chat, a handful of drafts: only latency counts
        dict(name="attn one request", op="attn_tree", fp8=False, batch=1, context=203, rows=8, q_heads=8, kv_heads=2,
             head_dim=64, page=16, shared=False),
        # a full serving batch of RAG prompts (16 chunks of 512 tokens and a question), 16 drafts per request
        dict(name="attn serving batch", op="attn_tree", fp8=False, batch=32, context=8256, rows=16, q_heads=32, kv_heads=8,
             head_dim=128, page=16, shared=False),
        # a large draft tree per request over long prompts that alias common chunks
        dict(name="attn wide trees", op="attn_tree", fp8=False, batch=8, context=16640, rows=96, q_heads=32, kv_heads=8,
             head_dim=128, page=16, shared=True),
        # very long prompts in 8-bit pages, 64-token pages
        dict(name="attn long fp8", op="attn_tree", fp8=True, batch=8, context=65536, rows=32, q_heads=32, kv_heads=8,
             head_dim=128, page=64, shared=False),
        # layout of one small tree, and of a large batch of large trees
        dict(name="layout one tree", op="tree_layout", batch=1, rows=8),
        dict(name="layout many trees", op="tree_layout", batch=128, rows=200),
        # verification of one small tree, and of a large batch
        dict(name="accept one tree", op="tree_accept", batch=1, rows=8),
        dict(name="accept many trees", op="tree_accept", batch=256, rows=64),
        # the step of a decode batch: a token or a few per request
        dict(name="tables decode step", op="step_tables", batch=32, context=8256, new=4, page=16),
        # a prompt batch: hundreds to thousands of rows per request
        dict(name="tables prompts", op="step_tables", batch=64, context=16640, new=2048, page=16),
        # the accepted rows of a serving batch, gathered out of the drafted ones
        dict(name="commit accepted", op="rows_commit", fp8=False, batch=32, new=4, gather=True, kv_heads=8, head_dim=128, page=16),
        # whole prompts into 8-bit pages
        dict(name="commit prompts fp8", op="rows_commit", fp8=True, batch=8, new=2048, gather=False, kv_heads=8, head_dim=128, page=16),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng: random.Random):
    op = rng.choice(["attn_tree", "attn_tree", "tree_layout", "tree_accept", "step_tables", "rows_commit"])
    if op == "attn_tree":
        q_heads, kv_heads, head_dim = rng.choice([(8, 2, 64), (32, 8, 128), (40, 8, 128), (8, 1, 128), (4, 4, 128), (6, 2, 64)])
        batch = _log_int(rng, 1, 64)
        context = _log_int(rng, 1, 65536 // max(1, batch // 4))
        most = 530_000_000 // (batch * context * q_heads)          # bounds the plain form's scores
        rows = _log_int(rng, 1, max(1, min(160, most)))
        return dict(op=op, fp8=head_dim == 128 and rng.random() < 0.4, batch=batch, context=context, rows=rows, q_heads=q_heads,
                    kv_heads=kv_heads, head_dim=head_dim, page=rng.choice([16, 16, 32, 64]), shared=rng.random() < 0.4)
    if op in ("tree_layout", "tree_accept"):
        return dict(op=op, batch=_log_int(rng, 1, 256), rows=_log_int(rng, 1, 128))
    if op == "step_tables":
        return dict(op=op, batch=_log_int(rng, 1, 64), context=_log_int(rng, 1, 16000), new=_log_int(rng, 1, 2000), page=rng.choice([16, 32, 64]))
    return dict(op=op, fp8=rng.random() < 0.5, batch=_log_int(rng, 1, 64), new=_log_int(rng, 1, 256), gather=rng.random() < 0.5,
                kv_heads=rng.choice([1, 2, 8]), head_dim=128, page=rng.choice([16, 32, 64]))


# ------------------------------------------------------------------------------------------------ shapes that follow from the case
def _ragged(n, most, least):
    """n whole numbers between least and most, uneven, the largest among them; a function of the arguments alone."""
    span = most - least + 1
    return np.array([most - (b * 7919 + (b * b) % 13) % span for b in range(n)], dtype=np.int64)


def _contexts(case):
    return _ragged(case["batch"], case["context"], max(1, (3 * case["context"]) // 4))


def _row_counts(case):
    return _ragged(case["batch"], case["rows"], max(1, case["rows"] // 2))


def _new_counts(case):
    return _ragged(case["batch"], case["new"], max(0, case["new"] // 2))


def _words(rows):
    return (rows + 31) // 32


def _max_accept(rows):
    return min(rows, 16)


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(shape, g, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * std).to(torch.bfloat16)


def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(dtype)


def _offsets(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)


def _parents(counts, rng):
    """A random tree per request: a row hangs under one of the eight rows before it or under the context."""
    total = int(counts.sum())
    parent = np.empty(total, dtype=np.int64)
    at = 0
    for n in counts:
        i = np.arange(n)
        parent[at:at + n] = np.maximum(i - 1 - rng.integers(0, 8, size=n), -1)
        at += n
    return parent


def _depths_and_masks(counts, parent, words):
    total = int(counts.sum())
    depth = np.zeros(total, dtype=np.int64)
    mask = np.zeros((total, words), dtype=np.uint32)
    at = 0
    for n in counts:
        for i in range(n):
            p = parent[at + i]
            if p >= 0:
                depth[at + i] = depth[at + p] + 1
                mask[at + i] = mask[at + p]
            mask[at + i, i // 32] |= np.uint32(1 << (i % 32))
        at += n
    return depth, mask.view(np.int32)


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


def _prepare_attn(case, seed):
    g, rng = _gen(seed), np.random.default_rng(seed)
    B, P, D, Hq, Hkv = case["batch"], case["page"], case["head_dim"], case["q_heads"], case["kv_heads"]
    kv, rows = _contexts(case), _row_counts(case)
    off, total = _offsets(rows), int(rows.sum())
    ents = -(-kv // P)
    stride = int(ents.max()) + 1
    common = int(ents.min()) // 2 if case["shared"] else 0                 # leading pages that every request aliases
    num_pages = common + int((ents - common).sum()) + 3
    perm = rng.permutation(num_pages)
    page_ids = np.zeros((B, stride), dtype=np.int64)
    pos_base = np.zeros((B, stride), dtype=np.int64)
    at = common
    for b in range(B):
        own_pages = int(ents[b]) - common
        page_ids[b, :ents[b]] = np.concatenate([perm[:common], perm[at:at + own_pages]])
        pos_base[b, :ents[b]] = np.arange(ents[b]) * P
        at += own_pages
    parent = _parents(rows, rng)
    depth, mask = _depths_and_masks(rows, parent, _words(int(rows.max())))
    row_pos = np.repeat(kv, rows) + depth
    qkv = _normal((total, (Hq + 2 * Hkv) * D), g)                          # one fused projection of the drafted rows
    s = dict(case=case, qkv=qkv, q=qkv[:, :Hq * D].view(total, Hq, D), k_new=qkv[:, Hq * D:(Hq + Hkv) * D].view(total, Hkv, D),
             v_new=qkv[:, (Hq + Hkv) * D:].view(total, Hkv, D), page_ids=_dev(page_ids), pos_base=_dev(pos_base), kv_len=_dev(kv),
             row_offsets=_dev(off), row_pos=_dev(row_pos), tree_mask=_dev(mask), rope=_rope_table(int(kv.max()) + int(rows.max()) + P, D, 5e5),
             sm_scale=1.0 / math.sqrt(D), max_rows=int(rows.max()), longest=int(kv.max()), num_pages=num_pages)
    k_pool, v_pool = _normal((num_pages, Hkv, P, D), g), _normal((num_pages, Hkv, P, D), g)
    if case["fp8"]:
        s["k_pool"], s["k_scales"] = _quantised(k_pool)
        s["v_pool"], s["v_scales"] = _quantised(v_pool)
    else:
        s["k_pool"], s["v_pool"] = k_pool, v_pool
    return s


def _prepare_layout(case, seed):
    rng = np.random.default_rng(seed)
    rows = _row_counts(case)
    kv = rng.integers(1, 4000, size=case["batch"])
    P, stride = 16, 251
    base = np.arange(stride)[None, :] * P + rng.integers(0, 50, size=(case["batch"], 1))
    return dict(case=case, parent=_dev(_parents(rows, rng)), row_offsets=_dev(_offsets(rows)), kv_len=_dev(kv), pos_base=_dev(base),
                page=P, mask_words=_words(int(rows.max())), max_rows=int(rows.max()), total=int(rows.sum()))


def _prepare_accept(case, seed):
    rng = np.random.default_rng(seed)
    rows = _row_counts(case)
    off, total = _offsets(rows), int(rows.sum())
    parent = _parents(rows, rng)
    target = rng.integers(0, VOCAB, size=total)
    root = rng.integers(0, VOCAB, size=case["batch"])
    start = np.repeat(off[:-1], rows)
    wanted = np.where(parent >= 0, target[start + np.maximum(parent, 0)], np.repeat(root, rows))
    draft = np.where(rng.random(total) < 0.7, wanted, rng.integers(0, VOCAB, size=total))
    return dict(case=case, parent=_dev(parent), row_offsets=_dev(off), draft=_dev(draft), target=_dev(target), root=_dev(root),
                max_rows=int(rows.max()), max_accept=_max_accept(int(rows.max())))


def _prepare_tables(case, seed):
    rng = np.random.default_rng(seed)
    B, P = case["batch"], case["page"]
    kv, new = _contexts(case), _new_counts(case)
    held, need = -(-kv // P), -(-(kv + new) // P)
    grow = need - held
    stride = int(need.max()) + 2
    perm = rng.permutation(int(held.sum() + grow.sum()) + 40)
    page_ids, pos_base = np.full((B, stride), -1, dtype=np.int64), np.zeros((B, stride), dtype=np.int64)
    first = rng.integers(0, 64, size=B)
    at = 0
    for b in range(B):
        page_ids[b, :held[b]] = perm[at:at + held[b]]
        pos_base[b, :held[b]] = first[b] + np.arange(held[b]) * P
        at += int(held[b])
    return dict(case=case, page_ids=_dev(page_ids), pos_base=_dev(pos_base), kv_len=_dev(kv), n_new=_dev(new), reserve=_dev(perm[at:]),
                reserve_used=_dev(np.array([5])), max_rows=int(new.sum()), num_pages=len(perm), page=P)


def _prepare_commit(case, seed):
    g, rng = _gen(seed), np.random.default_rng(seed)
    B, P, Hkv, D = case["batch"], case["page"], case["kv_heads"], case["head_dim"]
    new = _new_counts(case)
    off, total = _offsets(new), int(new.sum())
    start = rng.integers(0, P, size=B)                                      # in-page slot at which a request goes on
    start[:: 3] = 0                                                         # every third request starts a page
    pages = -(-(start + new) // P)
    num_pages = int((-(-(P - 1 + new) // P)).sum()) + 64
    perm = rng.permutation(num_pages)
    slot = np.empty(total, dtype=np.int64)
    at = 0
    for b in range(B):
        t = start[b] + np.arange(new[b])
        slot[off[b]:off[b + 1]] = perm[at + t // P] * P + t % P
        at += int(pages[b])
    s = dict(case=case, row_offsets=_dev(off), slot_map=_dev(slot, torch.int64), num_pages=num_pages, max_rows=total, batch_of=_dev(np.repeat(np.arange(B), new), torch.int64))
    sources = total
    if case["gather"]:
        # the accepted rows of each request among its drafted ones (four drafts for every kept row)
        width = max(1, int(new.max()))
        src = np.full((B, width), -1, dtype=np.int64)
        for b in range(B):
            src[b, :new[b]] = 4 * off[b] + np.sort(rng.choice(4 * new[b], size=new[b], replace=False)) if new[b] else []
        sources = 4 * total
        s["src_rows"] = _dev(src)
    fused = _normal((max(1, sources), 2 * Hkv * D), g)
    s["k_new"], s["v_new"] = fused[:, :Hkv * D].view(-1, Hkv, D), fused[:, Hkv * D:].view(-1, Hkv, D)
    k_pool, v_pool = _normal((num_pages, Hkv, P, D), g), _normal((num_pages, Hkv, P, D), g)
    if case["fp8"]:
        s["k_pool"], s["k_scales"] = _quantised(k_pool)
        s["v_pool"], s["v_scales"] = _quantised(v_pool)
    else:
        s["k_pool"], s["v_pool"] = k_pool, v_pool
    return s


_PREPARE = dict(attn_tree=_prepare_attn, tree_layout=_prepare_layout, tree_accept=_prepare_accept, step_tables=_prepare_tables,
                rows_commit=_prepare_commit)


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
    cfg = M.Config(s["page"] if "page" in s else s["case"]["page"], q_heads, kv_heads, head_dim, s.get("num_pages", 1), max_position, 5e5)
    if "k_scales" in s:
        dev = RT.Device.over(cfg, rope=rope, device=DEV)
        return RT, dev, RT.Fp8Pools.over(dev, s["k_pool"], s["v_pool"], s["k_scales"], s["v_scales"])
    return RT, RT.Device.over(cfg, s.get("k_pool"), s.get("v_pool"), rope=rope, device=DEV), None


def _handle(s):
    """The object a serving program keeps for the call: it binds the step's buffers and owns the outputs and the workspace."""
    case = s["case"]
    if case["op"] == "attn_tree":
        RT, dev, pools = _device(s, case["head_dim"], case["q_heads"], case["kv_heads"], s["rope"])
        return RT.TreeBatch(dev, q=s["q"], k_new=s["k_new"], v_new=s["v_new"], row_offsets=s["row_offsets"], row_pos=s["row_pos"],
                            tree_mask=s["tree_mask"], page_ids=s["page_ids"], pos_base=s["pos_base"], kv_len=s["kv_len"],
                            max_rows=s["max_rows"], pools=pools)
    if case["op"] == "tree_layout":
        RT, dev, _ = _device(s)
        return RT.TreeLayout(dev, parent=s["parent"], row_offsets=s["row_offsets"], pos_base=s["pos_base"], kv_len=s["kv_len"],
                             mask_words=s["mask_words"])
    if case["op"] == "tree_accept":
        RT, dev, _ = _device(dict(s, page=16))
        return RT.TreeAccept(dev, parent=s["parent"], row_offsets=s["row_offsets"], draft=s["draft"], target=s["target"], root=s["root"],
                             max_accept=s["max_accept"])
    if case["op"] == "step_tables":
        RT, dev, _ = _device(s)
        return RT.StepTables(dev, kv_len=s["kv_len"], n_new=s["n_new"], page_ids=s["page_ids"], pos_base=s["pos_base"],
                             reserve=s["reserve"], reserve_used=s["reserve_used"], max_rows=s["max_rows"])
    RT, dev, pools = _device(s, case["head_dim"], case["kv_heads"], case["kv_heads"])
    return RT.RowsCommit(dev, k_new=s["k_new"], v_new=s["v_new"], row_offsets=s["row_offsets"], slot_map=s["slot_map"],
                         src_rows=s.get("src_rows"), pools=pools)


def run(state):
    op = state["case"]["op"]
    if own:
        r = state["call"].run(state["sm_scale"]) if op == "attn_tree" else state["call"].run()
        if op == "rows_commit":
            return _pools_of(state)
        if op == "step_tables":
            return dict(page_ids=state["page_ids"], pos_base=state["pos_base"], **r)
        return r
    return _PLAIN[op](state)


def _pools_of(s):
    if s["case"]["fp8"]:
        return dict(k=s["k_pool"].view(torch.float8_e4m3fn), v=s["v_pool"].view(torch.float8_e4m3fn), k_scales=s["k_scales"], v_scales=s["v_scales"])
    return dict(k=s["k_pool"], v=s["v_pool"])


# ------------------------------------------------------------------------------------------------ plain forms
def _padded(s):
    """Row index of every (request, place) of a padded [batch, max_rows] layout, and which places hold a row."""
    off = s["row_offsets"].long()
    i = torch.arange(s["max_rows"], device=DEV)
    live = i[None, :] < (off[1:] - off[:-1])[:, None]
    return torch.where(live, off[:-1, None] + i[None, :], 0), live


def _rotate(x, cs):
    """x [..., heads, D] fp32 by the table rows cs [..., D/2, 2] of its positions."""
    c, n = cs[..., None, :, 0], cs[..., None, :, 1]
    lo, hi = x.chunk(2, dim=-1)
    return torch.cat([lo * c - hi * n, lo * n + hi * c], dim=-1)


def _plain_attn(s):
    case = s["case"]
    B, P, D, Hq, Hkv = case["batch"], case["page"], case["head_dim"], case["q_heads"], case["kv_heads"]
    G, L, T = Hq // Hkv, s["longest"], s["max_rows"]
    rows, live = _padded(s)
    t = torch.arange(L, device=DEV)
    have = t[None, :] < s["kv_len"][:, None]                                # [B, L]
    ent = (t // P).expand(B, L)
    page = torch.where(have, s["page_ids"].gather(1, ent), 0).long()
    pos = torch.where(have, s["pos_base"].gather(1, ent) + t % P, 0).long()

    def fetch(pool, scales):
        x = pool[page, :, (t % P).expand(B, L)]                             # [B, L, Hkv, D]
        if scales is None:
            return x.float()
        return x.view(torch.float8_e4m3fn).float() * scales[page][..., None]

    K = _rotate(fetch(s["k_pool"], s.get("k_scales")), s["rope"][pos])
    V = fetch(s["v_pool"], s.get("v_scales")) * have[..., None, None]
    dpos = s["rope"][s["row_pos"].long()[rows]]                            # [B, T, D/2, 2]
    K = torch.cat([K, _rotate(s["k_new"][rows].float(), dpos)], dim=1)
    V = torch.cat([V, s["v_new"][rows].float() * live[..., None, None]], dim=1)
    q = _rotate(s["q"][rows].float(), dpos) * s["sm_scale"]
    bits = (s["tree_mask"][rows][..., None] >> torch.arange(32, device=DEV, dtype=torch.int32)) & 1
    sees = bits.flatten(2)[..., :T].bool() & live[:, :, None] & live[:, None, :]
    sees = torch.cat([(have[:, None, :] & live[:, :, None]), sees], dim=2)   # [B, T, L + T]
    q = q.view(B, T, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * T, D)
    score = torch.matmul(q, K.permute(0, 2, 3, 1)).view(B, Hkv, G, T, L + T)
    score.masked_fill_(~sees[:, None, None], -math.inf)
    top = score.amax(dim=-1, keepdim=True)
    score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = score.sum(dim=-1, keepdim=True)
    out = torch.matmul(score.view(B, Hkv, G * T, L + T), V.transpose(1, 2)).view(B, Hkv, G, T, D)
    out = torch.where(total > 0, out / total, 0.0).permute(0, 3, 1, 2, 4).reshape(B, T, Hq, D)
    return out[live].to(torch.bfloat16)


def _closure(parent):
    """parent [B, T] (-1 = none) -> [B, T, T]: 1 where the column is the row itself or an ancestor of it."""
    T = parent.shape[1]
    reach = (parent[..., None] == torch.arange(T, device=DEV)).float() + torch.eye(T, device=DEV)
    for _ in range(max(1, (T - 1).bit_length())):                           # paths of 1, 2, 4, ... edges
        reach = (torch.matmul(reach, reach) > 0).float()
    return reach


def _plain_layout(s):
    rows, live = _padded(s)
    T, P, kv = s["max_rows"], s["page"], s["kv_len"].long()
    reach = _closure(torch.where(live, s["parent"].long()[rows], -1))
    depth = reach.sum(dim=2).long() - 1
    after = s["pos_base"].long().gather(1, ((kv - 1) // P).clamp(min=0)[:, None])[:, 0] + (kv - 1) % P + 1
    after = torch.where(kv > 0, after, 0)
    W = s["mask_words"]
    word = torch.nn.functional.pad(reach.long(), (0, 32 * W - T)).view(*reach.shape[:2], W, 32)
    word = (word << torch.arange(32, device=DEV)).sum(dim=3)
    return dict(row_pos=(after[:, None] + depth)[live].int(), tree_mask=torch.where(word >= 2 ** 31, word - 2 ** 32, word)[live].int())


def _plain_accept(s):
    rows, live = _padded(s)
    B, T, A = s["case"]["batch"], s["max_rows"], s["max_accept"]
    parent = torch.where(live, s["parent"].long()[rows], -2)
    target, draft = s["target"].long()[rows], s["draft"].long()[rows]
    wanted = torch.where(parent >= 0, target.gather(1, parent.clamp(min=0)), s["root"].long()[:, None])
    fits = live & (draft == wanted)
    earlier = torch.arange(T, device=DEV)[:, None] > torch.arange(T, device=DEV)[None, :]
    rival = ((parent[:, :, None] == parent[:, None, :]) & fits[:, None, :] & earlier).any(dim=2)
    fits = fits & ~rival                                                    # of several matching siblings the first
    reach = _closure(parent)
    path = torch.matmul(reach, fits.float()[..., None])[..., 0] == reach.sum(dim=2)
    step = torch.where(path, reach.sum(dim=2).long() - 1, A)                # place on the path
    path = path & (step < A)
    n = path.sum(dim=1)
    kept = torch.full((B, A + 1), -1, device=DEV, dtype=torch.long)
    kept.scatter_(1, torch.where(path, step, A), torch.where(path, rows, -1))
    kept = kept[:, :A]
    last = kept.gather(1, (n - 1).clamp(min=0)[:, None])[:, 0]
    nxt = torch.where(n > 0, s["target"].long()[last.clamp(min=0)], s["root"].long())
    return dict(n_accept=n.int(), accept_rows=kept.int(), next_token=nxt.int())


def _plain_tables(s):
    P, kv, new = s["page"], s["kv_len"].long(), s["n_new"].long()
    held, need = (kv + P - 1) // P, (kv + new + P - 1) // P
    grow = need - held
    taken = torch.cumsum(grow, 0) - grow + s["reserve_used"].long()
    e = torch.arange(s["page_ids"].shape[1], device=DEV)[None, :]
    fresh = (e >= held[:, None]) & (e < need[:, None])
    place = torch.where(fresh, taken[:, None] + e - held[:, None], 0)
    pages = torch.where(fresh, s["reserve"].long()[place], s["page_ids"].long())
    last = s["pos_base"].long().gather(1, (held - 1).clamp(min=0)[:, None])
    base = torch.where(held[:, None] > 0, last + (e - held[:, None] + 1) * P, e * P)
    base = torch.where(fresh, base, s["pos_base"].long())
    off = torch.cat([torch.zeros(1, device=DEV, dtype=torch.long), torch.cumsum(new, 0)])
    row = torch.arange(s["max_rows"], device=DEV)
    b = torch.searchsorted(off[1:], row, right=True).clamp(max=len(kv) - 1)
    live = row < off[-1]
    slot = kv[b] + row - off[b]
    flat = pages[b, (slot // P).clamp(max=e.shape[1] - 1)] * P + slot % P
    kv2 = kv + new
    pos = torch.where(kv2 > 0, base.gather(1, ((kv2 - 1) // P).clamp(min=0)[:, None])[:, 0] + (kv2 - 1) % P, -1)
    return dict(page_ids=pages.int(), pos_base=base.int(), row_offsets=off.int(), row_slot=torch.where(live, slot, -1).int(),
                slot_map=torch.where(live, flat, -1), kv_len=kv2.int(), q_pos=pos.int(), reserve_used=(s["reserve_used"].long() + grow.sum()).int())


def _plain_commit(s):
    case, P = s["case"], s["case"]["page"]
    page, place = s["slot_map"] // P, s["slot_map"] % P
    row = torch.arange(s["max_rows"], device=DEV)
    src = row
    if case["gather"]:
        src = s["src_rows"].long()[s["batch_of"], row - s["row_offsets"].long()[s["batch_of"]]]
    for pool, new, scales in ((s["k_pool"], s["k_new"], s.get("k_scales")), (s["v_pool"], s["v_new"], s.get("v_scales"))):
        x = new[src]                                                        # [rows, Hkv, D]
        if not case["fp8"]:
            pool[page, :, place] = x
            continue
        x = x.float()
        top = torch.zeros_like(scales).index_reduce_(0, page, x.abs().amax(dim=2), "amax")
        starts = torch.zeros(scales.shape[0], device=DEV).index_reduce_(0, page, (place == 0).float(), "amax")[:, None] > 0
        scales.copy_(torch.where(starts, torch.where(top > 0, top / E4M3_MAX, 1.0), scales))
        code = (x / scales[page][..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        pool[page, :, place] = code
    return _pools_of(s)


_PLAIN = dict(attn_tree=_plain_attn, tree_layout=_plain_layout, tree_accept=_plain_accept, step_tables=_plain_tables, rows_commit=_plain_commit)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    op = case["op"]
    if op == "attn_tree":
        kv, rows = _contexts(case), _row_counts(case)
        P, D, Hq, Hkv = case["page"], case["head_dim"], case["q_heads"], case["kv_heads"]
        ents = -(-kv // P)
        common = (int(ents.min()) // 2) * P if case["shared"] else 0
        unique = common + int((kv - common).sum())
        each = 1 if case["fp8"] else 2
        nbytes = 2 * unique * Hkv * D * each + (8 * Hkv * (unique // P) if case["fp8"] else 0)
        nbytes += int(rows.sum()) * D * 2 * (2 * Hq + 2 * Hkv) + int(ents.sum()) * 8
        seen = int((rows * (kv + (rows + 1) // 2)).sum())
        return dict(bytes=nbytes, flops=4.0 * seen * Hq * D)
    if op in ("tree_layout", "tree_accept"):
        total = int(_row_counts(case).sum())
        if op == "tree_layout":
            return dict(bytes=total * (8 + 4 * _words(case["rows"])) + 12 * case["batch"], flops=0)
        return dict(bytes=12 * total + case["batch"] * (16 + 4 * _max_accept(case["rows"])), flops=0)
    if op == "step_tables":
        kv, new = _contexts(case), _new_counts(case)
        grown = int((-(-(kv + new) // case["page"]) + kv // -case["page"]).sum())
        return dict(bytes=int(new.sum()) * 12 + 12 * grown + 24 * case["batch"], flops=0)
    total = int(_new_counts(case).sum())
    return dict(bytes=total * case["kv_heads"] * case["head_dim"] * 2 * (3 if case["fp8"] else 4) + 8 * total, flops=0)


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def _exact_attn(case, s):
    P, D, Hq, Hkv = case["page"], case["head_dim"], case["q_heads"], case["kv_heads"]
    G, scale = Hq // Hkv, 1.0 / math.sqrt(D)
    inv = torch.pow(torch.tensor(5e5, device=DEV, dtype=torch.float64), -2 * torch.arange(D // 2, device=DEV, dtype=torch.float64) / D)

    def turned(x, pos):                                                     # x [n, D] by its positions, as complex numbers
        z = torch.complex(x[:, :D // 2].contiguous(), x[:, D // 2:].contiguous()) * torch.exp(1j * (pos.double()[:, None] * inv))
        return torch.cat([z.real, z.imag], dim=1)

    off, kv = s["row_offsets"].tolist(), s["kv_len"].tolist()
    out = torch.zeros(off[-1], Hq, D, device=DEV, dtype=torch.float64)
    for b in range(case["batch"]):
        r0, r1 = off[b], off[b + 1]
        n = -(-kv[b] // P)
        ids = s["page_ids"][b, :n].long()
        pos = (s["pos_base"][b, :n, None] + torch.arange(P, device=DEV)).reshape(-1)[:kv[b]]
        word = s["tree_mask"][r0:r1].long() & 0xffffffff
        j = torch.arange(r1 - r0, device=DEV)
        sees = ((word[:, j // 32] >> (j % 32)) & 1).bool()
        sees = torch.cat([torch.ones(r1 - r0, kv[b], device=DEV, dtype=torch.bool), sees], dim=1).repeat_interleave(G, dim=0)
        for h in range(Hkv):
            kp, vp = s["k_pool"][ids, h], s["v_pool"][ids, h]
            if case["fp8"]:
                kp = kp.view(torch.float8_e4m3fn).double() * s["k_scales"][ids, h].double()[:, None, None]
                vp = vp.view(torch.float8_e4m3fn).double() * s["v_scales"][ids, h].double()[:, None, None]
            K = turned(torch.cat([kp.double().reshape(-1, D)[:kv[b]], s["k_new"][r0:r1, h].double()]), torch.cat([pos, s["row_pos"][r0:r1]]))
            V = torch.cat([vp.double().reshape(-1, D)[:kv[b]], s["v_new"][r0:r1, h].double()])
            q = turned(s["q"][r0:r1, h * G:(h + 1) * G].double().reshape(-1, D), s["row_pos"][r0:r1].repeat_interleave(G))
            w = torch.softmax((q @ K.T * scale).masked_fill(~sees, -math.inf), dim=1).nan_to_num(0.0)
            out[r0:r1, h * G:(h + 1) * G] = (w @ V).view(r1 - r0, G, D)
    return out


def _exact_commit(case, s):
    P = case["page"]
    off, slots = s["row_offsets"].tolist(), s["slot_map"].tolist()
    src = list(range(len(slots)))
    if case["gather"]:
        picked = s["src_rows"].tolist()
        src = [picked[b][i] for b in range(case["batch"]) for i in range(off[b + 1] - off[b])]
    src = torch.tensor(src, device=DEV, dtype=torch.long)
    found = {}
    for name in ("k", "v"):
        x = s[name + "_new"].double()[src]
        if not case["fp8"]:
            pool = s[name + "_pool"].double()
            rows = pool.transpose(1, 2).reshape(-1, case["kv_heads"], case["head_dim"]).clone()
            rows[s["slot_map"]] = x
            found[name] = rows.view(pool.shape[0], P, case["kv_heads"], case["head_dim"]).transpose(1, 2)
            continue
        scales = s[name + "_scales"].double().clone()
        by_page = {}
        for r, t in enumerate(slots):
            by_page.setdefault(t // P, []).append(r)
        firsts = [p for p, rs in by_page.items() if any(slots[r] % P == 0 for r in rs)]
        for p in firsts:
            top = x[by_page[p]].abs().amax(dim=(0, 2))
            scales[p] = torch.where(top > 0, top / E4M3_MAX, torch.ones_like(top))
        # the codes themselves are roundings: a value near the middle of two codes has no definite one in 64 bits
        found[name], found[name + "_scales"] = None, scales
    return found


def exact(case, seed):
    if case["op"] == "attn_tree":
        s = _prepare_attn(case, seed)
        return _exact_attn(case, s)
    if case["op"] == "rows_commit":
        return _exact_commit(case, _prepare_commit(case, seed))
    return None                                                             # whole numbers only
