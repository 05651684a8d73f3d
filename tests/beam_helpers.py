"""Inputs and plain statements shared by the tests of the beam calls."""
import math

import numpy as np
import torch

import paper_2512_16822_b200 as M
from paper_2512_16822_b200 import runtime as RT
from mepic_inputs import f32_to_bf16_bits, bf16_bits_to_f64
from oracle import mepic_oracle as O

NAN_BITS = 0x7fc0


def dev32(a, device="cuda:0"):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(device)


class BeamCase:
    """specs: per group (context, grown): `width` beams share the context's full pages; from there on the beams are re-drawn from one
    another at every page.  Pages lie anywhere in the pool, position bases are jittered, what nobody holds is NaN."""

    def __init__(self, seed, *, Hq, Hkv, D, P, width, specs, theta=1e4, fp8=False, lens=None, scale=1.0, extra_pages=5):
        rng = self.rng = np.random.default_rng(seed)
        self.Hq, self.Hkv, self.D, self.P, self.W, self.theta, self.fp8 = Hq, Hkv, D, P, width, theta, fp8
        n = len(specs)
        total = np.array([c + g for c, g in specs])
        ents = -(-total // P)
        stride = max(1, int(ents.max())) + 2
        tables = np.full((n, width, stride), -7, dtype=np.int64)
        base = np.full((n, width, stride), 1 << 30, dtype=np.int64)
        used = 0
        for b, (context, _) in enumerate(specs):
            full = min(context // P, int(ents[b]))
            tables[b, :, :full] = used + np.arange(full)
            used += full
            for e in range(full, int(ents[b])):
                tables[b] = tables[b, rng.integers(0, width, size=width)]
                tables[b, :, e] = used + np.arange(width)
                used += width
            base[b, :, :ents[b]] = np.arange(ents[b]) * P + np.cumsum(rng.integers(0, 30, size=ents[b]))
        self.num_pages = used + extra_pages
        perm = rng.permutation(self.num_pages)
        self.page_ids = np.where(tables >= 0, perm[np.maximum(tables, 0)], -7).reshape(n * width, stride).astype(np.int32)
        self.pos_base = base.reshape(n * width, stride).astype(np.int32)
        self.kv_len = (np.repeat(total, width) if lens is None else np.asarray(lens)).astype(np.int32)
        bits = lambda shape, std=1.0: f32_to_bf16_bits((rng.standard_normal(shape) * std).astype(np.float32))
        self.kp, self.vp = bits((self.num_pages, Hkv, P, D)), bits((self.num_pages, Hkv, P, D))
        self.q = bits((n * width, Hq, D), scale)
        self.finish()

    def finish(self):
        """q_pos, rope table size and config follow from the tables as they are now."""
        last = np.maximum(self.kv_len - 1, 0)
        pos = self.pos_base[np.arange(len(self.kv_len)), last // self.P].astype(np.int64) + last % self.P
        self.q_pos = np.where(self.kv_len > 0, pos, 0)
        self.max_position = max(64, self.P, int(self.q_pos.max())) + 1
        self.cfg = M.Config(self.P, self.Hq, self.Hkv, self.D, self.num_pages, self.max_position, self.theta)

    def poison(self):
        """NaN in every slot that no row's length reaches."""
        fill = np.zeros(self.num_pages, dtype=np.int64)
        for r, n in enumerate(self.kv_len):
            for e in range(-(-int(n) // self.P)):
                p = self.page_ids[r, e]
                fill[p] = max(fill[p], min(self.P, int(n) - e * self.P))
        for p in range(self.num_pages):
            self.kp[p, :, fill[p]:] = NAN_BITS
            self.vp[p, :, fill[p]:] = NAN_BITS

    def device(self):
        self.dev = RT.Device(self.cfg, self.kp, self.vp)
        self.pools = RT.Fp8Pools(self.dev) if self.fp8 else None
        self.d_ids, self.d_base, self.d_len, self.d_qpos = dev32(self.page_ids), dev32(self.pos_base), dev32(self.kv_len), dev32(self.q_pos)
        return self.dev

    def fused_q(self, pad=8):
        """q as a slice of rows that lie further apart than they need to."""
        w = self.Hq * self.D
        buf = torch.full((len(self.q), w + pad), float("nan"), dtype=torch.bfloat16, device="cuda:0")
        buf[:, :w] = RT.bf16_tensor(self.q, "cuda:0").view(len(self.q), -1)
        return buf[:, :w].unflatten(1, (self.Hq, self.D))

    def batch(self, q=None):
        self.plan = RT.BeamPlan(self.dev, page_ids=self.d_ids, pos_base=self.d_base, kv_len=self.d_len, width=self.W)
        self.attn = RT.BeamBatch(self.dev, q=self.fused_q() if q is None else q, q_pos=self.d_qpos, plan=self.plan, pools=self.pools)
        return self.attn

    def run(self, sm_scale):
        self.plan.run()
        return self.attn.run(sm_scale)

    def want(self, r, sm_scale):
        kp, vp = self.kp, self.vp
        if self.fp8:
            if not hasattr(self, "_deq"):
                with np.errstate(all="ignore"):
                    ks, vs = self.pools.k_scales.cpu().numpy(), self.pools.v_scales.cpu().numpy()
                    self._deq = (O.dequantize_pages(self.pools.k_codes.cpu().numpy(), ks), O.dequantize_pages(self.pools.v_codes.cpu().numpy(), vs))
            kp, vp = self._deq
        none = np.zeros((1, self.Hkv, self.D))
        out, sigma = O.tree_attention_one(self.q[r:r + 1], none, none, [int(self.q_pos[r])], np.zeros((1, 1), dtype=bool), kp, vp, self.page_ids[r],
                                          self.pos_base[r], int(self.kv_len[r]), sm_scale, self.theta)
        return out[0], sigma[0]

    def check(self, out, sm_scale, which=None):
        """|err| <= 7 sigma + 1e-4 (V ~ N(0,1)): seven standard deviations of the error that rounding the rotated q and K, the weights and
        the output to bf16 once each makes (the sum of many bounded independent terms: beyond 7 with probability under 1e-10 an
        element), and fp32 sums, ex2 and the table's (cos, sin).  8-bit pages round to fp16 instead: inside the same bound."""
        got = bf16_bits_to_f64(RT.bf16_bits(out))
        for r in range(len(self.kv_len)) if which is None else which:
            if self.kv_len[r] == 0:
                assert (got[r] == 0).all(), f"row {r}"
                continue
            want, sigma = self.want(r, sm_scale)
            assert np.isfinite(got[r]).all(), f"row {r}"
            err, tol = np.abs(got[r] - want), 7 * sigma + 1e-4
            bad = err > tol
            assert not bad.any(), (f"row {r} (len {self.kv_len[r]}): {int(bad.sum())} of {bad.size}", np.argwhere(bad)[:4].tolist(), float((err / tol).max()))


# ------------------------------------------------------------------ selection, in 64 bits
def select_group(logits, score, done, K, eos, pad):
    """One group: logits [W, V] fp64 -> list of (score, beam, token, done), best first, and the status it sets."""
    W, V = logits.shape
    cand, bad = [], False
    for w in range(W):
        s = float(score[w])
        if math.isnan(s) or s == math.inf:
            bad = True
            continue
        if s == -math.inf:
            continue
        if done is not None and done[w]:
            cand.append((np.array([s]), w, np.array([pad])))
            continue
        x = logits[w]
        if np.isnan(x).any() or (x == math.inf).any():
            bad = True
            continue
        top = x.max()
        if top == -math.inf:
            continue
        lse = top + math.log(np.exp(x - top).sum())
        tokens = np.nonzero(x > -math.inf)[0]
        cand.append((s + (x[tokens] - lse), w, tokens))
    if not cand:
        return [], bad
    val = np.concatenate([c[0] for c in cand])
    beam = np.concatenate([np.full(len(c[0]), c[1]) for c in cand])
    token = np.concatenate([c[2] for c in cand])
    order = np.lexsort((token, beam, -val))[:K + 1]
    return [(float(val[i]), int(beam[i]), int(token[i]), int(bool(done is not None and done[beam[i]]) or token[i] == eos)) for i in order], bad


# ------------------------------------------------------------------ fork, entry by entry
def fork(parent, kv_len, page_ids, pos_base, owned, reserve, used, P):
    """parent [G, Wo], rows [G * Wi] -> dict as BeamFork.run gives, with page_ids/pos_base as lists per row and the reserve."""
    G, Wo = parent.shape
    Wi = len(kv_len) // G
    freed, copies, rows = [], [], []
    for g in range(G):
        tab = [[int(p) for p in page_ids[g * Wi + w, :-(-int(kv_len[g * Wi + w]) // P)]] for w in range(Wi)]
        bas = [[int(p) for p in pos_base[g * Wi + w, :len(tab[w])]] for w in range(Wi)]
        new = [(list(tab[p]), list(bas[p]), int(kv_len[g * Wi + p])) if p >= 0 else ([], [], 0) for p in parent[g]]
        deepest = max([len(t) for t in tab] + [0])
        for e in range(deepest):
            held = {t[e] for t, _, _ in new if len(t) > e}
            for w in range(Wi):
                if len(tab[w]) > e and owned[tab[w][e]] and tab[w][e] not in held:
                    freed.append(tab[w][e])
                    held.add(tab[w][e])
        for k, (t, _, n) in enumerate(new):
            if n % P == 0:
                continue
            e, page = n // P, t[-1]
            others = [(j, m) for j, (u, _, m) in enumerate(new) if j != k and len(u) > e and u[e] == page]
            keeps = owned[page] and all(j > k and m < (e + 1) * P for j, m in others)
            if not keeps:
                copies.append((len(rows) + k, page, n % P))
        rows += [[list(t), list(b), n] for t, b, n in new]
    if used < 0 or used > len(reserve) or len(freed) > used:
        return dict(status=M.MEPIC_DEV_BAD_BEAM)
    if used - len(freed) + len(copies) > len(reserve):
        return dict(status=M.MEPIC_DEV_NO_PAGES)
    stack = list(reserve[:used - len(freed)]) + freed + list(reserve[used:])
    at = used - len(freed)
    out = []
    for i, (row, src, slots) in enumerate(copies):
        out.append((src, stack[at + i], slots))
        rows[row][0][-1] = stack[at + i]
    return dict(status=0, rows=rows, copies=out, reserve=stack, used=at + len(copies))
