"""Inputs shared by the tests of the drafted-token calls."""
import numpy as np
import torch

import paper_2512_16822_b200 as M
from paper_2512_16822_b200 import runtime as RT
from mepic_inputs import f32_to_bf16_bits, bf16_bits_to_f64
from oracle import mepic_oracle as O


def dev32(a, device="cuda:0"):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(device)


def random_parents(rng, n, kind="tree"):
    if kind == "chain":
        return np.arange(n) - 1
    if kind == "star":
        return np.full(n, -1)
    return np.array([max(-1, i - 1 - int(rng.integers(0, 6))) for i in range(n)], dtype=np.int64)


class TreeCase:
    """specs: per request (kv_len, n_rows).  Pages are a random permutation with gaps; position bases are jittered."""

    def __init__(self, seed, *, Hq, Hkv, D, P, specs, theta=1e4, kind="tree", jitter=True, fp8=False, stride_extra=0, scale=1.0):
        rng = self.rng = np.random.default_rng(seed)
        self.Hq, self.Hkv, self.D, self.P, self.theta, self.fp8 = Hq, Hkv, D, P, theta, fp8
        self.kv_len = np.array([k for k, _ in specs], dtype=np.int32)
        self.rows = np.array([n for _, n in specs], dtype=np.int64)
        self.off = np.concatenate([[0], np.cumsum(self.rows)]).astype(np.int32)
        B, ents = len(specs), -(-self.kv_len // P)
        self.num_pages = int(ents.sum()) + 5
        perm = rng.permutation(self.num_pages)
        stride = max(1, int(ents.max()) + 2)
        self.page_ids = np.full((B, stride), -7, dtype=np.int32)
        self.pos_base = np.full((B, stride), 1 << 30, dtype=np.int32)
        at = 0
        for b in range(B):
            self.page_ids[b, :ents[b]] = perm[at:at + ents[b]]
            at += int(ents[b])
            base = np.arange(ents[b]) * P
            if jitter and ents[b]:
                base = base + np.cumsum(rng.integers(0, 30, size=ents[b]))
            self.pos_base[b, :ents[b]] = base
        bits = lambda shape, std=1.0: f32_to_bf16_bits((rng.standard_normal(shape) * std).astype(np.float32))
        total = int(self.off[-1])
        self.kp, self.vp = bits((self.num_pages, Hkv, P, D)), bits((self.num_pages, Hkv, P, D))
        self.pad = stride_extra                                 # elements between the fused rows
        self.q, self.kn, self.vn = bits((total, Hq, D), scale), bits((total, Hkv, D)), bits((total, Hkv, D))
        self.parents, self.row_pos, self.sees = [], [], []
        for b in range(B):
            p = random_parents(rng, int(self.rows[b]), kind)
            n = int(self.kv_len[b])
            nxt = 0 if n == 0 else int(self.pos_base[b, (n - 1) // P]) + (n - 1) % P + 1
            pos, sees = O.tree_layout(p, nxt)
            self.parents.append(p), self.row_pos.append(pos), self.sees.append(sees)
        self.words = max(1, -(-int(self.rows.max()) // 32))
        self.max_position = max([int(x) for p in self.row_pos for x in p] + [64, P]) + 1
        self.cfg = M.Config(P, Hq, Hkv, D, self.num_pages, self.max_position, theta)

    def mask(self):
        return np.concatenate([O.pack_mask(s, self.words) for s in self.sees]) if self.off[-1] else np.zeros((0, self.words), np.int32)

    def device(self):
        self.dev = RT.Device(self.cfg, self.kp, self.vp)
        self.pools = RT.Fp8Pools(self.dev) if self.fp8 else None
        return self.dev

    def fused(self):
        """q, k_new, v_new as slices of one tensor whose rows lie further apart than they need to."""
        total, w = int(self.off[-1]), (self.Hq + 2 * self.Hkv) * self.D + self.pad
        buf = torch.full((total, w), float("nan"), dtype=torch.bfloat16, device="cuda:0")
        a, b = self.Hq * self.D, (self.Hq + self.Hkv) * self.D
        c = (self.Hq + 2 * self.Hkv) * self.D
        buf[:, :a] = RT.bf16_tensor(self.q, "cuda:0").view(total, -1)
        buf[:, a:b] = RT.bf16_tensor(self.kn, "cuda:0").view(total, -1)
        buf[:, b:c] = RT.bf16_tensor(self.vn, "cuda:0").view(total, -1)
        return buf[:, :a].unflatten(1, (self.Hq, self.D)), buf[:, a:b].unflatten(1, (self.Hkv, self.D)), buf[:, b:c].unflatten(1, (self.Hkv, self.D))

    def batch(self, max_rows=None, rows=None):
        q, k, v = rows if rows is not None else self.fused()
        self.d_kv = dev32(self.kv_len)
        return RT.TreeBatch(self.dev, q=q, k_new=k, v_new=v, row_offsets=dev32(self.off),
                            row_pos=dev32(np.concatenate(self.row_pos)), tree_mask=dev32(self.mask()), page_ids=dev32(self.page_ids),
                            pos_base=dev32(self.pos_base), kv_len=self.d_kv, max_rows=int(self.rows.max()) if max_rows is None else max_rows,
                            pools=self.pools)

    def want(self, b, sm_scale):
        kp, vp = self.kp, self.vp
        if self.fp8:
            if not hasattr(self, "_deq"):
                ks, vs = self.pools.k_scales.cpu().numpy(), self.pools.v_scales.cpu().numpy()
                self._deq = (O.dequantize_pages(self.pools.k_codes.cpu().numpy(), ks), O.dequantize_pages(self.pools.v_codes.cpu().numpy(), vs))
            kp, vp = self._deq
        r = slice(self.off[b], self.off[b + 1])
        return O.tree_attention_one(self.q[r], self.kn[r], self.vn[r], self.row_pos[b], self.sees[b], kp, vp, self.page_ids[b],
                                    self.pos_base[b], int(self.kv_len[b]), sm_scale, self.theta)

    def check(self, out, sm_scale, which=None):
        """|err| <= 7 sigma + 1e-4 (V ~ N(0,1)): seven standard deviations of the once-rounded operands' error (the sum of many bounded
        independent terms: beyond 7 with probability under 1e-10 per element), and fp32 sums, ex2 and (cos, sin) steps."""
        got = bf16_bits_to_f64(RT.bf16_bits(out))
        for b in range(len(self.rows)) if which is None else which:
            if self.rows[b] == 0:
                continue
            want, sigma = self.want(b, sm_scale)
            g = got[self.off[b]:self.off[b + 1]]
            assert np.isfinite(g).all(), f"request {b}"
            err, tol = np.abs(g - want), 7 * sigma + 1e-4
            bad = err > tol
            assert not bad.any(), (f"request {b}: {int(bad.sum())} of {bad.size}", np.argwhere(bad)[:4].tolist(), float((err / tol).max()))
            empty = np.array([self.kv_len[b] == 0 and not s.any() for s in self.sees[b]])
            assert (g[empty] == 0).all()
