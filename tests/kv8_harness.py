"""Waves over a cache held in 8 bits, on cuda:0 through the library and in 64 bits through the oracle."""
import numpy as np
import torch

import paper_2609_35263_b200 as wpp
from oracle import kv8 as okv8

from .kv4_harness import ctx


class Wave:
    """Requests with pages of their own in a shuffled pool of normal rows, blocks of unequal scales."""

    def __init__(self, prefix, chunks, Hq, Hkv, d, B, seed=0, spare=3, sm_scale=0.0, scales=(-8, -3)):
        rng = np.random.default_rng(seed)
        self.P, self.C = np.asarray(prefix, np.int32), np.asarray(chunks, np.int32)
        self.Hq, self.Hkv, self.d, self.B, self.sm_scale = Hq, Hkv, d, B, sm_scale
        blocks = (self.P.astype(int) + self.C + B - 1) // B
        self.pages = int(blocks.sum()) + spare
        perm = rng.permutation(self.pages)
        self.table = np.full((len(self.P), max(1, int(blocks.max(initial=0)))), -1, np.int32)
        at = 0
        for i, n in enumerate(blocks):
            self.table[i, :n] = perm[at:at + n]
            at += n
        self.T = int(self.C.sum())
        bits = lambda *shape: okv8.bf16_bits(rng.standard_normal(shape).astype(np.float32))
        self.q, self.k_new, self.v_new = bits(self.T, Hq, d), bits(self.T, Hkv, d), bits(self.T, Hkv, d)
        self.k_pool, self.v_pool = self._pool(rng, (-8, -6)), self._pool(rng, scales)

    def _pool(self, rng, scales):
        """Codes of normal numbers of size 64, and any number in a block's last twelve bytes."""
        pool = rng.integers(0, 256, (self.pages, self.Hkv, self.B * self.d + 16)).astype(np.uint8)
        pool[..., :self.B * self.d] = okv8.encode(64 * rng.standard_normal((self.pages, self.Hkv, self.B * self.d)))
        e = rng.integers(scales[0], scales[1] + 1, (self.pages, self.Hkv, 1))
        pool[..., self.B * self.d:self.B * self.d + 4] = (2.0 ** e).astype(np.float32).view(np.uint8)
        return pool

    def desc(self, **kw):
        return wpp.make_desc(len(self.P), self.Hq, self.Hkv, self.d, self.B, self.table.shape[1], self.pages, sm_scale=self.sm_scale,
                             dtype=wpp.WPP_KV8, **kw)

    def plan(self, opts=None, **kw):
        return wpp.wpp_plan_tiles(ctx(), self.desc(**kw), self.P, self.C, opts=opts).to_device()

    def device(self):
        bf = lambda x: torch.from_numpy(x.view(np.int16).copy()).cuda().view(torch.bfloat16)
        dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
        return dict(q=bf(self.q), k_new=bf(self.k_new), v_new=bf(self.v_new), k=dev(self.k_pool), v=dev(self.v_pool),
                    table=dev(self.table), P=dev(self.P), C=dev(self.C), status=torch.zeros(1, dtype=torch.int32, device="cuda"))

    def attend(self, g, plan=None, opts=None, lse=True, workspace=None, **kw):
        plan = plan or self.plan(opts, **kw)
        out = torch.full((self.T, self.Hq, self.d), float("nan"), dtype=torch.bfloat16, device="cuda")
        sums = torch.full((self.T, self.Hq), float("nan"), dtype=torch.float32, device="cuda") if lse else None
        ws = workspace if workspace is not None else torch.full((int(plan.info.workspace_bytes),), 255, dtype=torch.uint8, device="cuda")
        wpp.wpp_prefill_attention_varlen(ctx(), self.desc(**kw), g["q"], out, sums, g["k"], g["v"], g["table"], g["P"], g["C"], plan,
                                         workspace=ws, status=g["status"])
        return out, sums

    def append(self, g, plan=None, **kw):
        wpp.wpp_kv_append(ctx(), self.desc(**kw), g["k_new"], g["v_new"], g["k"], g["v"], g["table"], g["P"], g["C"],
                          plan or self.plan(**kw), status=g["status"])

    def appended(self):
        """The pools after the wave's append, by the oracle (kept in place of the ones before)."""
        self.k_pool, self.v_pool = okv8.append(self.k_new, self.v_new, self.k_pool, self.v_pool, self.table, self.P, self.C, self.B)
        return self.k_pool, self.v_pool

    def reference(self):
        return okv8.attention(okv8.bf16_values(self.q).astype(np.float64), self.k_pool, self.v_pool, self.table, self.P, self.C, self.B,
                              self.Hkv, self.sm_scale)

    def reach(self):
        """Per request row and head, at most: the sum of scale |q_e k_e|, and what an error of 2^-18 of the row's largest |q| in every q_e
        does to a score."""
        scale = self.sm_scale if self.sm_scale > 0 else self.d ** -0.5
        ks = float(np.nanmax(np.ascontiguousarray(self.k_pool[..., self.B * self.d:self.B * self.d + 4]).view(np.float32)))     # (of pages that are named)
        q = np.abs(okv8.bf16_values(self.q).astype(np.float64))
        return scale * 448.0 * ks * q.sum(-1), scale * 448.0 * ks * self.d * q.max(-1) * 2.0 ** -18

    def check(self, out, sums, ref):
        """lse: a score is a sum of d exact products in fp32, each addition off by 2^-23 (truncated) of at most `reach`, in some
        16 steps; queries may be taken with an error of 2^-18 of the row's largest; then a few roundings of z.
        out: rounded once (2^-8 of it); p rounded to bf16 (2^-8 of the terms, whose sizes add up to `spread`) or to f16 (less, but
        2^-23 of the row's largest p where p is far below it: `even`), and off by what the scores are off (dz, relative), in
        numerator and denominator."""
        o, z, spread, even = ref
        reach, of_q = self.reach()
        ztol = 16 * 2.0 ** -23 * (reach + np.abs(z) + 16) + of_q
        if sums is not None:
            dz = np.abs(sums.double().cpu().numpy() - z)
            assert np.all(dz <= ztol), float((dz / ztol).max())
        got = out.double().cpu().numpy()
        tol = 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 2.0 ** -18 + 2 * ztol[..., None]) * spread + 2.0 ** -23 * even + 1e-30
        assert np.all(np.abs(got - o) <= tol), float((np.abs(got - o) / tol).max())
