"""Waves over a cache held in 4 bits, on cuda:0 through the library and in 64 bits through the oracle."""
import numpy as np
import torch

import paper_2609_35263_b200 as wpp
from oracle import kv4 as okv4

_CTX = None


def ctx():
    global _CTX
    if _CTX is None:
        _CTX = wpp.Context(0)
    return _CTX


class Wave:
    """Requests with pages of their own in a shuffled pool whose blocks hold packed normal rows."""

    def __init__(self, prefix, chunks, Hq, Hkv, d, B, seed=0, spare=3, sm_scale=0.0):
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
        bits = lambda *shape: okv4.bf16_bits(rng.standard_normal(shape).astype(np.float32))
        self.q, self.k_new, self.v_new = bits(self.T, Hq, d), bits(self.T, Hkv, d), bits(self.T, Hkv, d)
        self.k_pool, self.v_pool = self._pool(rng), self._pool(rng)

    def _pool(self, rng):
        codes, pairs = okv4.pack_rows(okv4.bf16_bits(rng.standard_normal((self.pages, self.Hkv, self.B, self.d)).astype(np.float32)))
        codes = (codes[..., 0::2] | codes[..., 1::2] << 4).reshape(self.pages, self.Hkv, -1)
        return np.concatenate([codes, pairs.view(np.uint8).reshape(self.pages, self.Hkv, -1)], -1)

    def desc(self, **kw):
        return wpp.make_desc(len(self.P), self.Hq, self.Hkv, self.d, self.B, self.table.shape[1], self.pages, sm_scale=self.sm_scale,
                             dtype=wpp.WPP_KV4, **kw)

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

    def reference(self):
        return okv4.attention(okv4.bf16_values(self.q).astype(np.float64), self.k_pool, self.v_pool, self.table, self.P, self.C, self.B,
                              self.Hkv, self.sm_scale)

    def check(self, out, sums, ref):
        """out: rounded once (2^-8 of it); p and v rounded to bf16 before they are multiplied (2^-8 each of the terms, whose
        sizes add up to `spread`); fp32 work on the scores: an eighth of 2^-8 of `spread` more covers errors of p up to 4e-4.
        lse: fp32 sums of q times (128 + code), 16 roundings and truncations of 2^-23 of at most 143 scale sum |q|, and of the
        result."""
        o, z, spread = ref
        got = out.double().cpu().numpy()
        tol = 2.0 ** -8 * (np.abs(o) + 2.125 * spread) + 1e-30
        assert np.all(np.abs(got - o) <= tol), float((np.abs(got - o) / tol).max())
        if sums is not None:
            scale = self.sm_scale if self.sm_scale > 0 else self.d ** -0.5
            at = self.B * (self.d // 2)
            ks = okv4.bf16_values(np.ascontiguousarray(self.k_pool[..., at:]).view(np.uint16))[..., 1::2]
            ks = float(np.nanmax(np.abs(np.where(np.isfinite(ks), ks, np.nan))))
            reach = 143.0 * ks * np.abs(okv4.bf16_values(self.q).astype(np.float64)).sum(-1) * scale
            ztol = 16 * 2.0 ** -23 * (reach + np.abs(z) + 16)
            dz = np.abs(sums.double().cpu().numpy() - z)
            assert np.all(dz <= ztol), float((dz / ztol).max())
