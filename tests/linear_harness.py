"""Waves of the linear-attention layer, on cuda:0 through the library and in 64 bits through the oracle."""
import numpy as np
import torch

import paper_2609_35263_b200 as wpp
from oracle import linear as olinear

_CTX = None


def ctx():
    global _CTX
    if _CTX is None:
        _CTX = wpp.Context(0)
    return _CTX


class Wave:
    def __init__(self, chunks, H, d, seed=0, per_token=True, prefix=None, interval=0, scale=1.0, decay=None, resume=True):
        rng = np.random.default_rng(seed)
        R, self.H, self.d, self.scale, self.interval = len(chunks), H, d, scale, interval
        self.C = np.asarray(chunks, np.int64)
        self.P = np.zeros(R, np.int32) if prefix is None else np.asarray(prefix, np.int32)
        self.T = int(self.C.sum())
        bf = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).bfloat16()
        self.q, self.k, self.v = bf(self.T, H, d), bf(self.T, H, d) * d ** -0.5, bf(self.T, H, d)
        if decay is None:
            decay = -np.exp(rng.uniform(-6, 0.5, (self.T, H) if per_token else H))
        self.decay = torch.from_numpy(np.asarray(decay, np.float32))
        counts = (self.P + self.C) // interval - self.P // interval if interval else np.zeros(R, int)
        self.snaps = np.full((R, max(1, int(counts.max(initial=0)))), -1, np.int32)
        slots = 2 * R
        for i in range(R):
            self.snaps[i, :counts[i]] = slots + np.arange(counts[i])
            slots += int(counts[i])
        self.pool = torch.from_numpy(rng.standard_normal((max(1, slots), H, d, d)).astype(np.float32))
        self.state_in = np.arange(R, dtype=np.int32) if resume else np.full(R, -1, np.int32)
        self.state_out = np.arange(R, 2 * R, dtype=np.int32)

    def device(self):
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()
        return dict(q=self.q.cuda(), k=self.k.cuda(), v=self.v.cuda(), decay=self.decay.cuda(), pool=self.pool.cuda(),
                    rows=torch.from_numpy(np.concatenate([[0], np.cumsum(self.C)]).astype(np.int64)).cuda(), state_in=i32(self.state_in),
                    state_out=i32(self.state_out), prefix=i32(self.P), snaps=i32(self.snaps) if self.interval else None,
                    status=torch.zeros(1, dtype=torch.int32, device="cuda"))

    def workspace(self):
        n = wpp.wpp_linear_workspace_bytes(len(self.C), self.H, self.d, self.T)
        return torch.full((n,), 255, dtype=torch.uint8, device="cuda")

    def run(self, g, layout=0, out=None, **kw):
        if out is None:
            out = torch.full((self.T, self.H, self.d), float("nan"), dtype=torch.bfloat16, device="cuda")
        if "workspace" not in kw:
            kw["workspace"] = None if layout == 1 else self.workspace()
        return wpp.wpp_linear_chunk(ctx(), g["q"], g["k"], g["v"], g["decay"], g["rows"], g["pool"], g["state_in"], g["state_out"], out=out,
                                    prefix_lens=g["prefix"], snap_interval=self.interval, snap_slots=g["snaps"], status=g["status"],
                                    layout=layout, scale=self.scale, **kw)

    def reference(self):
        pool = self.pool.double().numpy().copy()
        f = lambda x: x.double().numpy()
        o, size = olinear.linear_chunk(f(self.q), f(self.k), f(self.v), f(self.decay), self.C, pool, self.state_in, self.state_out, self.P,
                                       self.interval, self.snaps if self.interval else None, self.scale)
        return o, size, pool

    def check(self, out, pool, ref):
        """Outputs: rounded once (2^-8), from terms of which some are products of numbers rounded to bf16 or f16 before (2^-8 of a
        term, of terms whose sizes add up to `size`).  States: fp32 sums of products whose one factor is held in 16 bits or more
        (2^-16), and of decays from logarithms (2^-20), which a state's terms have at most once: 2^-15 of the largest entries."""
        o, size, want = ref
        got = out.double().cpu().numpy()
        assert np.all(np.abs(got - o) <= 2.0 ** -8 * (np.abs(o) + size) + 1e-30), float(np.nanmax(np.abs(got - o) / (2.0 ** -8 * (np.abs(o) + size) + 1e-30)))
        diff = np.abs(pool.double().cpu().numpy() - want)
        top = np.abs(want).max((2, 3), keepdims=True)
        assert np.all(diff <= 2.0 ** -15 * top), float((diff / (2.0 ** -15 * top + 1e-300)).max())
