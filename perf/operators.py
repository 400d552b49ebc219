"""Operators of a serving stage's two kinds of cache, as measurable cases.

  append   the K/V rows of a wave's new tokens into the pages of a cache held in 4 bits
  attend   attention of a wave's queries over such a cache: single tokens behind long contexts, and chunks of prompts
  linear   the linear-attention layer with a decay per head over a pool of recurrent states: chunks of prompts, resumed from
           and left in slots of the pool, and single tokens

A row (page, KV head, slot) of the 4-bit cache holds d codes of 4 bits and two bf16 numbers, its least value and its scale; it
stands for least + scale * code.  A block (page, KV head) is the codes of its rows and, behind them, their number pairs.  The
append's result is those bytes, defined to the bit, and is returned as the pools themselves.

Ragged lengths are drawn from the case's own `lengths` number, so that the work of a case is fixed; values and physical page
ids come from the seed.
"""
import math

import numpy as np
import torch

own = False

_TINY = 2.0 ** -100          # rows whose scale would be less stand for their least value alone
_CTX = {}


def _ctx():
    import paper_2609_35263_b200 as wpp
    dev = torch.cuda.current_device()
    if dev not in _CTX:
        _CTX[dev] = wpp.Context(dev)
    return _CTX[dev]


def _device():
    return torch.device("cuda", torch.cuda.current_device())


# ------------------------------------------------------------------------------------------------------------ cases
def _cache(name, kind, requests, chunk, prefix, heads, lengths=0, lse=False):
    """chunk, prefix: (least, most) tokens, uniform per request; heads: (query heads, KV heads, head_dim, page size)."""
    c = dict(kind=kind, requests=requests, chunk_min=chunk[0], chunk_max=chunk[1], prefix_min=prefix[0], prefix_max=prefix[1],
             q_heads=heads[0], kv_heads=heads[1], head_dim=heads[2], page_size=heads[3], lengths=lengths, lse=lse)
    return dict(c, name=name) if name else c


def _linear(name, requests, chunk, heads, head_dim, lengths=0, per_token=False, prefix=0, snap_interval=0):
    """per_token: a decay for each token and head (a gate's output) instead of one for each head."""
    c = dict(kind="linear", requests=requests, chunk_min=chunk[0], chunk_max=chunk[1], heads=heads, head_dim=head_dim,
             lengths=lengths, per_token=per_token, prefix=prefix, snap_interval=snap_interval)
    return dict(c, name=name) if name else c


_SMALL_HEADS, _MID_HEADS, _BIG_HEADS = (8, 2, 64, 16), (32, 8, 128, 64), (64, 8, 128, 64)


def listed():
    return [
        # a generation step's new rows: 64 requests, one token each, anywhere in their pages
        _cache("append_step", "append", 64, (1, 1), (0, 16384), _BIG_HEADS, lengths=1),
        # a prefill wave's new rows: 32 ragged chunks
        _cache("append_prompts", "append", 32, (256, 2048), (0, 8192), _BIG_HEADS, lengths=2),
        # one user alone, one token behind 8,192 cached ones: latency
        _cache("token_one_request", "attend", 1, (1, 1), (8191, 8191), _MID_HEADS),
        # a generation step of a full batch with contexts of all lengths
        _cache("token_batch_64", "attend", 64, (1, 1), (255, 16383), _BIG_HEADS, lengths=3),
        # a few very long documents, one token each
        _cache("token_long_context", "attend", 4, (1, 1), (131071, 131071), _BIG_HEADS),
        # two drafted tokens to be checked per request, groups of five heads, odd lengths, log-sums for a later merge
        _cache("two_tokens_groups_of_5", "attend", 24, (2, 2), (77, 3001), (40, 8, 128, 32), lengths=4, lse=True),
        # a small model's short chunks behind short prefixes
        _cache("chunks_small_heads", "attend", 12, (1, 300), (0, 700), _SMALL_HEADS, lengths=5, lse=True),
        # an ordinary ragged prefill wave
        _cache("prompts_ragged", "attend", 16, (256, 2048), (0, 8192), _MID_HEADS, lengths=6, lse=True),
        # a chunk of a long document
        _cache("prompt_behind_long_prefix", "attend", 1, (4096, 4096), (32768, 32768), _BIG_HEADS),
        # a linear layer's prefill wave over eight lanes, one decay per head
        _linear("linear_prompts", 8, (2048, 2048), 32, 128),
        # one long prompt with a gate's decays and periodic snapshots for later reuse
        _linear("linear_long_prompt", 1, (16384, 16384), 32, 128, per_token=True, prefix=65536, snap_interval=4096),
        # a generation step of the linear layer
        _linear("linear_step", 64, (1, 1), 32, 128, per_token=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what, lengths = rng.random(), rng.randrange(1, 1 << 30)
    heads = rng.choice([_SMALL_HEADS, _MID_HEADS, _BIG_HEADS, (32, 8, 128, 128), (16, 4, 64, 32), (40, 8, 128, 32), (32, 2, 128, 16), (8, 8, 64, 64)])
    if what < 0.15:
        hi = _log_int(rng, 1, 2048)
        return _cache(None, "append", max(1, min(_log_int(rng, 1, 128), 65536 // hi)), (max(1, hi // 3), hi), (0, _log_int(rng, 1, 16384)), heads,
                      lengths=lengths)
    if what < 0.45:
        hi = _log_int(rng, 1, 131071)
        return _cache(None, "attend", max(1, min(_log_int(rng, 1, 64), 524288 // hi)), (1, rng.choice([1, 1, 1, 2, 4])), (hi // rng.choice([1, 4, 100]), hi),
                      heads, lengths=lengths, lse=rng.random() < 0.3)
    if what < 0.7:
        hi = _log_int(rng, 5, 4096)
        case = _cache(None, "attend", _log_int(rng, 1, 32), (max(1, int(hi * rng.random())), hi), (0, 0) if rng.random() < 0.3 else (0, _log_int(rng, 16, 32768)),
                      heads, lengths=lengths, lse=rng.random() < 0.3)
        while case["requests"] > 1 and work(case)["flops"] > 2e12:
            case["requests"] //= 2
        return case
    hi = 1 if rng.random() < 0.25 else _log_int(rng, 2, 16384)
    return _linear(None, max(1, min(_log_int(rng, 1, 64), 16384 // hi)), (max(1, int(hi * rng.choice([1.0, 0.5, 0.01]))), hi), rng.choice([8, 16, 32]),
                   rng.choice([64, 128, 128]), lengths=lengths, per_token=rng.random() < 0.5, prefix=rng.randrange(0, 65537),
                   snap_interval=rng.choice([0, 0, 1024, 2500, 4096]))


# ----------------------------------------------------------------------------------------------------------- lengths
def _lengths(case):
    rng = np.random.default_rng(case["lengths"])
    n = case["requests"]
    C = rng.integers(case["chunk_min"], case["chunk_max"] + 1, n).astype(np.int64)
    P = rng.integers(case["prefix_min"], case["prefix_max"] + 1, n).astype(np.int64) if "prefix_min" in case else np.full(n, case["prefix"], np.int64)
    return C, P


def _offsets(C):
    return np.concatenate([[0], np.cumsum(C)]).astype(np.int64)


# ------------------------------------------------------------------------------------------------------- 4-bit blocks
def _pack(x):
    """Rows [..., B, d] as blocks of bytes [..., B * (d / 2 + 4)]."""
    x = x.float()
    least = x.amin(-1, keepdim=True) + 0.0                       # (a least value of -0 is +0)
    extent = x.amax(-1, keepdim=True) - least
    fine = torch.isfinite(extent)
    scale = (extent / 15).bfloat16().float()
    scale = torch.where(fine & (scale >= _TINY), scale, 0.0)
    code = torch.where(scale > 0, torch.round((x - least) / torch.where(scale > 0, scale, 1.0)), 0.0).to(torch.uint8)
    least = torch.where(fine, least, torch.nan)                  # a row with an infinity or a NaN stands for NaN
    codes = (code[..., 0::2] | code[..., 1::2] << 4).flatten(-2)
    pairs = torch.cat([least, scale], -1).bfloat16().view(torch.int16)
    pairs = torch.where(torch.cat([fine, torch.ones_like(fine)], -1), pairs, 0x7FC0).contiguous()
    return torch.cat([codes, pairs.view(torch.uint8).flatten(-2)], -1)


def _unpack(blocks, B, d, dtype):
    """The rows [..., B, d] that blocks of bytes stand for."""
    codes = blocks[..., :B * d // 2].unflatten(-1, (B, d // 2))
    pairs = blocks[..., B * d // 2:].contiguous().view(torch.bfloat16).unflatten(-1, (B, 2)).to(dtype)
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).to(dtype)
    return pairs[..., :1] + pairs[..., 1:] * code


def _prepare_cache(case, seed):
    C, P = _lengths(case)
    R, B, Hq, Hkv, d = case["requests"], case["page_size"], case["q_heads"], case["kv_heads"], case["head_dim"]
    T = int(C.sum())
    blocks = (P + C + B - 1) // B
    pages = int(blocks.sum()) + 8
    perm = np.random.default_rng(seed).permutation(pages).astype(np.int32)
    table = np.full((R, int(blocks.max())), -1, np.int32)
    at = 0
    for i in range(R):
        table[i, :blocks[i]] = perm[at:at + blocks[i]]
        at += int(blocks[i])
    dev = _device()
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape):
        return torch.empty(*shape, dtype=torch.bfloat16, device=dev).normal_(generator=gen)

    def pool():
        # keys and values of other tokens, channels of unequal size among them
        size = torch.exp(0.5 * torch.randn(Hkv, 1, d, device=dev, generator=gen)).bfloat16()
        step = max(1, (1 << 26) // (Hkv * B * d))
        return torch.cat([_pack(normal(min(step, pages - a), Hkv, B, d) * size) for a in range(0, pages, step)])

    s = dict(k_cache=pool(), v_cache=pool(), prefix=P.astype(np.int32), chunks=C.astype(np.int32), starts=_offsets(C))
    if case["kind"] == "append":
        s.update(k_new=normal(T, Hkv, d), v_new=normal(T, Hkv, d))
    else:
        s.update(q=normal(T, Hq, d), out=torch.empty(T, Hq, d, dtype=torch.bfloat16, device=dev),
                 log_sums=torch.empty(T, Hq, dtype=torch.float32, device=dev) if case["lse"] else None)
    s["table"], s["prefix_dev"], s["chunks_dev"] = (torch.from_numpy(x).to(dev) for x in (table, s["prefix"], s["chunks"]))
    s["status"] = torch.zeros(1, dtype=torch.int32, device=dev)
    if own:
        import paper_2609_35263_b200 as wpp
        s["desc"] = wpp.make_desc(R, Hq, Hkv, d, B, table.shape[1], pages, dtype=wpp.WPP_KV4)
        s["plan"] = wpp.wpp_plan_tiles(_ctx(), s["desc"], s["prefix"], s["chunks"]).to_device(dev)
        s["workspace"] = torch.empty(int(s["plan"].info.workspace_bytes), dtype=torch.uint8, device=dev)
    return s


# --------------------------------------------------------------------------------------------------------------- append
def _run_append(case, s):
    if own:
        import paper_2609_35263_b200 as wpp
        wpp.wpp_kv_append(_ctx(), s["desc"], s["k_new"], s["v_new"], s["k_cache"], s["v_cache"], s["table"], s["prefix_dev"],
                          s["chunks_dev"], s["plan"], status=s["status"])
        return dict(k_cache=s["k_cache"], v_cache=s["v_cache"])
    B, Hkv, d, T = case["page_size"], case["kv_heads"], case["head_dim"], int(s["starts"][-1])
    dev = s["table"].device
    request = torch.repeat_interleave(torch.arange(case["requests"], device=dev), s["chunks_dev"].long(), output_size=T)
    starts = torch.cumsum(s["chunks_dev"], 0) - s["chunks_dev"]
    pos = s["prefix_dev"][request] + torch.arange(T, device=dev) - starts[request]
    page, slot = s["table"][request, pos // B].long(), pos % B
    for new, cache in ((s["k_new"], s["k_cache"]), (s["v_new"], s["v_cache"])):
        rows = _pack(new.unsqueeze(2))                                                   # [T, Hkv, d / 2 + 4]
        codes = cache.view(-1, Hkv, B * (d // 2 + 4))[..., :B * d // 2].unflatten(-1, (B, d // 2))
        pairs = cache.view(-1, Hkv, B * (d // 2 + 4))[..., B * d // 2:].unflatten(-1, (B, 4))
        codes[page, :, slot] = rows[..., :d // 2]
        pairs[page, :, slot] = rows[..., d // 2:]
    return dict(k_cache=s["k_cache"], v_cache=s["v_cache"])


# -------------------------------------------------------------------------------------------------------------- attend
_MOST_SCORES = 1 << 30          # of the plain form at a time


def _attend_plain(case, s, some, rows):
    """Rows `rows` of the chunks of the requests `some`: (out, log-sums), padded to the longest."""
    B, Hq, Hkv, d = case["page_size"], case["q_heads"], case["kv_heads"], case["head_dim"]
    dev = s["table"].device
    last = int((s["prefix"][some] + np.minimum(s["chunks"][some], rows.stop)).max())
    table = s["table"][some, :(last + B - 1) // B].clamp(min=0).long()
    k, v = (_unpack(c[table], B, d, torch.float32).transpose(1, 2).flatten(2, 3) for c in (s["k_cache"], s["v_cache"]))      # [r, Hkv, keys, d]
    t = torch.arange(rows.start, rows.stop, device=dev)
    starts = torch.from_numpy(s["starts"][:-1][some]).to(dev)
    at = (starts[:, None] + t).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][at].float().unflatten(2, (Hkv, Hq // Hkv)).permute(0, 2, 3, 1, 4).flatten(2, 3)                               # [r, Hkv, G * rows, d]
    score = (q @ k.transpose(2, 3)).mul_(d ** -0.5).unflatten(2, (Hq // Hkv, -1))
    seen = torch.arange(k.shape[2], device=dev) <= (s["prefix_dev"][some, None] + t)[..., None]                              # [r, rows, keys]
    score.masked_fill_(~seen[:, None, None], -torch.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    v = v.masked_fill(~seen.any(1)[:, None, :, None], 0.0)                    # what no row sees may hold anything
    out = (score.flatten(2, 3) @ v).unflatten(2, (Hq // Hkv, -1)) / total
    return out.permute(0, 3, 1, 2, 4).flatten(2, 3), (top + total.log()).squeeze(-1).permute(0, 3, 1, 2).flatten(2, 3)


def _slices(case, s):
    """Requests and rows that the plain form takes at a time."""
    C, N = s["chunks"].astype(np.int64), (s["prefix"] + s["chunks"]).astype(np.int64)
    if len(C) * int(C.max()) * int(N.max()) * case["q_heads"] <= _MOST_SCORES and len(C) * int(N.max()) * case["kv_heads"] * case["head_dim"] <= _MOST_SCORES:
        return [(slice(0, len(C)), range(0, int(C.max())))]
    step = [max(1, _MOST_SCORES // int(n * case["q_heads"])) for n in N]
    return [(slice(i, i + 1), range(a, min(a + step[i], int(C[i])))) for i in range(len(C)) for a in range(0, int(C[i]), step[i])]


def _run_attend(case, s):
    if own:
        import paper_2609_35263_b200 as wpp
        wpp.wpp_prefill_attention_varlen(_ctx(), s["desc"], s["q"], s["out"], s["log_sums"], s["k_cache"], s["v_cache"], s["table"],
                                         s["prefix_dev"], s["chunks_dev"], s["plan"], workspace=s["workspace"], status=s["status"])
        return dict(out=s["out"], lse=s["log_sums"])
    for some, rows in _slices(case, s):
        out, log_sums = _attend_plain(case, s, some, rows)
        there = torch.arange(rows.start, rows.stop, device=out.device) < s["chunks_dev"][some, None]
        at = (torch.from_numpy(s["starts"][:-1][some]).to(out.device)[:, None] + torch.arange(rows.start, rows.stop, device=out.device))[there]
        s["out"][at] = out[there].bfloat16()
        if s["log_sums"] is not None:
            s["log_sums"][at] = log_sums[there]
    return dict(out=s["out"], lse=s["log_sums"])


def _exact_attend(case, seed):
    s = _prepare_cache(case, seed)
    B, Hq, Hkv, d = case["page_size"], case["q_heads"], case["kv_heads"], case["head_dim"]
    if work(case)["flops"] > 2e13:
        return None
    G, outs, sums = Hq // Hkv, [], []
    for i in range(case["requests"]):
        P, C, r0 = int(s["prefix"][i]), int(s["chunks"][i]), int(s["starts"][i])
        pos = torch.arange(P + C, device=s["q"].device)
        page, slot = s["table"][i].long()[pos // B], pos % B

        def rows(cache):
            # byte by byte: codes of row `slot` at slot * d / 2, its two numbers behind all codes
            b = cache[page]                                                                                       # [keys, Hkv, bytes]
            at = (slot[:, None] * (d // 2) + torch.arange(d // 2, device=b.device))[:, None].expand(-1, Hkv, -1)
            byte = torch.gather(b, 2, at).long()
            at = (B * d // 2 + slot[:, None] * 4 + torch.arange(4, device=b.device))[:, None].expand(-1, Hkv, -1)
            n = torch.gather(b, 2, at).contiguous().view(torch.bfloat16).double()
            x = torch.empty(P + C, Hkv, d, dtype=torch.float64, device=b.device)
            x[..., 0::2] = (byte % 16) * n[..., 1:] + n[..., :1]
            x[..., 1::2] = (byte // 16) * n[..., 1:] + n[..., :1]
            return x

        k, v = rows(s["k_cache"]), rows(s["v_cache"])
        step = max(1, (1 << 28) // ((P + C) * G))
        for h in range(Hkv):
            for a in range(0, C, step):
                b = min(C, a + step)
                q = s["q"][r0 + a:r0 + b, h * G:(h + 1) * G].double()
                x = torch.einsum("tgd,kd->tgk", q, k[:, h]) / math.sqrt(d)
                x = torch.where(pos[None, None] > (P + torch.arange(a, b, device=pos.device))[:, None, None], -torch.inf, x)
                z = torch.logsumexp(x, -1)
                outs.append((r0 + a, r0 + b, h, torch.einsum("tgk,kd->tgd", torch.exp(x - z[..., None]), v[:, h])))
                sums.append(z)
    out = torch.empty(s["out"].shape, dtype=torch.float64, device=s["q"].device)
    lse = torch.empty(out.shape[:2], dtype=torch.float64, device=out.device)
    for (a, b, h, o), z in zip(outs, sums):
        out[a:b, h * G:(h + 1) * G], lse[a:b, h * G:(h + 1) * G] = o, z
    return dict(out=out, lse=lse if case["lse"] else None)


# ----------------------------------------------------------------------------------------------------- linear attention
def _prepare_linear(case, seed):
    C, P = _lengths(case)
    R, H, d, T = case["requests"], case["heads"], case["head_dim"], int(C.sum())
    dev = _device()
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape):
        return torch.empty(*shape, dtype=torch.float32, device=dev).normal_(generator=gen)

    interval, slots = case["snap_interval"], 2 * R
    counts = (P + C) // interval - P // interval if interval else np.zeros(R, np.int64)
    snaps = np.full((R, max(1, int(counts.max()))), -1, np.int32)
    for i in range(R):
        snaps[i, :counts[i]] = slots + np.arange(counts[i])
        slots += int(counts[i])
    s = dict(q=torch.nn.functional.silu(normal(T, H, d)).bfloat16(), k=(torch.nn.functional.silu(normal(T, H, d)) * d ** -0.5).bfloat16(),
             v=normal(T, H, d).bfloat16(), pool=0.1 * normal(slots, H, d, d), out=torch.empty(T, H, d, dtype=torch.bfloat16, device=dev),
             starts=_offsets(C), chunks=C, prefix=P, snap_slots=snaps)
    # natural logarithms of the decays: slopes that halve from head to head, or a gate's around them
    slope = -torch.exp2(-8.0 * torch.arange(1, H + 1, dtype=torch.float32, device=dev) / H)
    s["log_decay"] = slope * torch.nn.functional.softplus(normal(T, H)) if case["per_token"] else slope
    s["rows"] = torch.from_numpy(s["starts"]).to(dev)
    s["state_in"] = torch.arange(R, dtype=torch.int32, device=dev)
    s["state_out"] = s["state_in"] + R
    s["prefix_dev"] = torch.from_numpy(P.astype(np.int32)).to(dev)
    s["snaps_dev"] = torch.from_numpy(snaps).to(dev) if interval else None
    s["status"] = torch.zeros(1, dtype=torch.int32, device=dev)
    if own:
        import paper_2609_35263_b200 as wpp
        s["workspace"] = torch.empty(wpp.wpp_linear_workspace_bytes(R, H, d, T), dtype=torch.uint8, device=dev)
        _ctx()
    return s


_STEP = 256                     # tokens that the plain form takes at a time


def _run_linear(case, s):
    if own:
        import paper_2609_35263_b200 as wpp
        wpp.wpp_linear_chunk(_ctx(), s["q"], s["k"], s["v"], s["log_decay"], s["rows"], s["pool"], s["state_in"], s["state_out"],
                             out=s["out"], prefix_lens=s["prefix_dev"], snap_interval=case["snap_interval"], snap_slots=s["snaps_dev"],
                             status=s["status"], workspace=s["workspace"])
        return dict(out=s["out"], states=s["pool"])
    R, H, d, interval = case["requests"], case["heads"], case["head_dim"], case["snap_interval"]
    most, T, dev = int(s["chunks"].max()), int(s["starts"][-1]), s["q"].device
    chunks = s["rows"][1:] - s["rows"][:-1]
    t = torch.arange(most, device=dev)
    there = t < chunks[:, None]                                                                     # [R, tokens]
    at = (s["rows"][:-1, None] + t).clamp(max=T - 1)
    q, k, v = ((s[n][at].float() * there[..., None, None]).transpose(1, 2) for n in "qkv")          # [R, H, tokens, d]
    g = s["log_decay"].expand(T, H)[at].double() * there[..., None]
    g = g.cumsum(1).transpose(1, 2)                                                                 # [R, H, tokens], of the chunk so far
    state, first = s["pool"][s["state_in"].long()], torch.zeros(R, H, 1, dtype=torch.float64, device=dev)
    start = state
    for a in range(0, most, _STEP):
        qa, ka, va, ga = q[:, :, a:a + _STEP], k[:, :, a:a + _STEP], v[:, :, a:a + _STEP], g[:, :, a:a + _STEP]
        fall = (ga[..., :, None] - ga[..., None, :]).float().exp().tril()
        out = (qa @ ka.transpose(2, 3) * fall) @ va + (ga - first).float().exp()[..., None] * (qa @ state)
        keep = there[:, a:a + _STEP]
        s["out"][at[:, a:a + _STEP][keep]] = out.transpose(1, 2)[keep].bfloat16()
        last = ga[..., -1:]
        state = (last - first).float().exp()[..., None] * state + (ka * (last - ga).float().exp()[..., None]).transpose(2, 3) @ va
        first = last
    s["pool"][s["state_out"].long()] = state
    for n in range(s["snap_slots"].shape[1] if interval else 0):
        # the states after the n-th boundary in each chunk, straight from their definition
        some = torch.nonzero(s["snaps_dev"][:, n] >= 0).squeeze(1)
        end = (s["prefix_dev"][some] // interval + n + 1) * interval - s["prefix_dev"][some] - 1
        last = torch.gather(g[some], 2, end.long()[:, None, None].expand(-1, H, 1))
        weight = (last - g[some]).clamp(max=0).float().exp() * (t <= end[:, None])[:, None]
        s["pool"][s["snaps_dev"][some, n].long()] = last.float().exp()[..., None] * start[some] + (k[some] * weight[..., None]).transpose(2, 3) @ v[some]
    return dict(out=s["out"], states=s["pool"])


def _exact_linear(case, seed):
    s = _prepare_linear(case, seed)
    H, d, interval = case["heads"], case["head_dim"], case["snap_interval"]
    out, pool = torch.empty(s["out"].shape, dtype=torch.float64, device=s["q"].device), s["pool"].double()
    for i in range(case["requests"]):
        a, b, P = int(s["starts"][i]), int(s["starts"][i + 1]), int(s["prefix"][i])
        g = s["log_decay"].double()
        g = torch.cumsum(g[a:b], 0) if case["per_token"] else g * torch.arange(1, b - a + 1, device=g.device, dtype=torch.float64)[:, None]
        ends, slots = [b - a - 1], [case["requests"] + i]
        if interval:
            ends += [(P // interval + n + 1) * interval - P - 1 for n in range((P + b - a) // interval - P // interval)]
            slots += [int(x) for x in s["snap_slots"][i] if x >= 0]
        for h in range(H):
            q, k, v, c = s["q"][a:b, h].double(), s["k"][a:b, h].double(), s["v"][a:b, h].double(), g[:, h]
            start = s["pool"][i, h].double()
            for r in range(0, b - a, 4096):
                x = q[r:r + 4096] @ k[:r + 4096].T
                gap = c[r:r + 4096, None] - c[None, :r + 4096]
                gap = torch.where(torch.arange(x.shape[1], device=x.device)[None] > torch.arange(r, r + x.shape[0], device=x.device)[:, None], -torch.inf, gap)
                out[a + r:a + r + x.shape[0], h] = (x * torch.exp(gap)) @ v[:r + 4096] + torch.exp(c[r:r + 4096, None]) * (q[r:r + 4096] @ start)
            for end, slot in zip(ends, slots):
                pool[slot, h] = torch.exp(c[end]) * start + (k[:end + 1] * torch.exp(c[end] - c[:end + 1])[:, None]).T @ v[:end + 1]
    return dict(out=out, states=pool)


# ------------------------------------------------------------------------------------------------------------ interface
_RUN = {"append": _run_append, "attend": _run_attend, "linear": _run_linear}


def prepare(case, seed):
    return case, (_prepare_linear if case["kind"] == "linear" else _prepare_cache)(case, seed)


def run(state):
    case, s = state
    return _RUN[case["kind"]](case, s)


def exact(case, seed):
    if case["kind"] == "append":
        return None                                # bytes: equal or not
    return (_exact_linear if case["kind"] == "linear" else _exact_attend)(case, seed)


def work(case):
    C, P = _lengths(case)
    T = int(C.sum())
    if case["kind"] == "linear":
        H, d, interval = case["heads"], case["head_dim"], case["snap_interval"]
        snaps = int(((P + C) // interval - P // interval).sum()) if interval else 0
        # each token's q, k, v, out and decay, each state read and written; the recurrence's products and sums
        return {"bytes": T * H * (4 * 2 * d + (4 if case["per_token"] else 0)) + (2 * case["requests"] + snaps) * H * d * d * 4,
                "flops": T * H * 5 * d * d}
    Hq, Hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    row = 2 * Hkv * (d // 2 + 4)                   # a token's K and V in the cache
    if case["kind"] == "append":
        return {"bytes": T * (2 * Hkv * d * 2 + row), "flops": 0}
    return {"bytes": int((P + C).sum()) * row + T * Hq * (2 * 2 * d + (4 if case["lse"] else 0)),
            "flops": 4 * d * Hq * int((C * P + C * (C + 1) // 2).sum())}
