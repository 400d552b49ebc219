"""Operators around a serving stage's paged KV cache, as measurable cases.

  pages   the pages of a wave's new tokens out of a list of free ones: block tables, row offsets, positions and slots, from the
          requests' lengths, on the GPU
  rope    rotary positions of a wave's queries and keys
  write   the same with the rotated keys, and the values, written to their slots of a bf16 cache
  append  the K/V rows of a wave's new tokens into the pages of a cache held in 8 bits
  attend  attention of a wave's queries over such a cache: single tokens behind contexts, and chunks of prompts

A block (page, KV head) of the 8-bit cache holds a code for each element of its rows, an 8-bit floating-point number (e4m3), and
behind the codes one fp32 number, its scale, a power of two: an element stands for scale * code.  The scale is the least one with
which the rows appended so far are within 448 (between 2^-56 and 2^40); where new rows raise it, the codes that stand are scaled
down and rounded again.  The append's results are returned as codes and scales.

A position's angle is position * frequency: 64 bits where a position is far, and so in both forms here.

Ragged lengths are drawn from the case's own `lengths` number, so that the work of a case is fixed; values and physical page
ids come from the seed.
"""
import math

import numpy as np
import torch

own = False

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
def _case(name, kind, requests, chunk, prefix, heads, lengths=0, **more):
    """chunk, prefix: (least, most) tokens, uniform per request; heads: (query heads, KV heads, head_dim, page size)."""
    c = dict(kind=kind, requests=requests, chunk_min=chunk[0], chunk_max=chunk[1], prefix_min=prefix[0], prefix_max=prefix[1],
             q_heads=heads[0], kv_heads=heads[1], head_dim=heads[2], page_size=heads[3], lengths=lengths, **more)
    return dict(c, name=name) if name else c


def _rope(rot_dim, interleaved=False, base=10000.0, scaling="none", factor=1.0, original_context=0):
    return dict(rot_dim=rot_dim, interleaved=interleaved, base=base, scaling=scaling, factor=factor, original_context=original_context)


_SMALL_HEADS, _MID_HEADS, _BIG_HEADS = (8, 2, 64, 16), (32, 8, 128, 64), (64, 8, 128, 64)


def listed():
    return [
        # a generation step's pages: a full batch, one token each, most of them in a page that is there
        _case("pages_step", "pages", 256, (1, 1), (0, 16384), _MID_HEADS, lengths=1),
        # a prefill wave's pages, small ones, ragged chunks
        _case("pages_prompts", "pages", 64, (1, 2048), (0, 8192), _SMALL_HEADS, lengths=2),
        # a generation step's queries and keys
        _case("rope_step", "rope", 64, (1, 1), (0, 16384), _MID_HEADS, lengths=3, **_rope(128)),
        # a chunk of a long document beyond the trained context, neighbouring elements paired, half of each head
        _case("rope_long_context", "rope", 1, (8192, 8192), (122880, 122880), _MID_HEADS,
              **_rope(64, interleaved=True, base=500000.0, scaling="turns", factor=4.0, original_context=32768)),
        # a generation step's queries and keys, straight into the cache
        _case("write_step", "write", 64, (1, 1), (0, 16384), _BIG_HEADS, lengths=4, **_rope(128, base=500000.0, scaling="wavelength", factor=8.0,
                                                                                          original_context=8192)),
        # a prefill wave's
        _case("write_prompts", "write", 16, (256, 2048), (0, 8192), _BIG_HEADS, lengths=5, **_rope(128)),
        # a generation step's new rows: 64 requests, one token each, anywhere in their pages
        _case("append_step", "append", 64, (1, 1), (0, 8192), _BIG_HEADS, lengths=6),
        # a prefill wave's new rows: 32 ragged chunks
        _case("append_prompts", "append", 32, (256, 2048), (0, 4096), _BIG_HEADS, lengths=7),
        # one user alone, one token behind 8,192 cached ones: latency
        _case("token_one_request", "attend", 1, (1, 1), (8191, 8191), _MID_HEADS, lse=False),
        # a generation step of a full batch with contexts of all lengths
        _case("token_batch_64", "attend", 64, (1, 1), (255, 16383), _BIG_HEADS, lengths=8, lse=False),
        # an ordinary ragged prefill wave, log-sums for a later merge
        _case("prompts_ragged", "attend", 16, (256, 2048), (0, 8192), _MID_HEADS, lengths=9, lse=True),
        # a chunk of a long document
        _case("prompt_behind_long_prefix", "attend", 1, (4096, 4096), (32768, 32768), _BIG_HEADS, lse=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what, lengths = rng.random(), rng.randrange(1, 1 << 30)
    heads = rng.choice([_SMALL_HEADS, _MID_HEADS, _BIG_HEADS, (32, 8, 128, 128), (16, 4, 64, 32), (40, 8, 128, 32), (32, 2, 128, 16), (8, 8, 64, 64)])
    if what < 0.5:
        kind = rng.choice(["pages", "rope", "write", "append"])
        hi = _log_int(rng, 1, 2048)
        requests = max(1, min(_log_int(rng, 1, 256 if kind == "pages" else 64), (65536 if kind == "pages" else 16384) // hi))
        rope = {}
        if kind in ("rope", "write"):
            scaling = rng.choice(["none", "none", "linear", "base", "wavelength", "turns"])
            rope = _rope(rng.choice([heads[2], heads[2], heads[2] // 2, heads[2] // 4]), interleaved=rng.random() < 0.5, base=rng.choice([10000.0, 500000.0]),
                         scaling=scaling, factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0]),
                         original_context=rng.choice([4096, 8192, 32768]) if scaling in ("wavelength", "turns") else 0)
        return _case(None, kind, requests, (max(1, hi // 3), hi), (0, _log_int(rng, 1, 131072 if kind == "rope" else 8192)), heads, lengths=lengths, **rope)
    if what < 0.75:
        hi = _log_int(rng, 1, 131071)
        return _case(None, "attend", max(1, min(_log_int(rng, 1, 64), 491520 // hi)), (1, rng.choice([1, 1, 1, 2, 4])), (hi // rng.choice([1, 4, 100]), hi),
                     heads, lengths=lengths, lse=rng.random() < 0.3)
    hi = _log_int(rng, 5, 4096)
    case = _case(None, "attend", _log_int(rng, 1, 32), (max(1, int(hi * rng.random())), hi), (0, 0) if rng.random() < 0.3 else (0, _log_int(rng, 16, 32768)),
                 heads, lengths=lengths, lse=rng.random() < 0.3)
    while case["requests"] > 1 and (work(case)["flops"] > 2e12 or work(case)["bytes"] > 1e9 or _scores(case) > 1 << 33):
        case["requests"] //= 2
    while _scores(case) > 1 << 33:
        case["prefix_max"] //= 2
    return case


# ----------------------------------------------------------------------------------------------------------- lengths
def _lengths(case):
    rng = np.random.default_rng(case["lengths"])
    n = case["requests"]
    C = rng.integers(case["chunk_min"], case["chunk_max"] + 1, n).astype(np.int64)
    P = rng.integers(case["prefix_min"], case["prefix_max"] + 1, n).astype(np.int64)
    return C, P


def _scores(case):
    """Of the plain form at a time: every request padded to the longest."""
    C, P = _lengths(case)
    return case["requests"] * int(C.max()) * int((C + P).max()) * case["q_heads"]


def _capacity(case):
    """Rows of positions and slots that a captured step would keep: the tokens, rounded up."""
    return -(-int(_lengths(case)[0].sum()) // 64) * 64


# ------------------------------------------------------------------------------------------------------- 8-bit blocks
_LEAST, _MOST = -56, 40          # powers of two that a scale may be


def _scale(top):
    """The least power of two s with top <= 448 s."""
    m, e = torch.frexp(top)
    e = torch.where(m > 0.875, e - 8, e - 9).clamp(_LEAST, _MOST)
    return torch.ldexp(torch.ones_like(top), torch.where(top > 0, e, _LEAST))


def _codes(x, scale):
    x = torch.where(torch.isfinite(x), (x / scale).clamp(-448, 448), torch.nan)
    return x.to(torch.float8_e4m3fn)


def _views(cache, case):
    """Codes [pages, Hkv, B, d] and scales [pages, Hkv, 1] of a pool of blocks."""
    B, d = case["page_size"], case["head_dim"]
    return cache[..., :B * d].view(torch.float8_e4m3fn).unflatten(-1, (B, d)), cache[..., B * d:B * d + 4].view(torch.float32)


def _pool(case, pages, gen):
    # keys and values of other tokens, channels of unequal size among them, and pages
    B, Hkv, d = case["page_size"], case["kv_heads"], case["head_dim"]
    dev = _device()
    size = torch.exp(0.5 * torch.randn(Hkv, 1, d, device=dev, generator=gen))
    cache = torch.zeros(pages, Hkv, B * d + 16, dtype=torch.uint8, device=dev)
    codes, scales = _views(cache, case)
    step = max(1, (1 << 26) // (Hkv * B * d))
    for a in range(0, pages, step):
        x = torch.randn(min(step, pages - a), Hkv, B, d, device=dev, generator=gen) * size
        x *= torch.exp(0.3 * torch.randn(x.shape[0], Hkv, 1, 1, device=dev, generator=gen))
        s = _scale(x.abs().amax((2, 3))).unsqueeze(-1)
        scales[a:a + step] = s
        codes[a:a + step] = _codes(x, s.unsqueeze(-1))
    return cache


# ----------------------------------------------------------------------------------------------------------- prepare
def _frequencies(case):
    """Radians per position of the pairs, in 64 bits, and what the rotated elements are multiplied by."""
    n, base, factor, ctx = case["rot_dim"], case["base"], case["factor"], case["original_context"]
    if case["scaling"] == "base":
        base *= factor ** (n / (n - 2)) if n > 2 else 1.0
    f = [base ** (-2.0 * i / n) for i in range(n // 2)]
    if case["scaling"] == "linear":
        f = [x / factor for x in f]
    if case["scaling"] == "wavelength":
        # turns over the trained context: below 1 fully stretched, above 4 as they were, in between in between
        share = [min(1.0, max(0.0, (ctx * x / (2 * math.pi) - 1.0) / (4.0 - 1.0))) for x in f]
        f = [x * ((1 - s) / factor + s) for x, s in zip(f, share)]
    if case["scaling"] == "turns":
        # the pairs between those that make 32 and 1 turns over the trained context, by number
        at = [n * math.log(ctx / (2 * math.pi * b)) / (2 * math.log(base)) for b in (32.0, 1.0)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), n - 1)
        ramp = [min(1.0, max(0.0, (i - lo) / (hi - lo if hi != lo else 0.001))) for i in range(n // 2)]
        return [x * (r / factor + 1 - r) for x, r in zip(f, ramp)], 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _prepare(case, seed):
    C, P = _lengths(case)
    kind, R, B, Hq, Hkv, d = case["kind"], case["requests"], case["page_size"], case["q_heads"], case["kv_heads"], case["head_dim"]
    T = int(C.sum())
    dev = _device()
    gen = torch.Generator(device=dev).manual_seed(seed)
    blocks, there = (P + C + B - 1) // B, (P + B - 1) // B
    pages = int(blocks.sum()) + 8
    perm = np.random.default_rng(seed).permutation(pages).astype(np.int32)
    owner = np.concatenate([[0], np.cumsum(there if kind == "pages" else blocks)])
    at = np.arange(int(blocks.max()))
    table = np.where(at < (there if kind == "pages" else blocks)[:, None], perm[np.minimum(owner[:-1, None] + at, pages - 1)], -1).astype(np.int32)

    def normal(*shape):
        return torch.empty(*shape, dtype=torch.bfloat16, device=dev).normal_(generator=gen)

    s = dict(prefix=P.astype(np.int32), chunks=C.astype(np.int32), starts=np.concatenate([[0], np.cumsum(C)]).astype(np.int64))
    s["table"], s["prefix_dev"], s["chunks_dev"] = (torch.from_numpy(x).to(dev) for x in (table, s["prefix"], s["chunks"]))
    s["status"] = torch.zeros(1, dtype=torch.int32, device=dev)
    s["pages"] = pages
    if own:
        import paper_2609_35263_b200 as wpp
        kv8 = kind in ("append", "attend")
        s["desc"] = wpp.make_desc(R, Hq, Hkv, d, B, table.shape[1], pages, dtype=wpp.WPP_KV8 if kv8 else wpp.WPP_BF16)
        _ctx()
        if kv8:
            s["plan"] = wpp.wpp_plan_tiles(_ctx(), s["desc"], s["prefix"], s["chunks"]).to_device(dev)
            s["workspace"] = torch.empty(int(s["plan"].info.workspace_bytes), dtype=torch.uint8, device=dev)
    if kind == "pages":
        n = _capacity(case)
        s["free"] = torch.from_numpy(perm[owner[-1]:]).to(dev)
        s["cursor"] = torch.zeros(2, dtype=torch.int32, device=dev)          # entries of the list that are taken
        s["cursor_out"] = torch.zeros(2, dtype=torch.int32, device=dev)
        s["rows"] = torch.empty(R + 1, dtype=torch.int64, device=dev)
        s["positions"] = torch.empty(n, dtype=torch.int32, device=dev)
        s["slots"] = torch.empty(n, dtype=torch.int64, device=dev)
    if kind in ("rope", "write"):
        f, magnitude = _frequencies(case)
        s["frequencies"], s["magnitude"] = torch.tensor(f, dtype=torch.float64, device=dev), magnitude
        if own:
            import paper_2609_35263_b200 as wpp
            turns, s["magnitude"] = wpp.wpp_rope_frequencies(case["rot_dim"], base=case["base"], scaling=case["scaling"], factor=case["factor"],
                                                             original_context=case["original_context"])
            s["turns"] = turns.to(dev)
        request = np.repeat(np.arange(R), C)
        pos = (P - s["starts"][:-1])[request] + np.arange(T)
        s["positions"] = torch.from_numpy(pos.astype(np.int32)).to(dev)
        s["slots"] = torch.from_numpy(table[request, pos // B].astype(np.int64) * B + pos % B).to(dev)
        # as a projection leaves them: a token's query, key and value heads side by side
        s["qkv"] = normal(T, Hq + 2 * Hkv, d)
        s["q"], s["k_new"], s["v_new"] = s["qkv"].split([Hq, Hkv, Hkv], 1)
        s["q_out"], s["k_out"] = torch.empty(T, Hq, d, dtype=torch.bfloat16, device=dev), torch.empty(T, Hkv, d, dtype=torch.bfloat16, device=dev)
        if kind == "write":
            s["k_cache"], s["v_cache"] = (torch.zeros(pages, Hkv, B, d, dtype=torch.bfloat16, device=dev) for _ in range(2))
    if kind in ("append", "attend"):
        s["k_cache"], s["v_cache"] = _pool(case, pages, gen), _pool(case, pages, gen)
    if kind == "append":
        s.update(k_new=normal(T, Hkv, d), v_new=normal(T, Hkv, d))
    if kind == "attend":
        s.update(q=normal(T, Hq, d), out=torch.empty(T, Hq, d, dtype=torch.bfloat16, device=dev),
                 log_sums=torch.empty(T, Hq, dtype=torch.float32, device=dev) if case["lse"] else None)
    return s


# ------------------------------------------------------------------------------------------------------------- pages
def _run_pages(case, s):
    if own:
        import paper_2609_35263_b200 as wpp
        wpp.wpp_assign_pages(_ctx(), s["desc"], s["prefix_dev"], s["chunks_dev"], s["free"], s["cursor"], s["table"], s["rows"], s["positions"], s["slots"],
                             cursor_out=s["cursor_out"], status=s["status"])
        return dict(tables=s["table"], rows=s["rows"], positions=s["positions"], slots=s["slots"], taken=s["cursor_out"][:1])
    B, n = case["page_size"], s["slots"].numel()
    P, C = s["prefix_dev"].long(), s["chunks_dev"].long()
    there, blocks = (P + B - 1) // B, (P + C + B - 1) // B
    need = blocks - there
    last = need.cumsum(0) + s["cursor"][0]
    j = torch.arange(s["table"].shape[1], device=P.device)
    new = (j >= there[:, None]) & (j < blocks[:, None])
    at = (last - need - there)[:, None] + j
    s["table"].copy_(torch.where(new, s["free"][at.clamp(0, s["free"].numel() - 1)], s["table"]))
    s["rows"][0] = 0
    s["rows"][1:] = C.cumsum(0)
    t = torch.arange(n, device=P.device)
    request = torch.searchsorted(s["rows"][1:], t, right=True)
    real = request < case["requests"]
    request = request.clamp(max=case["requests"] - 1)
    pos = torch.where(real, P[request] + t - s["rows"][request], 0)
    s["positions"].copy_(pos)
    s["slots"].copy_(torch.where(real, s["table"][request, pos // B].long() * B + pos % B, -1))
    s["cursor_out"][0] = last[-1]
    return dict(tables=s["table"], rows=s["rows"], positions=s["positions"], slots=s["slots"], taken=s["cursor_out"][:1])


# --------------------------------------------------------------------------------------------------------- positions
def _rotate(case, x, cos, sin):
    n = case["rot_dim"]
    y = x[..., :n].float()
    a, b = (y[..., 0::2], y[..., 1::2]) if case["interleaved"] else (y[..., :n // 2], y[..., n // 2:])
    pairs = (a * cos - b * sin, a * sin + b * cos)
    y = torch.stack(pairs, -1).flatten(-2) if case["interleaved"] else torch.cat(pairs, -1)
    return torch.cat([y.bfloat16(), x[..., n:]], -1)


def _run_rope(case, s):
    if own:
        import paper_2609_35263_b200 as wpp
        if case["kind"] == "rope":
            wpp.wpp_rope(_ctx(), s["q"], s["k_new"], s["turns"], s["positions"], q_out=s["q_out"], k_out=s["k_out"], interleaved=case["interleaved"],
                         magnitude=s["magnitude"])
            return dict(q=s["q_out"], k=s["k_out"])
        wpp.wpp_rope_append(_ctx(), s["desc"], s["q"], s["k_new"], s["v_new"], s["q_out"], s["k_cache"], s["v_cache"], s["turns"], s["positions"], s["slots"],
                            interleaved=case["interleaved"], magnitude=s["magnitude"], status=s["status"])
        return dict(q=s["q_out"], k_cache=s["k_cache"], v_cache=s["v_cache"])
    angle = (s["positions"].double()[:, None] * s["frequencies"])[:, None]
    cos, sin = (angle.cos() * s["magnitude"]).float(), (angle.sin() * s["magnitude"]).float()
    s["q_out"].copy_(_rotate(case, s["q"], cos, sin))
    k = _rotate(case, s["k_new"], cos, sin)
    if case["kind"] == "rope":
        s["k_out"].copy_(k)
        return dict(q=s["q_out"], k=s["k_out"])
    page, slot = s["slots"] // case["page_size"], s["slots"] % case["page_size"]
    s["k_cache"][page, :, slot] = k
    s["v_cache"][page, :, slot] = s["v_new"]
    return dict(q=s["q_out"], k_cache=s["k_cache"], v_cache=s["v_cache"])


def _exact_rope(case, seed):
    s = _prepare(case, seed)
    n, pos = case["rot_dim"], s["positions"].double()
    f, magnitude = _frequencies(case)
    turned = []
    for x in (s["q"].double(), s["k_new"].double()):
        y = x.clone()
        for i in range(n // 2):
            a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + n // 2)
            turn = torch.polar(torch.full_like(pos, magnitude), pos * f[i])[:, None]
            z = torch.complex(x[..., a], x[..., b]) * turn
            y[..., a], y[..., b] = z.real, z.imag
        turned.append(y)
    if case["kind"] == "rope":
        return dict(q=turned[0], k=turned[1])
    caches = []
    for x in (turned[1], s["v_new"].double()):
        rows = torch.zeros(s["pages"] * case["page_size"], *x.shape[1:], dtype=torch.float64, device=x.device)
        rows[s["slots"]] = x
        caches.append(rows.unflatten(0, (-1, case["page_size"])).transpose(1, 2).contiguous())
    return dict(q=turned[0], k_cache=caches[0], v_cache=caches[1])


# ------------------------------------------------------------------------------------------------------------ append
def _run_append(case, s):
    if own:
        import paper_2609_35263_b200 as wpp
        wpp.wpp_kv_append(_ctx(), s["desc"], s["k_new"], s["v_new"], s["k_cache"], s["v_cache"], s["table"], s["prefix_dev"], s["chunks_dev"], s["plan"],
                          status=s["status"])
    else:
        _append_plain(case, s, s["k_new"], s["k_cache"])
        _append_plain(case, s, s["v_new"], s["v_cache"])
    (k, k_scale), (v, v_scale) = _views(s["k_cache"], case), _views(s["v_cache"], case)
    return dict(k=k, k_scale=k_scale, v=v, v_scale=v_scale)


def _touched(case, s):
    """(request, its touched page's number, the new token's place among the touched pages, its slot), per page and per token."""
    B, R, T = case["page_size"], case["requests"], int(s["starts"][-1])
    n = (s["prefix"].astype(np.int64) + s["chunks"] + B - 1) // B - s["prefix"] // B
    total = int(n.sum())
    dev, P, C = s["table"].device, s["prefix_dev"].long(), s["chunks_dev"].long()
    n_dev = (P + C + B - 1) // B - P // B
    first = n_dev.cumsum(0) - n_dev
    owner = torch.repeat_interleave(torch.arange(R, device=dev), n_dev, output_size=total)
    number = torch.arange(total, device=dev) - first[owner] + (P // B)[owner]
    request = torch.repeat_interleave(torch.arange(R, device=dev), C, output_size=T)
    pos = P[request] + torch.arange(T, device=dev) - (C.cumsum(0) - C)[request]
    return owner, number, first[request] + pos // B - (P // B)[request], pos % B


def _append_plain(case, s, new, cache):
    B = case["page_size"]
    codes, scales = _views(cache, case)
    owner, number, place, slot = _touched(case, s)
    page = s["table"][owner, number].long()
    x = new.float()
    size = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)                                        # [T, Hkv]
    top = torch.zeros(page.numel(), size.shape[1], device=x.device).scatter_reduce_(0, place[:, None].expand_as(size), size, "amax")
    stand = (s["prefix_dev"].long()[owner] - number * B).clamp(min=0)                                   # rows that stand in the page
    before = scales[page, :, 0]
    scale = torch.where((stand > 0)[:, None], torch.maximum(before, _scale(top)), _scale(top))
    kept = torch.arange(B, device=x.device) < stand[:, None]                                            # [pages, B]
    old = codes[page]
    again = _codes(old.float(), (scale / torch.where((stand > 0)[:, None], before, scale))[..., None, None])
    codes[page] = torch.where(kept[:, None, :, None], again.view(torch.uint8), old.view(torch.uint8)).view(torch.float8_e4m3fn)
    scales[page] = scale[..., None]
    codes[page[place], :, slot] = _codes(x, scale[place][..., None])


def _exact_append(case, seed):
    s = _prepare(case, seed)
    out = {}
    B = case["page_size"]
    for name in "kv":
        codes, scales = (x.double() for x in _views(s[name + "_cache"], case))
        for i in range(case["requests"]):
            P, C, r0 = int(s["prefix"][i]), int(s["chunks"][i]), int(s["starts"][i])
            for a in range(P // B * B, P + C, B):
                page, lo, hi = int(s["table"][i, a // B]), max(P, a), min(P + C, a + B)
                x = s[name + "_new"][r0 + lo - P:r0 + hi - P].double().transpose(0, 1)                  # [Hkv, rows, d]
                scale = torch.exp2(torch.ceil(torch.log2(x.abs().amax((1, 2)) / 448)).clamp(-56, 40))
                if lo > a:
                    scale = torch.maximum(scale, scales[page, :, 0])
                    codes[page, :, :lo - a] *= (scales[page, :, 0] / scale)[:, None, None]
                codes[page, :, lo - a:hi - a] = x / scale[:, None, None]
                scales[page, :, 0] = scale
        out[name], out[name + "_scale"] = codes, scales
    return out


# -------------------------------------------------------------------------------------------------------------- attend
def _run_attend(case, s):
    if own:
        import paper_2609_35263_b200 as wpp
        wpp.wpp_prefill_attention_varlen(_ctx(), s["desc"], s["q"], s["out"], s["log_sums"], s["k_cache"], s["v_cache"], s["table"], s["prefix_dev"],
                                         s["chunks_dev"], s["plan"], workspace=s["workspace"], status=s["status"])
        return dict(out=s["out"], lse=s["log_sums"])
    # every request padded to the longest, all at once
    Hq, Hkv, T = case["q_heads"], case["kv_heads"], int(s["starts"][-1])
    dev = s["table"].device
    table = s["table"].clamp(min=0).long()

    def rows(cache):
        codes, scales = _views(cache, case)
        return (codes[table].float() * scales[table][..., None]).transpose(1, 2).flatten(2, 3)                                # [R, Hkv, keys, d]

    most = int(s["chunks"].max())
    t = torch.arange(most, device=dev)
    starts = s["chunks_dev"].cumsum(0) - s["chunks_dev"]
    at = (starts[:, None] + t).clamp(max=T - 1)
    q = s["q"][at].float().unflatten(2, (Hkv, Hq // Hkv)).permute(0, 2, 3, 1, 4).flatten(2, 3)                               # [R, Hkv, G * rows, d]
    score = (q @ rows(s["k_cache"]).transpose(2, 3)).mul_(case["head_dim"] ** -0.5).unflatten(2, (Hq // Hkv, -1))
    v = rows(s["v_cache"])
    seen = torch.arange(v.shape[2], device=dev) <= (s["prefix_dev"][:, None] + t)[..., None]                                 # [R, rows, keys]
    score.masked_fill_(~seen[:, None, None], -torch.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    v = v.masked_fill_(~seen.any(1)[:, None, :, None], 0.0)                   # what no row sees may hold anything
    out = (score.flatten(2, 3) @ v).unflatten(2, (Hq // Hkv, -1)) / total
    there = t < s["chunks_dev"][:, None]
    at = torch.nonzero(there.flatten(), as_tuple=True)[0] if len(s["chunks"]) > 1 else slice(None)
    s["out"].copy_(out.permute(0, 3, 1, 2, 4).flatten(2, 3).flatten(0, 1)[at])
    if s["log_sums"] is not None:
        s["log_sums"].copy_((top + total.log()).squeeze(-1).permute(0, 3, 1, 2).flatten(2, 3).flatten(0, 1)[at])
    return dict(out=s["out"], lse=s["log_sums"])


def _exact_attend(case, seed):
    if work(case)["flops"] > 2e13:
        return None
    s = _prepare(case, seed)
    B, Hq, Hkv, d = case["page_size"], case["q_heads"], case["kv_heads"], case["head_dim"]
    G = Hq // Hkv
    out = torch.empty(s["out"].shape, dtype=torch.float64, device=s["q"].device)
    lse = torch.empty(out.shape[:2], dtype=torch.float64, device=out.device)
    # e4m3: sign, four bits of exponent biased by 7, three of mantissa; no infinities
    byte = torch.arange(256, device=out.device)
    e, m = byte // 8 % 16, byte % 8
    number = torch.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * torch.exp2(e.double() - 7)).double() * (1 - byte // 128 * 2)
    number[byte % 128 == 127] = torch.nan
    for i in range(case["requests"]):
        P, C, r0 = int(s["prefix"][i]), int(s["chunks"][i]), int(s["starts"][i])
        pos = torch.arange(P + C, device=out.device)
        page, slot = s["table"][i].long()[pos // B], pos % B
        step = max(1, (1 << 28) // ((P + C) * G))
        for h in range(Hkv):
            at = slot[:, None] * d + torch.arange(d, device=out.device)
            k, v = (number[torch.gather(c[page, h], 1, at).long()] * c[page, h, B * d:B * d + 4].contiguous().view(torch.float32).double()
                    for c in (s["k_cache"], s["v_cache"]))
            for a in range(0, C, step):
                b = min(C, a + step)
                x = torch.einsum("tgd,kd->tgk", s["q"][r0 + a:r0 + b, h * G:(h + 1) * G].double(), k) / math.sqrt(d)
                x = torch.where(pos[None, None] > (P + torch.arange(a, b, device=pos.device))[:, None, None], -torch.inf, x)
                z = torch.logsumexp(x, -1)
                out[r0 + a:r0 + b, h * G:(h + 1) * G] = torch.einsum("tgk,kd->tgd", torch.exp(x - z[..., None]), v)
                lse[r0 + a:r0 + b, h * G:(h + 1) * G] = z
    return dict(out=out, lse=lse if case["lse"] else None)


# ------------------------------------------------------------------------------------------------------------ interface
_RUN = {"pages": _run_pages, "rope": _run_rope, "write": _run_rope, "append": _run_append, "attend": _run_attend}
_EXACT = {"rope": _exact_rope, "write": _exact_rope, "append": _exact_append, "attend": _exact_attend}


def prepare(case, seed):
    return case, _prepare(case, seed)


def run(state):
    case, s = state
    return _RUN[case["kind"]](case, s)


def exact(case, seed):
    return _EXACT[case["kind"]](case, seed) if case["kind"] in _EXACT else None         # whole numbers: equal or not


def work(case):
    C, P = _lengths(case)
    T, R, B = int(C.sum()), case["requests"], case["page_size"]
    Hq, Hkv, d, kind = case["q_heads"], case["kv_heads"], case["head_dim"], case["kind"]
    if kind == "pages":
        new = int(((P + C + B - 1) // B - (P + B - 1) // B).sum())
        return {"bytes": 8 * R + 8 * new + 8 * (R + 1) + 12 * _capacity(case), "flops": 0}
    if kind in ("rope", "write"):
        heads = Hq + (Hkv if kind == "rope" else 2 * Hkv)
        return {"bytes": T * (4 * heads * d + 4 + (8 if kind == "write" else 0)), "flops": 3 * T * (Hq + Hkv) * case["rot_dim"]}
    if kind == "append":
        # the new rows and their codes, a scale for each touched page; the standing rows only where a scale rises
        pages = int(((P + C + B - 1) // B - P // B).sum())
        return {"bytes": 2 * Hkv * (T * d * (2 + 1) + 4 * pages), "flops": 2 * T * Hkv * d * 2}
    row = 2 * Hkv * d                              # a token's K and V in the cache
    pages = int(((P + C + B - 1) // B).sum())
    return {"bytes": int((P + C).sum()) * row + 8 * Hkv * pages + T * Hq * (2 * 2 * d + (4 if case["lse"] else 0)),
            "flops": 4 * d * Hq * int((C * P + C * (C + 1) // 2).sum())}
