"""The 8-bit cache's format, its oracle and what the host refuses of it (no GPU)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2609_35263_b200 as wpp
from oracle import kv8 as okv8

from .kv8_harness import Wave


def test_encode_is_the_nearest_e4m3_number():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(4000) * 2.0 ** rng.integers(-14, 9, 4000), okv8.NUMBERS[:127], -okv8.NUMBERS[:127],
                        (okv8.NUMBERS[:126] + okv8.NUMBERS[1:127]) / 2, [0.0, -0.0, 448.0, 449.0, 1e9, -1e9]]).astype(np.float32)
    want = torch.from_numpy(x).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(okv8.encode(x), want)
    assert okv8.encode(np.array([np.nan, np.inf, -np.inf])).tolist() == [0x7F] * 3
    values = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(values, okv8.NUMBERS, equal_nan=True)


def test_scale_is_the_least_power_of_two_that_holds_the_largest_value():
    for top, e in ((0.0, -56), (448.0, 0), (448.5, 1), (447.0, 0), (224.0, -1), (225.0, 0), (1.0, -8), (2.0 ** -70, -56), (3e38, 40), (np.inf, -56)):
        assert okv8.scale_exp([top, -top / 2 if np.isfinite(top) else 0.0]) == e, top


def test_append_in_pieces_gives_what_one_append_gives():
    """Powers of two: codes taken down are the codes that one append would have given, but where they leave the normal range."""
    whole = Wave([0], [45], 2, 1, 64, 32, seed=3)
    a, _ = whole.appended()
    pieces, row = Wave([0], [45], 2, 1, 64, 32, seed=3), 0
    k, v = pieces.k_pool, pieces.v_pool
    for n in (3, 1, 1, 20, 15, 5):
        k, v = okv8.append(pieces.k_new[row:row + n], pieces.v_new[row:row + n], k, v, pieces.table, [row], [n], 32)
        row += n
    x, s = okv8.rows_of(a, whole.table[0], 45, 32, 64, 0)
    y, r = okv8.rows_of(k, whole.table[0], 45, 32, 64, 0)
    assert np.array_equal(s, r) and np.all(np.abs(x - y) <= s[:, None] * 2.0 ** -9)


def test_block_bytes():
    assert [wpp.wpp_kv8_block_bytes(B, d) for B in (16, 32, 64, 128) for d in (64, 128)] == [B * d + 16 for B in (16, 32, 64, 128) for d in (64, 128)]
    assert wpp.wpp_kv8_block_bytes(48, 128) == wpp.wpp_kv8_block_bytes(16, 96) == wpp.wpp_kv8_block_bytes(0, 0) == wpp.wpp_kv8_block_bytes(-16, 128) == 0


def _plan(**kw):
    d = wpp.make_desc(1, 4, 2, 64, 16, 8, 8, dtype=wpp.WPP_KV8, **kw)
    return wpp.wpp_plan_tiles(None, d, [5], [7], pin=False)


def test_descriptions_that_are_refused():
    _plan()
    block = 16 * 64 + 16
    _plan(kv_head_stride=block, kv_page_stride=2 * block)
    _plan(kv_head_stride=3 * block, kv_page_stride=block)              # heads further apart than pages: a layout of one's own
    for bad in (dict(kv_token_stride=64), dict(kv_head_stride=block - 16), dict(kv_head_stride=block + 8), dict(kv_page_stride=block // 2),
                dict(q_token_stride=8 * 64 + 4), dict(o_head_stride=32)):
        with pytest.raises(wpp.WppError) as e:
            _plan(**bad)
        assert e.value.status == 1, bad
    for d, B in ((96, 16), (128, 48), (64, 256)):
        with pytest.raises(wpp.WppError) as e:
            wpp.wpp_plan_tiles(None, wpp.make_desc(1, 4, 2, d, B, 8, 8, dtype=wpp.WPP_KV8), [5], [7], pin=False)
        assert e.value.status == 2
    with pytest.raises(wpp.WppError) as e:
        wpp.wpp_plan_tiles(None, wpp.make_desc(1, 4, 2, 64, 16, 8, 8, dtype=5), [5], [7], pin=False)
    assert e.value.status == 2


def test_plans_of_one_cache_are_not_the_other_s():
    """A plan says whose it is: neither call takes one of another pool type."""
    lib = wpp.load_library()
    for mine, other in ((wpp.WPP_KV8, wpp.WPP_KV4), (wpp.WPP_KV4, wpp.WPP_KV8), (wpp.WPP_KV8, wpp.WPP_BF16)):
        d = wpp.make_desc(1, 4, 2, 64, 16, 8, 8, dtype=mine)
        plan = wpp.wpp_plan_tiles(None, wpp.make_desc(1, 4, 2, 64, 16, 8, 8, dtype=other), [5], [7], pin=False)
        fake = ctypes.c_void_p(256)                                    # (a context is only asked for not being null before the plan is looked at)
        assert lib.wpp_kv_append(fake, ctypes.byref(d), *([None] * 7), plan.host.data_ptr(), *([None] * 3)) == 6


def test_validate_batch_wants_written_pages_to_be_one_request_s():
    d = wpp.make_desc(2, 4, 2, 64, 16, 4, 16, dtype=wpp.WPP_KV8)
    ok = [[0, 1, 2, -1], [0, 1, 3, -1]]                                # two full pages shared, a page each behind them
    assert wpp.wpp_validate_batch(d, ok, [32, 32], [5, 9]) == 0
    assert wpp.wpp_validate_batch(d, [[0, 1, 2, -1], [0, 1, 2, -1]], [32, 40], [5, 3]) == 9        # different slots of a page: its scale may move
    bf16 = wpp.make_desc(2, 4, 2, 64, 16, 4, 16)
    assert wpp.wpp_validate_batch(bf16, [[0, 1, 2, -1], [0, 1, 2, -1]], [32, 40], [5, 3]) == 9     # (request 1 reads what request 0 writes)
    assert wpp.wpp_validate_batch(d, [[0, 1, 2, -1], [0, 2, 3, -1]], [36, 32], [5, 9]) == 9        # read by another
    assert wpp.wpp_validate_batch(bf16, [[0, 1, 2, -1], [0, 1, 2, -1]], [36, 32], [5, 0]) == 0
    assert wpp.wpp_validate_batch(d, [[0, 1, 2, -1], [0, 1, 2, -1]], [36, 32], [5, 0]) == 0        # (an empty chunk reads nothing)
    assert wpp.wpp_validate_batch(d, [[0, 1, 1, -1], [4, 5, 6, -1]], [20, 32], [20, 9]) == 9       # a page twice in one table
    assert wpp.wpp_validate_batch(d, ok, [32, 32], [5, 40]) == 3
    assert wpp.wpp_validate_batch(d, [[0, 1, 16, -1], [0, 1, 3, -1]], [32, 32], [5, 9]) == 3
    assert wpp.wpp_validate_batch(d, ok, [32, -1], [5, 9]) == 1


@pytest.mark.parametrize("shape", [0, 1, 2])
@pytest.mark.parametrize("Hq,Hkv,d,B", [(8, 1, 128, 64), (10, 2, 64, 16), (64, 8, 128, 64)])
def test_plans_are_deterministic_and_count_their_work(shape, Hq, Hkv, d, B):
    P, C = [0, 700, 20_000, 5], [1, 300, 1, 0]
    desc = wpp.make_desc(4, Hq, Hkv, d, B, 1300, 5000, dtype=wpp.WPP_KV8)
    plan = wpp.wpp_plan_tiles(None, desc, P, C, opts=wpp.PlanOpts(0, 0, 0, 0, 0, shape), pin=False)
    assert plan.info.shape == 3 and plan.info.total_new_tokens == 302
    assert plan.info.flops == 4 * d * Hq * sum(c * p + c * (c + 1) // 2 for p, c in zip(P, C))
    assert plan.host_bytes() == wpp.wpp_plan_tiles(None, desc, P, C, opts=wpp.PlanOpts(0, 0, 0, 0, 0, shape), pin=False).host_bytes()


def _units(plan):
    """(units as dicts, how many are of the kernel for few rows, how those are handed out, touched pages) of a host plan."""
    import struct
    raw = plan.host_bytes()
    f = struct.unpack_from("<IIQ" + "i" * 8 + "qqq" + "QQ" + "IIII" + "iiiiiii" + "I", raw, 0)
    num_units, num_combine, off_units, off_combine = f[5], f[6], f[18], f[19]
    touched, deal, few = f[21], f[23], f[24]
    u = np.frombuffer(raw, np.int32, num_units * 12, off_units).reshape(num_units, 12)
    pages = np.frombuffer(raw, np.int32, 2 * touched, off_combine + 32 * num_combine).reshape(-1, 2)
    return u, few, deal, pages


WAVES = {"dealt": (([3000, 500, 2000, 10, 7000], [1, 2, 1, 1, 1], 8, 4), 2, 1), "cluster of 16": (([8191], [1], 8, 2), 0, 5), "cluster of 8": (([5000, 700, 3], [1, 3, 2], 16, 8), 0, 4),
         "cluster of 4": (([2000] * 8, [1] * 8, 16, 8), 0, 3), "cluster of 2": (([1200, 600, 64] * 8, [1] * 24, 6, 6), 0, 2), "tail cut": (([3000, 3000], [300, 300], 4, 1), 4, 0),
         "dealt, with tiles": (([9000, 9000, 600, 4000, 8000], [1, 1, 400, 1, 1], 8, 4), 2, 1)}


@pytest.mark.parametrize("name", list(WAVES))
def test_plan_covers_every_key_of_every_row_once(name):
    (P, C, Hq, Hkv), ctas, deal = WAVES[name]
    d, B, G = 128, 32, Hq // Hkv
    desc = wpp.make_desc(len(P), Hq, Hkv, d, B, 400, 5000, dtype=wpp.WPP_KV8)
    plan = wpp.wpp_plan_tiles(None, desc, P, C, opts=wpp.PlanOpts(0, 0, 0, ctas), pin=False)
    units, few, how, pages = _units(plan)
    assert how == deal and (name != "tail cut" or (plan.info.num_split_tiles > 0 and few == 0))
    steps = {}
    for k, u in enumerate(units):
        i, b, e, slot, row0, row1, rows0, rows1, head0, head1, _, pack = (int(x) for x in u)
        blocks = [(row0, rows0, range(head0, head0 + rows1))] if k < few else \
            [(r, n, range(h, h + min(pack, G))) for r, n, h in ((row0, rows0, head0), (row1, rows1, head1)) if n > 0]
        for r, n, heads in blocks:
            for t in range(r, r + n):
                for h in heads:
                    steps.setdefault((i, t, h), []).append((b, e))
    for i in range(len(P)):
        for t in range(C[i]):
            for h in range(Hq):
                at = 0
                for b, e in sorted(steps.pop((i, t, h))):
                    assert b == at or b == e
                    at = max(at, e)
                assert at * 128 >= P[i] + t + 1
    assert not steps
    assert pages.tolist() == [[i, b] for i in range(len(P)) if C[i] for b in range(P[i] // B, -(-(P[i] + C[i]) // B))]
    assert plan.info.workspace_bytes <= wpp.wpp_static_scratch_bytes()


def _workspace(dtype, heads, P, C, opts=None):
    Hq, Hkv, d, B = heads
    blocks = max(-(-(p + c) // B) for p, c in zip(P, C))
    return int(wpp.wpp_plan_tiles(None, wpp.make_desc(len(P), Hq, Hkv, d, B, blocks, blocks, dtype=dtype), P, C, opts=opts, pin=False).info.workspace_bytes)


def test_dealt_parts_take_no_wave_from_the_built_in_scratch():
    """What the array holds otherwise it holds of an 8-bit cache too: a wave of long and short parts is planned again without them where its
    tiles' parts no longer fit beside them.  (Equal shares of one wave are cut alike for both kinds of cache.)"""
    most = wpp.wpp_static_scratch_bytes()
    assert _workspace(wpp.WPP_KV8, (40, 8, 128, 64), [23213, 25029, 9801], [133, 204, 33]) <= most
    rng, hits = np.random.default_rng(5), 0
    for _ in range(3000):
        heads = [(40, 8, 128, 64), (64, 8, 128, 64), (32, 8, 128, 16), (8, 2, 64, 16)][rng.choice(4, p=(0.7, 0.1, 0.1, 0.1))]
        n = int(rng.integers(2, 6))
        P, C = rng.integers(0, 40000, n), np.exp(rng.uniform(0, np.log(300), n)).astype(int)
        a, b = _workspace(wpp.WPP_KV8, heads, P, C), _workspace(wpp.WPP_KV4, heads, P, C)
        assert a <= most or b > most, (heads, P, C, a, b)
        hits += b > most
    assert hits < 2000                                                  # (the waves are not all too large for it anyway)


def test_a_wave_that_the_built_in_scratch_does_not_hold_in_any_case_keeps_its_dealt_parts():
    """Nothing is won by planning it without them: and what comes back is that plan, to the byte of what a second call gives."""
    heads, P, C = (32, 8, 128, 16), [25486, 33879, 32130, 4978], [65, 2, 9, 3]
    assert min(_workspace(dtype, heads, P, C) for dtype in (wpp.WPP_KV8, wpp.WPP_KV4)) > wpp.wpp_static_scratch_bytes()
    desc = wpp.make_desc(4, *heads, 2200, 2200, dtype=wpp.WPP_KV8)
    a, b = (wpp.wpp_plan_tiles(None, desc, P, C, pin=False) for _ in range(2))
    units, few, how, pages = _units(a)
    assert how == 1 and 0 < few < len(units) == a.info.num_tiles and a.host_bytes() == b.host_bytes()
    ends = {}                                                           # (key steps of every block of rows, whose parts have to meet)
    for u in sorted(units[:few].tolist(), key=lambda u: (u[0], u[4], u[8], u[1])):
        assert u[1] == ends.get((u[0], u[4], u[8]), 0)
        ends[u[0], u[4], u[8]] = u[2]
    assert pages.tolist() == [[i, x] for i in range(4) for x in range(P[i] // 16, -(-(P[i] + C[i]) // 16))]


@pytest.fixture
def calls(monkeypatch):
    """The library's append and attention replaced by one that takes everything and counts."""
    from paper_2609_35263_b200 import binding
    lib, P, seen = wpp.load_library(), ctypes.c_void_p, []
    stubs = [ctypes.CFUNCTYPE(ctypes.c_int, *([P] * n))(lambda *a: seen.append(a) or 0) for n in (13, 16)]
    rest = [ctypes.cast(f, P).value for f in (lib.wpp_kda_chunk, lib.wpp_linear_chunk)]
    kinds = (binding.BatchDesc, binding.KdaDesc, binding.LinearDesc)
    binding._call.init(*(ctypes.cast(f, P).value for f in stubs), *rest, *kinds)
    monkeypatch.setattr(lib, "wpp_prefill_attention_varlen_static", lambda *a: seen.append(a) or 0)
    yield seen
    binding._call.init(*(ctypes.cast(f, P).value for f in (lib.wpp_kv_append, lib.wpp_prefill_attention_varlen)), *rest, *kinds)


def test_pools_that_end_too_early_are_refused(calls):
    """Both calls go to computed places of the pools: a 4-bit cache's, half as large, or one of fewer pages must not pass for one of 8 bits."""
    class Context:
        handle, device = ctypes.c_void_p(), -1

    class Stream:
        cuda_stream = 0

    class Address:
        def data_ptr(self):
            return 4096

    x, block = torch.zeros(4), 16 * 64 + 16
    plan = type("Plan", (), dict(host=x, dev=x))()
    u8 = lambda *n: torch.zeros(*n, dtype=torch.uint8)

    def run(k, v, **kw):
        desc = wpp.make_desc(1, 4, 2, 64, 16, 8, 8, **dict(dict(dtype=wpp.WPP_KV8), **kw))
        for call in (lambda: wpp.wpp_kv_append(Context, desc, x, x, k, v, x, x, x, plan, stream=Stream),
                     lambda: wpp.wpp_prefill_attention_varlen(Context, desc, x, x, None, k, v, x, x, x, plan, workspace=x, stream=Stream),
                     lambda: wpp.wpp_prefill_attention_varlen_static(Context, desc, x, x, None, k, v, x, x, x, plan, stream=Stream)):
            yield call
    good, both = u8(8, 2, block), u8(8, 2, 3, block)
    apart = dict(kv_page_stride=6 * block, kv_head_stride=3 * block)
    for k, v, kw in ((good, good, {}), (u8(9, 2, block), u8(8 * 2 * block), {}), (both, both[:, :, 2], apart), (both[:, :, 0], both.view(-1)[2 * block:], apart),
                     (good.view(torch.int8), good.view(torch.float8_e4m3fn), {}), (u8(8, 2, 2, 2, 2, block), torch.nn.Parameter(good, requires_grad=False), {}),
                     (None, None, {}), (Address(), Address(), {}), (x, x, dict(dtype=wpp.WPP_KV4)), (x, x, dict(dtype=wpp.WPP_BF16)), (x.byte(), x.byte(), dict(kv_page_stride=-16))):
        for call in run(k, v, **kw):
            n = len(calls)
            call()
            assert len(calls) == n + 1, kw
    for bad in (u8(7, 2, block), u8(8, 1, block), u8(8, 2, wpp.wpp_kv4_block_bytes(16, 64)), u8(8 * 2 * block - 1), good[1:], good[:0], u8(1, 2, block).expand(8, 2, block),
                torch.zeros(8, 2, block, dtype=torch.bfloat16), x):
        for k, v in ((bad, good), (good, bad)):
            for call in run(k, v):
                n = len(calls)
                with pytest.raises(wpp.WppError) as e:
                    call()
                assert e.value.status == 1 and len(calls) == n
    for call in run(both[:, :, 0], both[:, :, 1], kv_page_stride=6 * block, kv_head_stride=3 * block + 16):
        with pytest.raises(wpp.WppError) as e:
            call()
        assert e.value.status == 1


def test_a_head_shard_of_blocks_with_room_behind_them():
    """Bytes behind a block of 8 bits must not make one of 4 bits of it."""
    from paper_2609_35263_b200.stages import head_shard
    q, kv, block = torch.zeros(3, 8, 64), torch.zeros(3, 4, 64), wpp.wpp_kv8_block_bytes(16, 64)

    def shard(n, **kw):
        pool = torch.zeros(9, 4, n, dtype=kw.pop("of", torch.uint8))
        desc, views = head_shard(1, 2, 1, 8, 4, 64, 16, 9, 9, q, q, kv, kv, pool, pool, **kw)
        assert views["k_pool"].data_ptr() == pool[:, 2].data_ptr() and desc.kv_head_stride == n and desc.kv_page_stride == 4 * n
        return desc.dtype
    assert shard(block) == wpp.WPP_KV8 and shard(wpp.wpp_kv4_block_bytes(16, 64)) == wpp.WPP_KV4
    assert shard(640) == wpp.WPP_KV4                                    # (576 bytes of codes, and room)
    assert shard(block + 16, dtype=wpp.WPP_KV8) == wpp.WPP_KV8 and shard(block + 16, dtype=wpp.WPP_KV4) == wpp.WPP_KV4 == shard(block, dtype=wpp.WPP_KV4)
    with pytest.raises(ValueError, match="dtype"):
        shard(block + 16)
    for kw in (dict(dtype=wpp.WPP_BF16), dict(dtype=wpp.WPP_KV8, of=torch.bfloat16)):
        with pytest.raises(ValueError):
            shard(block, **kw)
