"""The cache held in 8 bits on the GPU: the append bit for bit, attention against 64 bits over what the codes stand for."""
import numpy as np
import pytest
import torch

import paper_2609_35263_b200 as wpp
from oracle import kv8 as okv8
from tests.kv8_harness import Wave, ctx

pytestmark = pytest.mark.gpu


def _bits(x):
    """bf16 bit patterns, cut off and not rounded (NaN and infinities stay what they are)."""
    return (np.ascontiguousarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)


def _same(g, w):
    assert np.array_equal(g["k"].cpu().numpy(), w.k_pool) and np.array_equal(g["v"].cpu().numpy(), w.v_pool) and int(g["status"].item()) == 0


# ---------------------------------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("d,B,Hkv", [(128, 64, 8), (64, 16, 2), (128, 16, 3), (64, 128, 1), (128, 32, 5), (128, 128, 2)])
@pytest.mark.parametrize("P,C", [([0], [1]), ([13, 0, 64, 127], [1, 1, 1, 1]), ([5, 0, 63, 200, 16], [40, 0, 3, 129, 16])])
@pytest.mark.parametrize("stands", ["lower", "higher"])
def test_append_is_exact_to_the_bit(d, B, Hkv, P, C, stands):
    """Prefix rows that stand in a page, of a scale that the new rows raise, or do not."""
    w = Wave(P, C, Hkv, Hkv, d, B, seed=d + B, scales=(-14, -9) if stands == "lower" else (-5, 3))
    g = w.device()
    w.append(g)
    w.appended()
    _same(g, w)


def test_append_of_values_of_any_size():
    """Zeros of both signs, NaN, infinities, the largest and the smallest numbers, values on halves, a page of nothing but zeros."""
    w = Wave([3], [157], 2, 2, 128, 32, seed=7)
    rng = np.random.default_rng(8)
    x = rng.integers(-64, 65, w.k_new.shape).astype(np.float32) / 8
    x[:29] *= 1e-6
    x[0, :, ::2] = -0.0
    x[1, :, 7], x[2, :, 70], x[3, :, 127] = np.nan, np.inf, -np.inf
    x[29:61] = np.where(rng.random(x[29:61].shape) < 0.5, 0.0, -0.0)                      # a page of zeros
    x[61:93] = np.exp(rng.standard_normal((32, 2, 128)) * 20)
    x[93:125] = np.float32(3.3e38) * np.sign(rng.standard_normal((32, 2, 128)))           # beyond the largest scale
    x[125:] = 1e-38
    w.k_new, w.v_new = _bits(x), _bits(x[::-1])
    g = w.device()
    w.append(g)
    w.appended()
    _same(g, w)


def test_append_of_every_code_and_halfway_between():
    w = Wave([0], [16], 1, 1, 64, 16, seed=9)
    grid = okv8.NUMBERS[:127]
    x = np.zeros((16, 1, 64), np.float32)
    x.reshape(-1)[:127], x.reshape(-1)[128:254] = grid, (grid[1:] + grid[:-1]) / 2
    x.reshape(-1)[256:383], x.reshape(-1)[384:510] = -grid, -(grid[1:] + grid[:-1]) / 2
    w.k_new = w.v_new = _bits(x)
    assert np.array_equal(okv8.bf16_values(w.k_new), x)
    g = w.device()
    w.append(g)
    w.appended()
    _same(g, w)


def test_append_of_many_rows_and_empty_requests():
    rng = np.random.default_rng(9)
    C = np.where(rng.random(300) < 0.5, 0, rng.integers(0, 60, 300))
    w = Wave(rng.integers(0, 100, 300), C, 4, 4, 64, 16, seed=9)
    w.table[C == 0] = -1                                               # (nothing of an empty chunk's request is looked at)
    g = w.device()
    w.append(g)
    w.appended()
    _same(g, w)


def test_append_token_by_token_raises_a_page_s_scale():
    w = Wave([5], [60], 2, 2, 64, 64, seed=10, scales=(-30, -30))
    w.k_new = _bits(okv8.bf16_values(w.k_new) * np.exp2(np.arange(60) / 3 - 8)[:, None, None])
    whole, row = w.device(), 0
    for n in (1,) * 40 + (7, 13):
        one = Wave([5 + row], [n], 2, 2, 64, 64)
        one.table, one.pages = w.table, w.pages
        one.k_new, one.v_new, one.k_pool, one.v_pool = w.k_new[row:row + n], w.v_new[row:row + n], w.k_pool, w.v_pool
        g = dict(one.device(), k=whole["k"], v=whole["v"])
        one.append(g)
        w.k_pool, w.v_pool = one.appended()
        _same(g, w)
        row += n


# ------------------------------------------------------------------------------------------------------------- attention
HEADS = [(64, 8, 128, 64), (8, 2, 64, 16), (40, 8, 128, 32), (6, 2, 128, 128), (32, 2, 64, 32), (4, 4, 128, 16), (20, 1, 128, 16),
         (33, 1, 64, 64), (14, 2, 128, 64), (8, 1, 64, 128)]


@pytest.mark.parametrize("Hq,Hkv,d,B", HEADS)
@pytest.mark.parametrize("P,C", [([0, 15, 16, 300], [1, 1, 1, 1]), ([0, 127, 129, 61], [2, 2, 4, 3]), ([0, 70, 0, 33], [7, 17, 40, 0])])
@pytest.mark.parametrize("splits", [0, 1, 3])
@pytest.mark.parametrize("shape", [1, 2])
def test_attention_of_few_rows(Hq, Hkv, d, B, P, C, splits, shape):
    w = Wave(P, C, Hq, Hkv, d, B, seed=Hq + d)
    g = w.device()
    out, lse = w.attend(g, opts=wpp.PlanOpts(0, 0, splits, 0, 0, shape))
    assert int(g["status"].item()) == 0
    w.check(out, lse, w.reference())


@pytest.mark.parametrize("Hq,Hkv,d,B", HEADS)
@pytest.mark.parametrize("P,C", [([0, 200], [129, 60]), ([77, 0, 5], [64, 257, 33])])
@pytest.mark.parametrize("splits", [0, 1, 2])
@pytest.mark.parametrize("shape", [1, 2])
def test_attention_of_chunks(Hq, Hkv, d, B, P, C, splits, shape):
    w = Wave(P, C, Hq, Hkv, d, B, seed=Hq + d + 1)
    g = w.device()
    out, lse = w.attend(g, opts=wpp.PlanOpts(0, 0, splits, 0, 0, shape))
    assert int(g["status"].item()) == 0
    w.check(out, lse, w.reference())


@pytest.mark.parametrize("C", [[1, 1], [2, 200], [2, 1200]])
def test_append_then_attention(C):
    """As a stage calls them: the new rows into the pages, then attention over all of them, one plan for both."""
    w = Wave([130, 61], C, 16, 4, 128, 32, seed=11)
    g = w.device()
    plan = w.plan()
    w.append(g, plan)
    out, lse = w.attend(g, plan)
    w.appended()
    w.check(out, lse, w.reference())
    _same(g, w)


@pytest.mark.parametrize("B", [16, 64])
@pytest.mark.parametrize("P,C", [([100, 3], [1, 1]), ([100, 3, 0], [2, 150, 40])])
@pytest.mark.parametrize("shape", [1, 2])
def test_what_lies_behind_a_sequence_never_counts(P, C, shape, B):
    """Slots behind the last row hold NaN codes, pages nobody names NaN codes and scales."""
    w = Wave(P, C, 8, 2, 128, B, seed=12)
    used = np.zeros((w.pages, w.B), bool)
    for i in range(len(P)):
        for j in range(P[i] + C[i]):
            used[w.table[i, j // w.B], j % w.B] = True
    for pool in (w.k_pool, w.v_pool):
        codes = pool[..., :B * 128].reshape(w.pages, 2, B, 128).copy()
        codes[np.repeat(~used[:, None], 2, 1)] = 255
        pool[..., :B * 128] = codes.reshape(w.pages, 2, -1)
        pool[~used.any(1)] = 255
    g = w.device()
    for splits in (1, 2):
        out, lse = w.attend(g, opts=wpp.PlanOpts(0, 0, splits, 0, 0, shape))
        w.check(out, lse, w.reference())


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("d,B", [(128, 32), (64, 16)])
@pytest.mark.parametrize("C", [4, 150])
@pytest.mark.parametrize("shape", [1, 2])
@pytest.mark.parametrize("splits", [1, 2])
def test_a_nan_code_reaches_the_rows_that_see_it_and_no_others(which, C, shape, splits, d, B):
    """Of V the output's element of the same place, of K all of the row."""
    w = Wave([90], [C], 8, 2, d, B, seed=13)
    good, hurt = w.reference(), 90 + C // 2
    for place, code in ((7, 0x7F), (d - 2, 0xFF)):
        (w.k_pool if which == "k" else w.v_pool)[w.table[0, hurt // B], 1, hurt % B * d + place] = code
    g = w.device()
    out, lse = w.attend(g, opts=wpp.PlanOpts(0, 0, splits, 0, 0, shape))
    o, hit = out.float().cpu().numpy(), np.zeros(out.shape, bool)
    hit[C // 2:, 4:] = True
    if which == "v":
        hit[..., [x for x in range(d) if x not in (7, d - 2)]] = False
    assert np.array_equal(np.isnan(o), hit)
    for x, y in zip(good, (out, lse)):
        x[hit if x.ndim == 3 else hit.any(-1)] = 0.0
        y[torch.from_numpy(hit if x.ndim == 3 else hit.any(-1)).cuda()] = 0.0
    w.check(out, lse if which == "k" else None, good)


@pytest.mark.parametrize("C", [1, 100])
@pytest.mark.parametrize("shape", [1, 2])
def test_scores_that_keep_growing(C, shape):
    """Keys that get longer along the sequence: the references move all the time."""
    w = Wave([500], [C], 8, 2, 128, 64, seed=14, sm_scale=0.3)
    for j, page in enumerate(w.table[0]):
        w.k_pool[page, :, 64 * 128:64 * 128 + 4] = np.array([2.0 ** (j // 2 - 8)], np.float32).view(np.uint8)
    g = w.device()
    out, lse = w.attend(g, opts=wpp.PlanOpts(0, 0, 0, 0, 0, shape))
    w.check(out, lse, w.reference())


@pytest.mark.parametrize("shape", [1, 2])
@pytest.mark.parametrize("factor", [2.0 ** -60, 2.0 ** 40, 3.0])
def test_queries_of_any_size(shape, factor):
    """Rows of unequal elements: a query whose largest element is far above the others, zeros, one of nothing but zeros."""
    w = Wave([300], [40], 8, 2, 128, 64, seed=15, sm_scale=0.1 / factor)
    q = okv8.bf16_values(w.q) * np.exp2(np.random.default_rng(2).integers(-12, 1, w.q.shape)) * factor
    q[3], q[5, :, ::2] = 0.0, 0.0
    w.q = okv8.bf16_bits(q.astype(np.float32))
    g = w.device()
    out, lse = w.attend(g, opts=wpp.PlanOpts(0, 0, 0, 0, 0, shape))
    w.check(out, lse, w.reference())


@pytest.mark.parametrize("C", [1, 90])
@pytest.mark.parametrize("shape", [1, 2])
def test_strides(C, shape):
    """K and V blocks side by side in one allocation, queries and new rows out of one packed buffer, outputs inside a larger one."""
    w = Wave([40, 7], [C, 2], 8, 2, 64, 16, seed=15)
    block = wpp.wpp_kv8_block_bytes(16, 64)
    g = w.device()
    both = torch.full((w.pages, 2, 3, block), 255, dtype=torch.uint8, device="cuda")
    both[:, :, 0], both[:, :, 2] = g["k"], g["v"]
    packed = torch.randn(w.T, 16, 72, device="cuda").bfloat16()
    packed[:, :8, :64], packed[:, 8:10, :64], packed[:, 10:12, :64] = g["q"], g["k_new"], g["v_new"]
    kw = dict(kv_page_stride=6 * block, kv_head_stride=3 * block, q_token_stride=16 * 72, q_head_stride=72, kvnew_token_stride=16 * 72,
              kvnew_head_stride=72, o_token_stride=10 * 80, o_head_stride=80)
    desc, plan = w.desc(**kw), w.plan(wpp.PlanOpts(0, 0, 0, 0, 0, shape), **kw)
    wpp.wpp_kv_append(ctx(), desc, packed[:, 8:], packed[:, 10:], both, both[:, :, 2], g["table"], g["P"], g["C"], plan, status=g["status"])
    out = torch.full((w.T, 10, 80), 5.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(int(plan.info.workspace_bytes), dtype=torch.uint8, device="cuda")
    wpp.wpp_prefill_attention_varlen(ctx(), desc, packed, out, None, both, both[:, :, 2], g["table"], g["P"], g["C"], plan, workspace=ws,
                                     status=g["status"])
    w.appended()
    got = both.cpu().numpy()
    assert np.array_equal(got[:, :, 0], w.k_pool) and np.array_equal(got[:, :, 2], w.v_pool) and (got[:, :, 1] == 255).all()
    w.check(out[:, :8, :64].contiguous(), None, w.reference())
    rest = out.float().cpu().numpy()
    rest[:, :8, :64] = 5.0
    assert (rest == 5.0).all() and int(g["status"].item()) == 0


@pytest.mark.parametrize("shape", [1, 2])
def test_offsets_beyond_32_bits(shape):
    """Pages 2^28 bytes apart: the pool's end lies behind 2^32 bytes."""
    w = Wave([150, 70], [1, 65], 8, 1, 128, 16, seed=16)
    g = w.device()
    stride = 1 << 28
    big = torch.empty(w.pages * stride, dtype=torch.uint8, device="cuda").view(w.pages, stride)
    n = wpp.wpp_kv8_block_bytes(16, 128)
    big[:, :n], big[:, n:2 * n] = g["k"][:, 0], g["v"][:, 0]
    assert w.pages * stride > 1 << 32
    kw = dict(kv_page_stride=stride)
    desc, plan = w.desc(**kw), w.plan(wpp.PlanOpts(0, 0, 0, 0, 0, shape), **kw)
    v = big.view(-1)[n:]
    out = torch.empty(w.T, 8, 128, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(int(plan.info.workspace_bytes), dtype=torch.uint8, device="cuda")
    wpp.wpp_kv_append(ctx(), desc, g["k_new"], g["v_new"], big, v, g["table"], g["P"], g["C"], plan, status=g["status"])
    wpp.wpp_prefill_attention_varlen(ctx(), desc, g["q"], out, None, big, v, g["table"], g["P"], g["C"], plan, workspace=ws, status=g["status"])
    w.appended()
    w.check(out, None, w.reference())
    assert np.array_equal(big[:, :n].cpu().numpy(), w.k_pool[:, 0])


# ---------------------------------------------------------------------------------------------- refusals, streams, capture
@pytest.mark.parametrize("shape", [1, 2])
def test_other_lengths_than_the_plans_are_refused_per_request(shape):
    w = Wave([50, 20, 30], [1, 100, 2], 8, 2, 128, 32, seed=17)
    good = w.reference()
    g = w.device()
    plan = w.plan(wpp.PlanOpts(0, 0, 2, 0, 0, shape))
    before = w.k_pool
    w.appended()
    for name, i in (("P", 0), ("C", 1)):
        h = dict(g, status=torch.zeros_like(g["status"]), k=g["k"].clone(), v=g["v"].clone())
        h[name] = g[name].clone()
        h[name][i] += -1 if name == "C" else 1
        out, lse = w.attend(h, plan)
        assert int(h["status"].item()) == 6
        o, at = out.double().cpu().numpy(), np.concatenate([[0], np.cumsum(w.C)])
        for j in range(3):
            rows = slice(at[j], at[j + 1])
            if j != i:
                assert np.all(np.abs(o[rows] - good[0][rows]) <= 2.0 ** -7 * (np.abs(good[0][rows]) + good[2][rows]))
        w.append(h, plan)
        for j in range(3):
            pages = w.table[j][w.table[j] >= 0]
            assert np.array_equal(h["k"].cpu().numpy()[pages], (before if j == i else w.k_pool)[pages])


@pytest.mark.parametrize("shape", [1, 2])
def test_a_bad_page_id_is_reported(shape):
    for C in ([1], [140]):
        w = Wave([100], C, 8, 2, 64, 32, seed=18)
        for bad in (-1, w.pages, 2 ** 31 - 1):
            g = w.device()
            g["table"][0, 1] = bad
            w.attend(g, opts=wpp.PlanOpts(0, 0, 0, 0, 0, shape))
            assert int(g["status"].item()) == 3
            g["status"].zero_()
            g["table"][0, 1] = int(w.table[0, 1])
            g["table"][0, -1] = bad
            k = g["k"].clone()
            w.append(g)
            assert int(g["status"].item()) == 3
            keep = [p for p in range(w.pages) if p not in w.table[0]]
            assert torch.equal(g["k"][keep], k[keep])


def test_refusals_before_a_launch():
    w = Wave([100], [1], 8, 2, 64, 32, seed=19)
    g, plan = w.device(), w.plan(wpp.PlanOpts(0, 0, 1, 0))
    n = ctx().launch_count()

    def attend(status, **kw):
        a = dict(g, workspace=torch.empty(int(plan.info.workspace_bytes), dtype=torch.uint8, device="cuda"), out=torch.empty_like(g["q"]))
        a.update(kw)
        with pytest.raises(wpp.WppError) as e:
            wpp.wpp_prefill_attention_varlen(ctx(), w.desc(), a["q"], a["out"], None, a["k"], a["v"], a["table"], a["P"], a["C"], plan,
                                             workspace=a["workspace"], status=a["status"])
        assert e.value.status == status
    attend(5, workspace=torch.empty(128, dtype=torch.uint8, device="cuda"))
    attend(1, workspace=None)
    attend(1, q=None)
    attend(1, k=g["k"].view(-1)[4:])
    attend(1, out=g["q"].view(-1)[1:])
    with pytest.raises(wpp.WppError) as e:
        wpp.wpp_kv_append(ctx(), w.desc(), g["k_new"], g["v_new"], g["k"], g["v"].view(-1)[8:], g["table"], g["P"], g["C"], plan)
    assert e.value.status == 1 and ctx().launch_count() == n


def test_the_built_in_scratch():
    w = Wave([700], [3], 8, 2, 128, 32, seed=20)
    g, plan = w.device(), w.plan(wpp.PlanOpts(0, 0, 3, 0))
    out, lse = w.attend(g, plan)
    again, sums = torch.zeros_like(out), torch.zeros_like(lse)
    wpp.wpp_prefill_attention_varlen_static(ctx(), w.desc(), g["q"], again, sums, g["k"], g["v"], g["table"], g["P"], g["C"], plan,
                                            status=g["status"])
    assert torch.equal(out, again) and torch.equal(lse, sums)


@pytest.mark.parametrize("C", [[1, 1, 1], [1, 40, 150], [1, 40, 950]])
@pytest.mark.parametrize("shape", [0, 1])
def test_captured_and_replayed_and_on_two_streams(C, shape):
    w = Wave([300, 64, 0], C, 16, 4, 128, 64, seed=21)
    g, plan = w.device(), w.plan(wpp.PlanOpts(0, 0, 2, 0, 0, shape))
    out, lse = w.attend(g, plan)
    ws = [torch.full((int(plan.info.workspace_bytes),), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = [torch.empty_like(out) for _ in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s, x, o in zip(streams, ws, outs):
        wpp.wpp_prefill_attention_varlen(ctx(), w.desc(), g["q"], o, None, g["k"], g["v"], g["table"], g["P"], g["C"], plan, workspace=x,
                                         status=g["status"], stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], out) and torch.equal(outs[1], out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        w.append(g, plan)
        wpp.wpp_prefill_attention_varlen(ctx(), w.desc(), g["q"], outs[0], None, g["k"], g["v"], g["table"], g["P"], g["C"], plan,
                                         workspace=ws[0], status=g["status"])
    w.appended()
    for _ in range(3):
        outs[0].zero_()
        graph.replay()
        torch.cuda.synchronize()
        _same(g, w)
    w.check(outs[0], None, w.reference())


def test_head_shards_of_its_pools():
    from paper_2609_35263_b200 import stages
    w = Wave([90, 33], [1, 40], 16, 4, 128, 32, seed=22)
    g = w.device()
    out = torch.empty_like(g["q"])
    for rank in range(2):
        desc, v = stages.head_shard(rank, 2, 2, 16, 4, 128, 32, w.table.shape[1], w.pages, g["q"], out, g["k_new"], g["v_new"], g["k"], g["v"])
        assert desc.dtype == wpp.WPP_KV8
        plan = wpp.wpp_plan_tiles(ctx(), desc, w.P, w.C).to_device()
        ws = torch.empty(int(plan.info.workspace_bytes), dtype=torch.uint8, device="cuda")
        wpp.wpp_kv_append(ctx(), desc, v["k_new"], v["v_new"], v["k_pool"], v["v_pool"], g["table"], g["P"], g["C"], plan, status=g["status"])
        wpp.wpp_prefill_attention_varlen(ctx(), desc, v["q"], v["out"], None, v["k_pool"], v["v_pool"], g["table"], g["P"], g["C"], plan,
                                         workspace=ws, status=g["status"])
    w.appended()
    _same(g, w)
    w.check(out, None, w.reference())


# --------------------------------------------------------------------------------------------------- pages of unequal sizes
def _along(w, rng, scores, values):
    """Keys whose score with every query is about scores[j] (natural logarithms) and value rows values[j], of request 0 and head 0."""
    n, d = values.shape
    base = rng.standard_normal(d)
    w.q = okv8.bf16_bits(np.broadcast_to(base, w.q.shape).astype(np.float32) + 0.02 * rng.standard_normal(w.q.shape).astype(np.float32))
    keys = scores[:, None] * base / (d ** -0.5 * (base @ base)) + 0.05 * rng.standard_normal((n, d))
    fill = Wave([0], [n], 1, 1, d, w.B)
    fill.table, fill.pages, fill.k_pool, fill.v_pool = w.table, w.pages, w.k_pool, w.v_pool
    fill.k_new, fill.v_new = (okv8.bf16_bits(x.astype(np.float32))[:, None] for x in (keys, values))
    w.k_pool, w.v_pool = fill.appended()


def _values(kind, n, d, rng):
    """(scores, value rows) of n keys."""
    scores, values = rng.uniform(-3, 3, n), rng.standard_normal((n, d))
    if kind.startswith("one wide row that nobody attends to"):
        scores[n // 3], values[n // 3] = -60.0, values[n // 3] * 2.0 ** int(kind.split()[-1])
    elif kind.startswith("a dominant key, a flat tail and one wide row"):
        gap, width = (float(x) for x in kind.split()[-2:])
        scores[:], scores[5] = 0.0, gap * np.log(2)
        values[:] = values[0]
        values[n // 2] *= width
    elif kind == "a dominant key beside a wide row that takes its codes":
        scores[40], scores[41], values[41] = 12.0, -60.0, values[41] * 2.0 ** 36
    elif kind == "tiny":                                               # (scales just above 2^-56, below which a page has none)
        values *= 2.0 ** -49
    elif kind == "large":
        values *= 2.0 ** 46
    elif kind == "pages of any size":
        values *= 2.0 ** np.repeat(rng.uniform(-30, 30, (n + 63) // 64), 64)[:n, None]
    elif kind == "wider as the scores fall":
        scores = np.linspace(25, -25, n)
        values *= np.exp(-scores[:, None])
    elif kind == "narrower as the scores rise":
        scores = np.linspace(-25, 25, n)
        values *= np.exp(-scores[:, None])
    elif kind == "rows of zeros behind others":
        scores[n // 2:] += np.linspace(0, 70, n - n // 2)
        values[n // 2:] = 0.0
    return scores, values


@pytest.mark.parametrize("kind", [f"one wide row that nobody attends to, 2 ** {e}" for e in (6, 20, 40)] +
                         [f"a dominant key, a flat tail and one wide row, {a} {b}" for a, b in ((18, 256), (16, 1000), (14, 4000))] +
                         ["a dominant key beside a wide row that takes its codes", "tiny", "large", "pages of any size", "wider as the scores fall",
                          "narrower as the scores rise", "rows of zeros behind others"])
@pytest.mark.parametrize("d,Hq,C,n", [(128, 4, 1, 12000), (64, 5, 3, 3000), (128, 3, 40, 1100)])
def test_value_pages_of_unequal_sizes(kind, d, Hq, C, n):
    """What a row of V weighs decides what it does, not how wide its page is."""
    w = Wave([n - C], [C], Hq, 1, d, 64, seed=n + d)
    rng = np.random.default_rng(n)
    _along(w, rng, *_values(kind, n, d, rng))
    g, ref = w.device(), w.reference()
    for shape, splits in ((2, 1), (2, 3), (1, 1), (1, 2)):
        out, lse = w.attend(g, opts=wpp.PlanOpts(0, 0, splits, 0, 0, shape))
        assert int(g["status"].item()) == 0
        w.check(out, lse, ref)


# ------------------------------------------------------------------------------------------------ how units reach the CTAs
DEALS = {"dealt": (([3000, 500, 2000, 10, 7000], [1, 2, 1, 1, 1], 8, 4), 2), "dealt, with tiles": (([9000, 9000, 600, 4000, 8000], [1, 1, 400, 1, 1], 8, 4), 2),
         "cluster of 16": (([8191], [1], 8, 2), 0), "cluster of 8": (([5000, 700, 3], [1, 3, 2], 16, 8), 0), "cluster of 4": (([2000] * 8, [1] * 8, 16, 8), 0),
         "cluster of 2": (([1200, 600, 64] * 8, [1] * 24, 6, 6), 0), "cluster, two row blocks": (([3000], [3], 12, 1), 0), "tail cut": (([3000, 3000], [300, 300], 4, 1), 4)}


@pytest.mark.parametrize("d,B", [(128, 32), (64, 16)])
@pytest.mark.parametrize("name", list(DEALS))
def test_parts_that_are_dealt_out_joined_in_clusters_or_cut_from_the_last_tiles(name, d, B):
    """Every way a plan has of spreading a wave, with a workspace full of ones, twice in a row, replayed, and with a request that is refused."""
    (P, C, Hq, Hkv), ctas = DEALS[name]
    w = Wave(P, C, Hq, Hkv, d, B, seed=len(P) + d)
    g, plan = w.device(), w.plan(wpp.PlanOpts(0, 0, 0, ctas))
    ref = w.reference()
    ws = torch.full((int(plan.info.workspace_bytes),), 255, dtype=torch.uint8, device="cuda")
    out, lse = w.attend(g, plan, workspace=ws)
    again, sums = w.attend(g, plan, workspace=ws)
    assert int(g["status"].item()) == 0 and torch.equal(out, again) and torch.equal(lse, sums)
    w.check(out, lse, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wpp.wpp_prefill_attention_varlen(ctx(), w.desc(), g["q"], again, sums, g["k"], g["v"], g["table"], g["P"], g["C"], plan, workspace=ws, status=g["status"])
    for _ in range(3):
        again.zero_()
        graph.replay()
    assert torch.equal(out, again) and torch.equal(lse, sums)
    g["P"][0] += 1
    again.fill_(7.0)
    graph.replay()
    rows = slice(C[0], None)
    assert int(g["status"].item()) == 6 and torch.equal(out[rows], again[rows])


@pytest.mark.parametrize("name", list(DEALS))
def test_a_plan_that_the_kernel_before_writes_and_the_built_in_scratch(name):
    """The append and the attention see the plan that stands in plan_dev when the work before them has ended; the array of the library
    serves for every way of spreading a wave."""
    (P, C, Hq, Hkv), ctas = DEALS[name]
    w = Wave(P, C, Hq, Hkv, 128, 32, seed=len(P))
    g, plan = w.device(), w.plan(wpp.PlanOpts(0, 0, 0, ctas))
    w.append(g, plan)
    out, lse = w.attend(g, plan)
    pools, sums, ws = (g["k"].clone(), g["v"].clone()), torch.zeros_like(lse), torch.full((int(plan.info.workspace_bytes),), 255, dtype=torch.uint8, device="cuda")
    bits = plan.dev.clone()
    for _ in range(3):
        again = torch.zeros_like(out)
        g["k"].copy_(torch.from_numpy(w.k_pool)), g["v"].copy_(torch.from_numpy(w.v_pool))
        plan.dev.zero_()
        torch.cuda.synchronize()
        torch.bitwise_or(bits, 0, out=plan.dev)
        w.append(g, plan)
        plan.dev.zero_()
        torch.bitwise_or(bits, 0, out=plan.dev)
        wpp.wpp_prefill_attention_varlen(ctx(), w.desc(), g["q"], again, sums, g["k"], g["v"], g["table"], g["P"], g["C"], plan, workspace=ws, status=g["status"])
        assert torch.equal(out, again) and torch.equal(lse, sums) and torch.equal(g["k"], pools[0]) and torch.equal(g["v"], pools[1])
    again.zero_(), sums.zero_()
    wpp.wpp_prefill_attention_varlen_static(ctx(), w.desc(), g["q"], again, sums, g["k"], g["v"], g["table"], g["P"], g["C"], plan, status=g["status"])
    assert torch.equal(out, again) and torch.equal(lse, sums) and int(g["status"].item()) == 0


def test_a_nan_score_in_a_part_that_a_cluster_joins():
    w = Wave([8191], [1], 8, 2, 128, 64, seed=3)
    w.k_pool[w.table[0, 50], 1, 5] = 0x7F
    w.v_pool[w.table[0, 90], 0, 64 * 128 - 1] = 0xFF
    g = w.device()
    out, lse = w.attend(g)
    o = out.float().cpu().numpy()
    assert np.isnan(o[0, 4:]).all() and np.isnan(o[0, :4, 127]).all() and not np.isnan(o[0, :4, :127]).any()
    assert torch.isinf(lse[0, 4:]).all() and torch.isfinite(lse[0, :4]).all()


def test_a_long_cache():
    """131,072 keys of one request; values that the sums' order would show in, were they not added up in fp32."""
    w = Wave([131071], [1], 8, 1, 64, 128, seed=4)
    g = w.device()
    for opts in (None, wpp.PlanOpts(0, 0, 0, 0, 0, 1), wpp.PlanOpts(0, 0, 0, 8)):
        out, lse = w.attend(g, opts=opts)
        w.check(out, lse, w.reference())


# ---------------------------------------------------------------------------------------------------- NaN codes in any step
@pytest.mark.parametrize("d,B", [(128, 64), (64, 16)])
@pytest.mark.parametrize("shape,splits", [(1, 1), (1, 2), (2, 1), (2, 3)])
@pytest.mark.parametrize("apart", [0, 6, -14, 20])
def test_a_nan_code_of_v_behind_which_every_row_stands(d, B, shape, splits, apart):
    """A key that all rows see, far from the diagonal, in a page whose scale is 2^apart times the others'."""
    w = Wave([900], [150], 8, 2, d, B, seed=31, scales=(-8, -8))
    page, slot = w.table[0, 500 // B], 500 % B
    w.v_pool[page, 1, B * d:B * d + 4] = np.array([2.0 ** (apart - 8)], np.float32).view(np.uint8)
    good = w.reference()
    w.v_pool[page, 1, [slot * d + 7, slot * d + d - 2]] = 0x7F, 0xFF
    g = w.device()
    out, lse = w.attend(g, opts=wpp.PlanOpts(0, 0, splits, 0, 0, shape))
    hit = np.zeros(out.shape, bool)
    hit[:, 4:, [7, d - 2]] = True
    assert np.array_equal(np.isnan(out.float().cpu().numpy()), hit)
    for x, y in zip(good, (out, None, None, None)):
        if x.ndim == 3:
            x[hit] = 0.0
        if y is not None:
            y[torch.from_numpy(hit).cuda()] = 0.0
    w.check(out, lse, good)


@pytest.mark.parametrize("d,B", [(128, 64), (64, 16)])
@pytest.mark.parametrize("shape,splits", [(1, 1), (1, 2), (2, 1), (2, 3)])
def test_a_page_of_infinite_values_as_the_append_leaves_it(d, B, shape, splits):
    """Nothing in it is finite: its scale is the least there is, 2^48 below the others'."""
    w = Wave([10 * B + 400], [150], 8, 2, d, B, seed=32, scales=(-8, -8))
    good = w.reference()
    fill = Wave([5 * B], [B], 8, 2, d, B, seed=33)
    fill.table, fill.pages, fill.k_pool, fill.v_pool = w.table, w.pages, w.k_pool, w.v_pool
    x = okv8.bf16_values(fill.v_new).copy()
    x[:, 1] = np.where(np.arange(B * d).reshape(B, d) % 3 == 0, np.nan, np.inf)
    fill.v_new = _bits(x)
    g = fill.device()
    fill.append(g)
    w.k_pool, w.v_pool = fill.appended()
    _same(g, w)
    assert okv8.block_scale(w.v_pool[w.table[0, 5], 1], B, d) == 2.0 ** -56
    hit = np.zeros(good[0].shape, bool)
    hit[:, 4:] = True
    out, lse = w.attend(w.device(), opts=wpp.PlanOpts(0, 0, splits, 0, 0, shape))
    assert np.array_equal(np.isnan(out.float().cpu().numpy()), hit)
    w.v_pool[w.table[0, 5], 1] = 0                                      # (of the heads that see nothing of it, and of the sums)
    w.v_pool[w.table[0, 5], 1, B * d:B * d + 4] = np.array([1.0], np.float32).view(np.uint8)
    good = w.reference()
    for i in (0, 2, 3):
        good[i][hit] = 0.0
    out[torch.from_numpy(hit).cuda()] = 0.0
    w.check(out, lse, good)


# ----------------------------------------------------------------------------------------------- probabilities far apart
@pytest.mark.parametrize("gap", [12.0, 18.0, 23.45, 28.0])
@pytest.mark.parametrize("shape,splits", [(1, 1), (1, 2), (2, 1), (2, 3)])
@pytest.mark.parametrize("d,Hq,C", [(128, 4, 40), (64, 4, 130), (128, 2, 2)])
def test_a_key_far_above_a_flat_tail_leaves_it_its_weight(gap, shape, splits, d, Hq, C):
    """One of the first keys 2^gap above all others, with a value of zeros, so that the output is the others'.  Scores are one product each.  A
    probability is off by 2^-11 of itself or by 2^-25, half of f16's last step, where the largest is from 2^7 on (few rows: whose reference is
    a whole number, from 2^6 on); the exponent by five roundings of 2^-24 of a number below 2^5,
    its power by 2^-22, the sums over at most 2^7 steps by 2^-23 each: under 2^-14 together; the result by 2^-8."""
    n = 1500
    w = Wave([n - C], [C], Hq, 1, d, 64, seed=34, sm_scale=gap * np.log(2))
    q, k, v = np.zeros((C, Hq, d), np.float32), np.zeros((n, 1, d), np.float32), np.ones((n, 1, d), np.float32)
    q[..., 0], k[5, 0, 0], v[5] = 1.0, 1.0, 0.0
    w.q = okv8.bf16_bits(q)
    fill = Wave([0], [n], 1, 1, d, 64)
    fill.table, fill.pages, fill.k_pool, fill.v_pool, fill.k_new, fill.v_new = w.table, w.pages, w.k_pool, w.v_pool, okv8.bf16_bits(k), okv8.bf16_bits(v)
    w.k_pool, w.v_pool = fill.appended()
    out, _ = w.attend(w.device(), opts=wpp.PlanOpts(0, 0, splits, 0, 0, shape))
    o, _, spread, even = w.reference()
    got = out.double().cpu().numpy()
    tol = (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -14) * np.abs(o) + 2.0 ** (-32 if shape == 1 else -31) * even
    assert np.all(np.abs(got - o) <= tol), float((np.abs(got - o) / tol).max())


@pytest.mark.parametrize("shape,splits", [(1, 1), (1, 2), (2, 1), (2, 3), (0, 0)])
@pytest.mark.parametrize("d,Hq,C", [(128, 4, 40), (64, 4, 130), (128, 2, 1)])
def test_probabilities_have_the_bits_of_f16_where_the_scales_of_v_are_near(shape, splits, d, Hq, C):
    """Keys of two kinds, whose weights differ by 0.45 * 2^-8 and whose values are 1 and -1: with probabilities of 8 bits both would weigh the
    same, and the output would be off by 0.45 * 2^-9 of `spread`, above the 2^-11 that it may be.  (Scores are one product each, below 2^-9:
    their errors, those of the exponents around 2^3 and of the power are under 2^-18; the sums' under 2^-15.)"""
    n = 1500
    w = Wave([n - C], [C], Hq, 1, d, 64, seed=35, sm_scale=-np.log(1 - 0.45 * 2.0 ** -8))
    q, k, v = np.zeros((C, Hq, d), np.float32), np.zeros((n, 1, d), np.float32), np.ones((n, 1, d), np.float32)
    q[..., 0], k[::2, 0, 0], v[::2] = 1.0, 1.0, -1.0
    w.q = okv8.bf16_bits(q)
    fill = Wave([0], [n], 1, 1, d, 64)
    fill.table, fill.pages, fill.k_pool, fill.v_pool, fill.k_new, fill.v_new = w.table, w.pages, w.k_pool, w.v_pool, okv8.bf16_bits(k), okv8.bf16_bits(v)
    w.k_pool, w.v_pool = fill.appended()
    out, _ = w.attend(w.device(), opts=wpp.PlanOpts(0, 0, splits, 0, 0, shape))
    o, _, spread, _ = w.reference()
    got = out.double().cpu().numpy()
    tol = 2.0 ** -8 * np.abs(o) + (2.0 ** -11 + 2.0 ** -15) * spread
    assert np.all(np.abs(got - o) <= tol), float((np.abs(got - o) / tol).max())
