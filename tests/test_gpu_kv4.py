"""The cache held in 4 bits on the GPU: the append bit for bit, attention against 64 bits over what the codes stand for."""
import numpy as np
import pytest
import torch

import paper_2609_35263_b200 as wpp
from oracle import kv4 as okv4
from tests.kv4_harness import Wave, ctx

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("d,B,Hkv", [(128, 64, 8), (64, 16, 2), (128, 16, 3), (64, 128, 1), (128, 32, 5)])
@pytest.mark.parametrize("P,C", [([0], [1]), ([13, 0, 64, 127], [1, 1, 1, 1]), ([5, 0, 63, 200, 16], [40, 0, 3, 129, 16])])
def test_append_is_exact_to_the_bit(d, B, Hkv, P, C):
    w = Wave(P, C, Hkv, Hkv, d, B, seed=d + B)
    g = w.device()
    w.append(g)
    k, v = okv4.append(w.k_new, w.v_new, w.k_pool, w.v_pool, w.table, w.P, w.C, w.B)
    assert int(g["status"].item()) == 0
    assert np.array_equal(g["k"].cpu().numpy(), k) and np.array_equal(g["v"].cpu().numpy(), v)


def test_append_of_rows_that_have_no_scale_and_of_quotients_on_halves():
    w = Wave([3], [40], 2, 2, 128, 32, seed=7)
    rng = np.random.default_rng(8)
    x = rng.integers(-64, 65, w.k_new.shape).astype(np.float32) / 8               # many quotients lie on a half
    x[0] = 2.5
    x[1] = np.where(rng.random(x[1].shape) < 0.5, 0.0, -0.0)
    x[2, :, 7] = np.nan
    x[3, :, 70] = np.inf
    x[4, :, 127] = -np.inf
    x[5, :, :2] = [3.3e38, -3.3e38]
    x[6] *= 1e-36
    x[7] = 1e-38
    x[8] *= 1e36
    x[9] = x[9] * 1e-6 + 100.0
    x[10] = np.exp(rng.standard_normal(x[10].shape) * 20)
    w.k_new = (np.ascontiguousarray(x).view(np.uint32) >> 16).astype(np.uint16)
    w.v_new = w.k_new[::-1].copy()
    g = w.device()
    w.append(g)
    k, v = okv4.append(w.k_new, w.v_new, w.k_pool, w.v_pool, w.table, w.P, w.C, w.B)
    assert np.array_equal(g["k"].cpu().numpy(), k) and np.array_equal(g["v"].cpu().numpy(), v)


def test_append_of_many_rows_and_empty_requests():
    rng = np.random.default_rng(9)
    C = np.where(rng.random(300) < 0.5, 0, rng.integers(0, 60, 300))
    w = Wave(rng.integers(0, 100, 300), C, 4, 4, 64, 16, seed=9)
    g = w.device()
    w.append(g)
    k, v = okv4.append(w.k_new, w.v_new, w.k_pool, w.v_pool, w.table, w.P, w.C, w.B)
    assert np.array_equal(g["k"].cpu().numpy(), k) and np.array_equal(g["v"].cpu().numpy(), v)


# ------------------------------------------------------------------------------------------------------------- attention
HEADS = [(64, 8, 128, 64), (8, 2, 64, 16), (40, 8, 128, 32), (6, 2, 128, 128), (32, 2, 64, 32), (4, 4, 128, 16), (20, 1, 128, 16),
         (33, 1, 64, 64), (14, 2, 128, 64)]


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
    w.k_pool, w.v_pool = okv4.append(w.k_new, w.v_new, w.k_pool, w.v_pool, w.table, w.P, w.C, w.B)
    w.check(out, lse, w.reference())
    assert int(g["status"].item()) == 0


@pytest.mark.parametrize("P,C", [([100, 3], [1, 1]), ([100, 3, 0], [2, 150, 40])])
@pytest.mark.parametrize("shape", [1, 2])
def test_what_lies_behind_a_sequence_never_counts(P, C, shape):
    """Slots behind the last row and pages nobody names hold all ones: NaN pairs."""
    w = Wave(P, C, 8, 2, 128, 64, seed=12)
    used = np.zeros((w.pages, w.B), bool)
    for i in range(len(P)):
        for j in range(P[i] + C[i]):
            used[w.table[i, j // w.B], j % w.B] = True
    unused = np.repeat(~used[:, None], 2, 1)
    for pool in (w.k_pool, w.v_pool):
        codes, pairs = pool[..., :w.B * 64].reshape(w.pages, 2, w.B, 64), pool[..., w.B * 64:].reshape(w.pages, 2, w.B, 4)
        codes[unused], pairs[unused] = 255, 255
        pool[..., :w.B * 64], pool[..., w.B * 64:] = codes.reshape(w.pages, 2, -1), pairs.reshape(w.pages, 2, -1)
    g = w.device()
    for splits in (1, 2):
        out, lse = w.attend(g, opts=wpp.PlanOpts(0, 0, splits, 0, 0, shape))
        w.check(out, lse, w.reference())


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("C", [4, 150])
@pytest.mark.parametrize("shape", [1, 2])
@pytest.mark.parametrize("splits", [1, 2])
def test_a_nan_row_reaches_the_rows_that_see_it_and_no_others(which, C, shape, splits):
    w = Wave([90], [C], 8, 2, 128, 32, seed=13)
    hurt = 90 + C // 2
    pool = w.k_pool if which == "k" else w.v_pool
    okv4.write_row(pool, w.table[0, hurt // w.B], 1, hurt % w.B, w.B, np.zeros(w.d, np.uint8), np.array([0x7FC0, 0], np.uint16))
    g = w.device()
    out, _ = w.attend(g, opts=wpp.PlanOpts(0, 0, splits, 0, 0, shape))
    o = out.float().cpu().numpy()
    assert not np.isnan(o[:, :4]).any() and not np.isnan(o[:C // 2]).any() and np.isnan(o[C // 2:, 4:]).all()


@pytest.mark.parametrize("C", [1, 100])
@pytest.mark.parametrize("shape", [1, 2])
def test_scores_that_keep_growing(C, shape):
    """Keys that get longer along the sequence: the references move all the time."""
    w = Wave([500], [C], 8, 2, 128, 64, seed=14, sm_scale=0.3)
    codes, pairs = okv4.pack_rows(okv4.bf16_bits((np.random.default_rng(1).standard_normal((500 + C, 2, 128))
                                                  * np.linspace(0.1, 12, 500 + C)[:, None, None]).astype(np.float32)))
    for j in range(500 + C):
        for h in range(2):
            okv4.write_row(w.k_pool, w.table[0, j // 64], h, j % 64, 64, codes[j, h], pairs[j, h])
    g = w.device()
    out, lse = w.attend(g, opts=wpp.PlanOpts(0, 0, 0, 0, 0, shape))
    w.check(out, lse, w.reference())


@pytest.mark.parametrize("C", [1, 90])
@pytest.mark.parametrize("shape", [1, 2])
def test_strides(C, shape):
    """K and V blocks side by side in one allocation, queries and new rows out of one packed buffer, outputs inside a larger one."""
    w = Wave([40, 7], [C, 2], 8, 2, 64, 16, seed=15)
    block = wpp.wpp_kv4_block_bytes(16, 64)
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
    w.k_pool, w.v_pool = okv4.append(w.k_new, w.v_new, w.k_pool, w.v_pool, w.table, w.P, w.C, w.B)
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
    n = wpp.wpp_kv4_block_bytes(16, 128)
    big[:, :n], big[:, n:2 * n] = g["k"][:, 0], g["v"][:, 0]
    assert w.pages * stride > 1 << 32
    kw = dict(kv_page_stride=stride)
    desc, plan = w.desc(**kw), w.plan(wpp.PlanOpts(0, 0, 0, 0, 0, shape), **kw)
    v = big.view(-1)[n:]
    out = torch.empty(w.T, 8, 128, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(int(plan.info.workspace_bytes), dtype=torch.uint8, device="cuda")
    wpp.wpp_kv_append(ctx(), desc, g["k_new"], g["v_new"], big, v, g["table"], g["P"], g["C"], plan, status=g["status"])
    wpp.wpp_prefill_attention_varlen(ctx(), desc, g["q"], out, None, big, v, g["table"], g["P"], g["C"], plan, workspace=ws, status=g["status"])
    w.k_pool, w.v_pool = okv4.append(w.k_new, w.v_new, w.k_pool, w.v_pool, w.table, w.P, w.C, w.B)
    w.check(out, None, w.reference())
    assert np.array_equal(big[:, :n].cpu().numpy(), w.k_pool[:, 0])


# ---------------------------------------------------------------------------------------------- refusals, streams, capture
@pytest.mark.parametrize("shape", [1, 2])
def test_other_lengths_than_the_plans_are_refused_per_request(shape):
    w = Wave([50, 20, 30], [1, 100, 2], 8, 2, 128, 32, seed=17)
    good = w.reference()
    g = w.device()
    plan = w.plan(wpp.PlanOpts(0, 0, 2, 0, 0, shape))
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
                assert np.all(np.abs(o[rows] - good[0][rows]) <= 2.0 ** -8 * (np.abs(good[0][rows]) + 2.125 * good[2][rows]))
        w.append(h, plan)
        k, _ = okv4.append(w.k_new, w.v_new, w.k_pool, w.v_pool, w.table, w.P, w.C, w.B)
        for j in range(3):
            pages = w.table[j][w.table[j] >= 0]
            assert np.array_equal(h["k"].cpu().numpy()[pages], (w.k_pool if j == i else k)[pages])


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
    want_k, want_v = okv4.append(w.k_new, w.v_new, w.k_pool, w.v_pool, w.table, w.P, w.C, w.B)
    for _ in range(3):
        outs[0].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(g["k"].cpu().numpy(), want_k) and np.array_equal(g["v"].cpu().numpy(), want_v)
    w.k_pool, w.v_pool = want_k, want_v
    w.check(outs[0], None, w.reference())
    assert int(g["status"].item()) == 0


# --------------------------------------------------------------------------------------------------- value rows of unequal sizes
def _along(w, rng, scores, values):
    """Keys whose score with every query is about scores[j] (natural logarithms) and value rows values[j], of request 0 and head 0."""
    n, d = values.shape
    base = rng.standard_normal(d)
    w.q = okv4.bf16_bits(np.broadcast_to(base, w.q.shape).astype(np.float32) + 0.02 * rng.standard_normal(w.q.shape).astype(np.float32))
    keys = scores[:, None] * base / (d ** -0.5 * (base @ base)) + 0.05 * rng.standard_normal((n, d))
    for pool, x in ((w.k_pool, keys), (w.v_pool, values)):
        codes, pairs = okv4.pack_rows(okv4.bf16_bits(x.astype(np.float32)))
        for j in range(n):
            okv4.write_row(pool, w.table[0, j // w.B], 0, j % w.B, w.B, codes[j], pairs[j])


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
    elif kind == "tiny":                                               # (scales just above 2^-100, below which a row has none)
        values *= 2.0 ** -90
    elif kind == "any size":
        values *= 2.0 ** rng.uniform(-30, 30, (n, 1))
    elif kind == "wider as the scores fall":
        scores = np.linspace(30, -30, n)
        values *= np.exp(-scores[:, None])
    elif kind == "narrower as the scores rise":
        scores = np.linspace(-30, 30, n)
        values *= np.exp(-scores[:, None])
    elif kind == "rows of one value behind others":
        scores[n // 2:] += np.linspace(0, 70, n - n // 2)
        values[n // 2:] = np.round(values[n // 2:, :1], 1)
        values[n // 2::3] = 0.0
    return scores, values


@pytest.mark.parametrize("kind", [f"one wide row that nobody attends to, 2 ** {e}" for e in (6, 20, 40)] +
                         [f"a dominant key, a flat tail and one wide row, {a} {b}" for a, b in ((18, 256), (16, 1000), (14, 4000))] +
                         ["tiny", "any size", "wider as the scores fall", "narrower as the scores rise", "rows of one value behind others"])
@pytest.mark.parametrize("d,Hq,C,n", [(128, 4, 1, 12000), (64, 5, 3, 3000), (128, 3, 40, 1100)])
def test_value_rows_of_unequal_sizes(kind, d, Hq, C, n):
    """What a row of V weighs decides what it does, not how wide it is."""
    w = Wave([n - C], [C], Hq, 1, d, 64, seed=n + d)
    rng = np.random.default_rng(n)
    _along(w, rng, *_values(kind, n, d, rng))
    g, ref = w.device(), w.reference()
    for shape, splits in ((2, 1), (2, 3), (1, 1), (1, 2)):
        out, lse = w.attend(g, opts=wpp.PlanOpts(0, 0, splits, 0, 0, shape))
        assert int(g["status"].item()) == 0
        w.check(out, lse, ref)
