"""Linear attention with a decay per head on the GPU against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2609_35263_b200 as wpp
from tests.linear_harness import Wave, ctx

pytestmark = pytest.mark.gpu
LAYOUTS = (0, 1, 2)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("chunks,H", [([1], 1), ([1] * 5, 3), ([0, 1, 0], 2), ([2, 15, 16, 17], 2), ([63, 64, 65], 2), ([128, 0, 129, 1], 3), ([300, 40], 2),
                                      ([1000], 1)])
@pytest.mark.parametrize("per_token", [False, True])
def test_chunks(layout, d, chunks, H, per_token):
    w = Wave(chunks, H, d, seed=sum(chunks) + d, per_token=per_token)
    g = w.device()
    out = w.run(g, layout)
    assert int(g["status"].item()) == 0
    w.check(out, g["pool"], w.reference())


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("chunks,prefix,interval", [([200, 70], [0, 33], 64), ([130], [5], 1), ([257, 1, 64], [100, 63, 64], 50), ([40], [7], 1000),
                                                    ([600], [64], 128), ([300], [128], 100)])
@pytest.mark.parametrize("d", [64, 128])
def test_snapshots(layout, chunks, prefix, interval, d):
    w = Wave(chunks, 2, d, seed=3, prefix=prefix, interval=interval, scale=0.25)
    g = w.device()
    out = w.run(g, layout)
    w.check(out, g["pool"], w.reference())


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("d", [64, 128])
def test_the_zero_state_and_slots_that_are_not_stored(layout, d):
    w = Wave([100, 3], 2, d, seed=4, resume=False)
    w.state_out[1] = -1
    g = w.device()
    out = w.run(g, layout)
    w.check(out, g["pool"], w.reference())
    assert torch.equal(g["pool"][:2].cpu(), w.pool[:2]) and torch.equal(g["pool"][3].cpu(), w.pool[3])


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("d", [64, 128])
def test_a_state_in_place(layout, d):
    w = Wave([150, 1], 3, d, seed=5)
    w.state_out = w.state_in.copy()
    g = w.device()
    out = w.run(g, layout)
    w.check(out, g["pool"], w.reference())


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("d", [64, 128])
def test_decays_from_none_to_all(layout, d):
    """No decay at all, decays that leave nothing after a few tokens, and ones that forget at once."""
    rng = np.random.default_rng(6)
    decay = -np.exp(rng.uniform(-12, 4, (400, 4)))
    decay[:, 0] = 0.0
    decay[:, 1] = -30.0
    decay[rng.random((400, 4)) < 0.05] = -np.inf
    decay[rng.random((400, 4)) < 0.02] = -3e38
    decay[100:300, 2] = 0.0
    w = Wave([270, 130], 4, d, seed=7, decay=decay)
    g = w.device()
    out = w.run(g, layout)
    w.check(out, g["pool"], w.reference())


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("d", [64, 128])
def test_views_of_packed_buffers(layout, d):
    w = Wave([170, 9], 3, d, seed=8)
    g = w.device()
    packed = torch.randn(w.T, 3 * 3 * d + 64, device="cuda").bfloat16()
    views = [packed[:, i * 3 * d:(i + 1) * 3 * d].unflatten(1, (3, d)) for i in range(3)]
    for x, n in zip(views, "qkv"):
        x.copy_(g[n])
        g[n] = x
    gates = torch.full((w.T, 8), 7.0, device="cuda")
    gates[:, 2:5] = g["decay"]
    g["decay"] = gates[:, 2:5]
    wide = torch.full((w.T, 4, d), 3.0, dtype=torch.bfloat16, device="cuda")
    out = w.run(g, layout, out=wide[:, :3])
    w.check(out, g["pool"], w.reference())
    assert bool((wide[:, 3] == 3.0).all())


@pytest.mark.parametrize("layout", LAYOUTS)
def test_cut_chunks_end_where_whole_ones_do(layout):
    """A prompt in three waves, each resumed from the one before, and in one."""
    w = Wave([500], 2, 128, seed=9)
    g = w.device()
    ref = w.reference()
    pool, at = g["pool"].clone(), 0
    outs = []
    for n in (130, 1, 369):
        part = dict(g, pool=pool, rows=torch.tensor([0, n], device="cuda"), state_in=torch.tensor([1 if at else 0], dtype=torch.int32, device="cuda"))
        for x in ("q", "k", "v", "decay"):
            part[x] = g[x][at:at + n]
        outs.append(w.run(part, layout, out=torch.empty_like(part["q"])))
        at += n
    w.check(torch.cat(outs), pool, ref)


@pytest.mark.parametrize("layout", (0, 2))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("chunks,H,interval", [([3100], 1, 0), ([2000, 900, 0, 2300], 2, 0), ([2900, 1], 1, 700), ([1537, 2048], 3, 512)])
def test_chains_in_segments(layout, d, chunks, H, interval):
    """Few long chains: several segments of each, whose states before come from the segments before; the same slot in and out; a
    first token that forgets in some segment; no workspace, which leaves whole chains."""
    w = Wave(chunks, H, d, seed=sum(chunks), interval=interval, prefix=[5] * len(chunks))
    w.state_out = w.state_in.copy()
    w.decay[1200] = -np.inf
    ref = w.reference()
    assert wpp.wpp_linear_workspace_bytes(len(chunks), H, d, w.T) > 256
    for kw in ({}, dict(workspace=None), dict(workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))):
        g = w.device()
        out = w.run(g, layout, **kw)
        assert int(g["status"].item()) == 0
        w.check(out, g["pool"], ref)


@pytest.mark.parametrize("d", [64, 128])
def test_rows_of_others_never_count(d):
    """A request of NaN between two others: blocks that end inside its rows read them, and nothing of them."""
    w = Wave([100, 60, 150], 2, d, seed=15)
    ref = w.reference()
    for name in "qkv":
        getattr(w, name)[100:160] = float("nan")
    w.decay[100:160] = float("nan")
    for layout in LAYOUTS:
        g = w.device()
        out = w.run(g, layout)
        o, size, pool = ref
        keep = np.r_[0:100, 160:310]
        assert np.all(np.abs(out.double().cpu().numpy()[keep] - o[keep]) <= 2.0 ** -8 * (np.abs(o[keep]) + size[keep]))
        got = g["pool"].double().cpu().numpy()
        for slot in (3, 5):
            assert np.all(np.abs(got[slot] - pool[slot]) <= 2.0 ** -15 * np.abs(pool[slot]).max())


def test_a_misaligned_workspace_is_refused():
    w = Wave([3000], 1, 128, seed=16)
    g = w.device()
    with pytest.raises(wpp.WppError) as e:
        w.run(g, workspace=torch.empty(w.workspace().numel() + 256, dtype=torch.uint8, device="cuda")[16:])
    assert e.value.status == 1


@pytest.mark.parametrize("d", [64, 128])
def test_bad_slots_are_reported(d):
    for layout in LAYOUTS:
        w = Wave([80, 5], 2, d, seed=10, interval=64)
        ref = w.reference()
        for name in ("state_in", "state_out", "snaps"):
            for bad in (-2, int(w.pool.shape[0]), 2 ** 31 - 1):
                g = w.device()
                g[name].view(-1)[0] = bad
                pool = g["pool"].clone()
                out = w.run(g, layout)
                assert int(g["status"].item()) == 3
                # the other request is not touched
                assert np.allclose(out[80:].double().cpu().numpy(), ref[0][80:], atol=2.0 ** -8 * float(ref[1].max()))
                assert torch.equal(g["pool"][:2], pool[:2])


def test_refusals_before_a_launch():
    w = Wave([20], 2, 64, seed=11, interval=16)
    g, n = w.device(), ctx().launch_count()
    for change in (dict(prefix=None), dict(pool=g["pool"].view(-1)[1:-127].view(-1, 2, 64, 1)), dict(q=None)):
        with pytest.raises((wpp.WppError, AttributeError, TypeError)):
            w.run(dict(g, **change))
    with pytest.raises(wpp.WppError):
        w.run(g, layout=3)
    with pytest.raises(wpp.WppError):
        w.run(g, out=torch.empty(20 * 128 + 8, dtype=torch.bfloat16, device="cuda")[4:-4].view(20, 2, 64))
    assert ctx().launch_count() == n


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("chunks", [[1, 1, 1], [200, 64]])
def test_captured_and_replayed_and_on_two_streams(layout, chunks):
    w = Wave(chunks, 3, 128, seed=12)
    g = w.device()
    ref = w.reference()
    pools = [g["pool"].clone() for _ in range(2)]
    spaces = [w.workspace() for _ in range(2)]
    outs = [torch.empty_like(g["q"]) for _ in range(2)]
    torch.cuda.synchronize()
    for s, x, ws, o in zip([torch.cuda.Stream() for _ in range(2)], pools, spaces, outs):
        w.run(dict(g, pool=x), layout, out=o, workspace=ws, stream=s)
    torch.cuda.synchronize()
    w.check(outs[0], pools[0], ref)
    assert torch.equal(outs[0], outs[1]) and torch.equal(*pools)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        w.run(g, layout, out=outs[0], workspace=spaces[0])
    for _ in range(3):
        outs[0].zero_()
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(g["pool"], pools[1])
    assert int(g["status"].item()) == 0


def test_beside_the_attention_of_the_same_wave():
    """A hybrid stage's two layers of one wave: append and attention over a cache held in 4 bits, and the linear layer."""
    from tests.kv4_harness import Wave as CacheWave
    from oracle import kv4 as okv4
    a = CacheWave([40, 100], [90, 1], 8, 2, 64, 32, seed=13)
    w = Wave([90, 1], 4, 64, seed=14, prefix=[40, 100])
    ga, g = a.device(), w.device()
    plan = a.plan()
    a.append(ga, plan)
    out, lse = a.attend(ga, plan)
    o = w.run(g)
    a.k_pool, a.v_pool = okv4.append(a.k_new, a.v_new, a.k_pool, a.v_pool, a.table, a.P, a.C, a.B)
    a.check(out, lse, a.reference())
    w.check(o, g["pool"], w.reference())


# single tokens and empty chunks among long ones: more chains than the SMs hold, both forms in one call, long chains in segments
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("interval", [0, 96])
@pytest.mark.parametrize("in_place", [False, True])
def test_single_tokens_among_long_chunks(d, interval, in_place):
    C = [1, 0, 11, 12, 13, 1500, 1, 1, 64, 65, 128, 129, 700, 2] + [1] * 30 + [513]
    assert len(C) * 8 > 2 * 148
    w = Wave(C, 8, d, seed=d + interval, interval=interval, prefix=[5 * i for i in range(len(C))])
    if in_place:
        w.state_out = w.state_in.copy()
    ref = w.reference()
    assert wpp.wpp_linear_workspace_bytes(len(C), 8, d, w.T) > 256
    for workspace in (True, False):
        g = w.device()
        out = w.run(g) if workspace else w.run(g, workspace=None)
        w.check(out, g["pool"], ref)
        assert int(g["status"].item()) == 0
    g, first = w.device(), w.device()
    ws, a, b = w.workspace(), None, None
    a = w.run(first, workspace=ws)
    torch.cuda.synchronize()
    b = w.run(g, workspace=ws)                         # a workspace that a call before has used
    assert torch.equal(a, b) and torch.equal(g["pool"], first["pool"])


def test_single_tokens_among_long_chunks_captured():
    C = [1] * 40 + [900]
    w = Wave(C, 8, 128, seed=3)
    ref, ws, out = w.reference(), w.workspace(), torch.zeros(w.T, 8, 128, dtype=torch.bfloat16, device="cuda")
    g = w.device()
    w.run(g, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        w.run(g, out=out, workspace=ws)
    for _ in range(3):
        out.zero_()
        graph.replay()
    torch.cuda.synchronize()
    w.check(out, g["pool"], ref)


# ------------------------------------------------------------------------------------- decays and values that are no numbers, growth
def _same(out, pool, ref, rows, head, columns=slice(None), slot=None):
    """These outputs and, of this slot, these columns of the state are what they are without the spoilt input (tolerances as in
    Wave.check)."""
    o, size, want = ref
    got = out.double().cpu().numpy()[rows, head][..., columns]
    o, size = o[rows, head][..., columns], size[rows, head][..., columns]
    assert np.all(np.abs(got - o) <= 2.0 ** -8 * (np.abs(o) + size) + 1e-30)
    if slot is not None:
        diff = np.abs(pool[slot, head].double().cpu().numpy() - want[slot, head])[..., columns]
        assert np.all(diff <= 2.0 ** -15 * np.abs(want[slot, head]).max())


SPOILT = [([40], 17), ([30, 200, 70], 30 + 131), ([90, 350], 90 + 2), ([2900], 1501)]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("chunks,at", SPOILT)
def test_a_nan_decay_counts_from_its_own_token_on(layout, d, chunks, at):
    """The state forgets nothing and is no number from there on, in the request and head that the decay belongs to."""
    w = Wave(chunks, 2, d, seed=at + d, interval=64)
    ref = w.reference()
    w.decay[at, 1] = float("nan")
    g = w.device()
    out = w.run(g, layout)
    assert int(g["status"].item()) == 0
    starts = np.concatenate([[0], np.cumsum(w.C)])
    for i, (a, b) in enumerate(zip(starts, starts[1:])):
        slot = int(w.state_out[i])
        _same(out, g["pool"], ref, slice(a, b), 0, slot=slot)
        if not a <= at < b:
            _same(out, g["pool"], ref, slice(a, b), 1, slot=slot)
            continue
        _same(out, g["pool"], ref, slice(a, at), 1)
        assert bool(torch.isnan(out[at:b, 1]).all()) and bool(torch.isnan(g["pool"][slot, 1]).all())
        for n, snap in enumerate(int(x) for x in w.snaps[i] if x >= 0):
            if 64 * (n + 1) > at - a:
                assert bool(torch.isnan(g["pool"][snap, 1]).all())
            else:
                _same(out, g["pool"], ref, slice(a, a), 1, slot=snap)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("d", [64, 128])
def test_a_nan_decay_of_a_head(layout, d):
    w = Wave([150, 3], 3, d, seed=d, per_token=False)
    ref = w.reference()
    w.decay[1] = float("nan")
    g = w.device()
    out = w.run(g, layout)
    for head in (0, 2):
        _same(out, g["pool"], ref, slice(0, 153), head, slot=2)
        _same(out, g["pool"], ref, slice(0, 153), head, slot=3)
    assert bool(torch.isnan(out[:, 1]).all()) and bool(torch.isnan(g["pool"][2:, 1]).all())


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("chunks,per_token", [([70, 9], False), ([300, 1], True), ([2000], True)])
def test_decays_above_zero_and_of_both_signs(layout, d, chunks, per_token):
    rng = np.random.default_rng(chunks[0] + d)
    decay = rng.uniform(-0.4, 0.3, (sum(chunks), 2)) if per_token else np.array([0.04, -0.02])
    w = Wave(chunks, 2, d, seed=5, per_token=per_token, decay=decay)
    g = w.device()
    out = w.run(g, layout)
    assert int(g["status"].item()) == 0
    w.check(out, g["pool"], w.reference())


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("chunks,at", SPOILT)
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_a_value_that_is_no_number_counts_from_its_own_token_on(layout, d, chunks, at, value):
    """o_i depends on v_j for j <= i alone, and column by column: the tokens before it in the same block and the other columns
    are what they are without it."""
    w = Wave(chunks, 2, d, seed=at + d + 1)
    ref = w.reference()
    w.v[at, 1, 5] = value
    w.v[at, 1, d - 1] = -value
    w.v[at + 1, 1, 5] = float("nan")
    w.v[at + 4, 1, 40] = value
    first = {5: at, d - 1: at, 40: at + 4}
    others = np.array([c for c in range(d) if c not in first])
    g = w.device()
    out = w.run(g, layout)
    assert int(g["status"].item()) == 0
    starts = np.concatenate([[0], np.cumsum(w.C)])
    for i, (a, b) in enumerate(zip(starts, starts[1:])):
        slot = int(w.state_out[i])
        _same(out, g["pool"], ref, slice(a, b), 0, slot=slot)
        _same(out, g["pool"], ref, slice(a, b), 1, others, slot)
        if not a <= at < b:
            _same(out, g["pool"], ref, slice(a, b), 1, slot=slot)
            continue
        for c, j in first.items():
            _same(out, g["pool"], ref, slice(a, j), 1, np.array([c]))
            assert not bool(torch.isfinite(out[j:b, 1, c]).any()) and not bool(torch.isfinite(g["pool"][slot, 1, :, c]).any())


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("d", [64, 128])
def test_a_key_and_a_query_that_are_no_numbers_count_from_their_own_tokens_on(layout, d):
    w = Wave([200, 30], 2, d, seed=d + 2)
    ref = w.reference()
    w.q[20, 0, 3] = float("nan")
    w.k[140, 1, 7] = float("inf")
    g = w.device()
    out = w.run(g, layout)
    _same(out, g["pool"], ref, np.r_[0:20, 21:230], 0, slot=2)
    _same(out, g["pool"], ref, np.r_[0:140, 200:230], 1, slot=3)
    assert bool(torch.isnan(out[20, 0]).all()) and not bool(torch.isfinite(out[140:200, 1]).any())
    rows = np.array([c for c in range(d) if c != 7])
    diff = np.abs(g["pool"][2, 1].double().cpu().numpy() - ref[2][2, 1])[rows]
    assert np.all(diff <= 2.0 ** -15 * np.abs(ref[2][2, 1]).max()) and not bool(torch.isfinite(g["pool"][2, 1, 7]).any())
