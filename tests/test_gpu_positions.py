"""Pages from lengths, rotary positions and both on the way into a cache, on the GPU."""
import numpy as np
import pytest
import torch

import paper_2609_35263_b200 as wpp
from oracle import positions as opos
from tests.kv4_harness import ctx

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


# ----------------------------------------------------------------------------------------------------------------- pages
class Pages:
    def __init__(self, P, C, B, seed=0, most=None, spare=5, taken=0, pages=None):
        rng = np.random.default_rng(seed)
        self.P, self.C, self.B, self.taken = np.asarray(P, np.int32), np.asarray(C, np.int32), B, taken
        there = -(-np.maximum(self.P, 0).astype(np.int64) // B)
        blocks = -(-(np.maximum(self.P, 0).astype(np.int64) + np.maximum(self.C, 0)) // B)
        self.most = int(blocks.max(initial=0)) + 2 if most is None else most
        self.num_pages = int(blocks.sum()) + spare + taken if pages is None else pages
        perm = rng.permutation(int(blocks.sum()) + spare + taken).astype(np.int32)
        self.table = np.full((len(self.P), self.most), -7, np.int32)
        at = 0
        for i, n in enumerate(np.minimum(there, self.most)):
            self.table[i, :n] = perm[at:at + n]
            at += n
        self.free = perm[at:]
        self.total = int(np.maximum(self.C, 0).sum())

    def desc(self):
        return wpp.make_desc(len(self.P), 4, 2, 64, self.B, self.most, self.num_pages)

    def run(self, capacity=None, separate=False, **kw):
        n = self.total + 9 if capacity is None else capacity
        g = dict(table=_i32(self.table), cursor=_i32([self.taken, 0]), rows=torch.full((len(self.P) + 1,), -5, dtype=torch.int64, device="cuda"),
                 positions=torch.full((n,), -5, dtype=torch.int32, device="cuda"), slots=torch.full((n,), -5, dtype=torch.int64, device="cuda"),
                 status=torch.zeros(1, dtype=torch.int32, device="cuda"))
        out = _i32([-5, 0]) if separate else None
        g.update(P=_i32(self.P), C=_i32(self.C), free=_i32(self.free))
        wpp.wpp_assign_pages(ctx(), self.desc(), g["P"], g["C"], g["free"], g["cursor"], g["table"], g["rows"], g["positions"], g["slots"],
                             cursor_out=out, status=g["status"], **kw)
        if separate:
            assert g["cursor"].tolist() == [self.taken, 0]
            g["cursor"] = out
        return g

    def check(self, g):
        n = g["slots"].numel()
        table, rows, positions, slots, taken, error = opos.assign(self.P, self.C, self.free, self.taken, self.table, self.B, self.num_pages, n)
        assert np.array_equal(g["table"].cpu().numpy(), table)
        for name, want in (("rows", rows), ("positions", positions), ("slots", slots)):
            assert np.array_equal(g[name].cpu().numpy(), want), name
        assert g["cursor"].tolist() == [taken, 0]
        assert bool(g["status"].item()) == bool(error) and (not error or int(g["status"].item()) in (1, 3))


@pytest.mark.parametrize("B", [16, 32, 64, 128])
@pytest.mark.parametrize("P,C", [([], []), ([0], [0]), ([0], [1]), ([15, 16, 17, 127, 128], [1, 1, 1, 1, 1]), ([0, 5, 0, 64, 0, 200], [0, 40, 1, 0, 129, 0]),
                                 ([3], [5000])])
@pytest.mark.parametrize("separate", [False, True])
def test_pages(B, P, C, separate):
    w = Pages(P, C, B, seed=B, taken=3)
    w.check(w.run(separate=separate))


@pytest.mark.parametrize("R,most", [(511, 3), (512, 40), (513, 300), (2000, 20), (16384, 4)])
def test_pages_of_many_requests(R, most):
    rng = np.random.default_rng(R)
    w = Pages(rng.integers(0, 300, R), np.where(rng.random(R) < 0.3, 0, rng.integers(0, most + 1, R)), 16, seed=R)
    w.check(w.run())


def test_pages_of_far_positions():
    P, C, B = np.array([1 << 30, 5], np.int32), np.array([40, 3], np.int32), 128
    most = (1 << 23) + 1
    table = torch.full((2, most), 1, dtype=torch.int32, device="cuda")
    rows, status = torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    positions, slots = torch.zeros(43, dtype=torch.int32, device="cuda"), torch.zeros(43, dtype=torch.int64, device="cuda")
    cursor = _i32([0, 0])
    big = 2 ** 30 - 1                                                  # a page id whose slots lie behind 2^32
    wpp.wpp_assign_pages(ctx(), wpp.make_desc(2, 4, 2, 64, B, most, 2 ** 30), _i32(P), _i32(C), _i32([big, 9]), cursor, table, rows, positions, slots,
                         status=status)
    assert positions.tolist() == [(1 << 30) + j for j in range(40)] + [5, 6, 7]
    assert slots.tolist() == [big * B + j for j in range(40)] + [B + 5, B + 6, B + 7]
    assert cursor.tolist() == [1, 0] and int(table[0, 1 << 23]) == big and int(status.item()) == 0 and rows.tolist() == [0, 40, 43]


@pytest.mark.parametrize("case", ["list runs out", "list is empty", "bad page in the list", "bad page in a table", "short table", "negative lengths",
                                  "too many tokens", "cursor behind the list", "cursor below zero", "no room for tokens"])
def test_pages_that_cannot_be_given(case):
    w = Pages([20, 0, 40, 7], [30, 100, 1, 60], 16, seed=4)
    capacity = None
    if case == "list runs out":
        w.free = w.free[:6]
    elif case == "list is empty":
        w.free = w.free[:0]
    elif case == "bad page in the list":
        w.free[[2, 5]] = [-3, w.num_pages]
    elif case == "bad page in a table":
        w.table[0, 1] = w.num_pages
    elif case == "short table":
        w.table, w.most = np.ascontiguousarray(w.table[:, :3]), 3
    elif case == "negative lengths":
        w.P[2], w.C[3] = -1, -60
    elif case == "too many tokens":
        capacity = 77
    elif case == "cursor behind the list":
        w.taken = len(w.free) + 9
    elif case == "cursor below zero":
        w.taken = -2
    elif case == "no room for tokens":
        capacity = 0
    g = w.run(capacity)
    w.check(g)
    assert int(g["status"].item()) == (1 if case == "negative lengths" else 3)


def test_pages_replayed_take_others():
    """One captured call on a cursor of its own, replayed as lengths grow: a step of every request, token by token."""
    R, B = 5, 16
    rng = np.random.default_rng(6)
    P, table = rng.integers(0, 40, R).astype(np.int32), np.full((R, 9), -1, np.int32)
    there = -(-P // B)
    perm = rng.permutation(80).astype(np.int32)
    at = np.concatenate([[0], np.cumsum(there)])
    for i in range(R):
        table[i, :there[i]] = perm[at[i]:at[i + 1]]
    free = perm[at[-1]:]
    g = [_i32(P), _i32(np.ones(R)), _i32(free), _i32([0, 0]), _i32(table)]
    rows, positions = torch.zeros(R + 1, dtype=torch.int64, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    slots, status = torch.zeros(8, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    desc = wpp.make_desc(R, 4, 2, 64, B, 9, 80)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        wpp.wpp_assign_pages(ctx(), desc, *g, rows, positions, slots, status=status)
        g[0].add_(1)
    taken = 0
    for _ in range(60):
        graph.replay()
        table, r, pos, s, taken, error = opos.assign(P, np.ones(R, np.int32), free, taken, table, B, 80, 8)
        P = P + 1
        assert not error and np.array_equal(slots.cpu().numpy(), s) and np.array_equal(positions.cpu().numpy(), pos)
    assert np.array_equal(g[4].cpu().numpy(), table) and g[3].tolist() == [taken, 0] and int(status.item()) == 0


# ------------------------------------------------------------------------------------------------------------- positions
def _normal(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


def _near(got, x, turns, positions, interleaved, magnitude):
    """Rounded once (2^-8); sine and cosine within 2^-20, their products' rounding: 2^-19 of the pair's absolute sum."""
    want, size = opos.rotate(x.double().cpu().numpy(), turns.tolist(), positions.tolist(), interleaved, magnitude)
    d = np.abs(got.double().cpu().numpy() - want)
    assert np.all(d <= 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * magnitude * size)
    n = 2 * turns.numel()
    assert torch.equal(got[..., n:], x[..., n:])


FAR = [0, 1, 2, 77, 4095, 131071, 10 ** 6 + 7, 2 ** 31 - 1]


@pytest.mark.parametrize("T", [1, 5, 333])
@pytest.mark.parametrize("Hq,Hkv,d,n", [(8, 2, 64, 64), (5, 1, 128, 128), (40, 8, 128, 64), (3, 3, 64, 16), (64, 8, 128, 96), (1, 1, 128, 32)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope(T, Hq, Hkv, d, n, interleaved):
    q, k = _normal(T, T, Hq, d), _normal(T + 1, T, Hkv, d)
    turns, magnitude = wpp.wpp_rope_frequencies(n, base=500000.0, scaling="turns", factor=4.0, original_context=8192)
    pos = _i32(np.random.default_rng(T).permutation(np.resize(FAR, T)))
    q_out, k_out = torch.full_like(q, 9.0), torch.full_like(k, 9.0)
    before = q.clone(), k.clone()
    wpp.wpp_rope(ctx(), q, k, turns.cuda(), pos, q_out=q_out, k_out=k_out, interleaved=interleaved, magnitude=magnitude)
    _near(q_out, q, turns, pos, interleaved, magnitude)
    _near(k_out, k, turns, pos, interleaved, magnitude)
    assert torch.equal(q, before[0]) and torch.equal(k, before[1])
    wpp.wpp_rope(ctx(), q, k, turns.cuda(), pos, interleaved=interleaved, magnitude=magnitude)
    assert torch.equal(q, q_out) and torch.equal(k, k_out)


def test_rope_of_queries_or_keys_alone_and_of_nothing():
    q, pos = _normal(1, 7, 4, 128), _i32(range(7))
    turns = wpp.wpp_rope_frequencies(128)[0].cuda()
    a, b = torch.empty_like(q), torch.empty_like(q)
    wpp.wpp_rope(ctx(), q, None, turns, pos, q_out=a)
    wpp.wpp_rope(ctx(), None, q, turns, pos, k_out=b)
    assert torch.equal(a, b)
    _near(a, q, turns, pos, False, 1.0)
    n = ctx().launch_count()
    wpp.wpp_rope(ctx(), q[:0], None, turns, pos[:0])
    assert ctx().launch_count() == n


def test_rope_of_positions_below_zero_turns_back():
    q, pos = _normal(2, 9, 2, 64), _i32(range(9))
    turns = wpp.wpp_rope_frequencies(64)[0].cuda()
    a, b = torch.empty_like(q), torch.empty_like(q)
    wpp.wpp_rope(ctx(), q, None, turns, -pos, q_out=a)
    _near(a, q, turns, -pos, False, 1.0)


def test_rope_of_values_that_are_no_numbers_stays_in_its_pairs():
    q, pos = _normal(3, 4, 2, 64), _i32([3, 4, 5, 6])
    turns = wpp.wpp_rope_frequencies(32)[0].cuda()
    q[1, 0, 5], q[2, 1, 50], q[3, 0, 20] = float("nan"), float("inf"), float("inf")
    out = torch.empty_like(q)
    wpp.wpp_rope(ctx(), q, None, turns, pos, q_out=out)
    bad = ~torch.isfinite(out)
    want = torch.zeros_like(bad)
    want[1, 0, [5, 21]] = want[3, 0, [4, 20]] = True
    want[2, 1, 50] = True
    assert torch.equal(bad, want)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_inside_a_packed_buffer(interleaved):
    """Query, key and value heads side by side, with room between them, in place: what is not a turned head stays."""
    T, d = 50, 64
    buf = _normal(4, T, 20, 72)
    before = buf.clone()
    q, k = buf[:, :8, :d], buf[:, 10:12, :d]
    turns, pos = wpp.wpp_rope_frequencies(32)[0], _i32(np.arange(T) * 37)
    wpp.wpp_rope(ctx(), q, k, turns.cuda(), pos, interleaved=interleaved)
    _near(q, before[:, :8, :d], turns, pos, interleaved, 1.0)
    _near(k, before[:, 10:12, :d], turns, pos, interleaved, 1.0)
    for lo, hi in ((8, 10), (12, 20)):
        assert torch.equal(buf[:, lo:hi], before[:, lo:hi])
    assert torch.equal(buf[..., d:], before[..., d:])


def test_rope_on_another_stream_and_replayed():
    q, k, pos = _normal(5, 30, 8, 128), _normal(6, 30, 2, 128), _i32(np.arange(30) + 1000)
    turns = wpp.wpp_rope_frequencies(128)[0].cuda()
    want = [torch.empty_like(q), torch.empty_like(k)]
    wpp.wpp_rope(ctx(), q, k, turns, pos, q_out=want[0], k_out=want[1])
    torch.cuda.synchronize()
    s, out = torch.cuda.Stream(), [torch.zeros_like(q), torch.zeros_like(k)]
    wpp.wpp_rope(ctx(), q, k, turns, pos, q_out=out[0], k_out=out[1], stream=s)
    s.synchronize()
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wpp.wpp_rope(ctx(), q, k, turns, pos, q_out=out[0], k_out=out[1])
    pos.sub_(900)
    graph.replay()
    _near(out[0], q, turns, pos, False, 1.0)


# ------------------------------------------------------------------------------------------------- straight into the cache
@pytest.mark.parametrize("T", [1, 70, 1000])
@pytest.mark.parametrize("Hq,Hkv,d,B,n", [(8, 2, 64, 16, 64), (40, 8, 128, 32, 64), (5, 5, 128, 128, 128)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_append_is_rope_and_a_copy_into_slots(T, Hq, Hkv, d, B, n, interleaved):
    rng = np.random.default_rng(T)
    pages = T // B + 9
    packed = _normal(T + 2, T, Hq + 2 * Hkv, d)
    q, k, v = packed.split([Hq, Hkv, Hkv], 1)
    turns, pos = wpp.wpp_rope_frequencies(n)[0].cuda(), _i32(rng.integers(0, 100000, T))
    slots = rng.permutation(pages * B)[:T]
    slots[rng.random(T) < 0.2] = -1
    slots_dev, status = torch.from_numpy(slots).cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    desc = wpp.make_desc(1, Hq, Hkv, d, B, pages, pages)
    pools = [_normal(i, pages, Hkv, B, d) for i in (1, 2)]
    want = [p.clone() for p in pools]
    q_want, k_want = torch.empty(T, Hq, d, dtype=torch.bfloat16, device="cuda"), torch.empty(T, Hkv, d, dtype=torch.bfloat16, device="cuda")
    wpp.wpp_rope(ctx(), q, k, turns, pos, q_out=q_want, k_out=k_want, interleaved=interleaved)
    there = torch.from_numpy(np.flatnonzero(slots >= 0)).cuda()
    at = slots_dev[there]
    want[0][at // B, :, at % B], want[1][at // B, :, at % B] = k_want[there], v[there]
    before = packed.clone()
    out = torch.empty_like(q_want)
    wpp.wpp_rope_append(ctx(), desc, q, k, v, out, *pools, turns, pos, slots_dev, interleaved=interleaved, status=status)
    assert torch.equal(out, q_want) and torch.equal(pools[0], want[0]) and torch.equal(pools[1], want[1]) and torch.equal(packed, before)
    wpp.wpp_rope_append(ctx(), desc, None, k, v, None, *pools, turns, pos, slots_dev, interleaved=interleaved, status=status)
    assert torch.equal(pools[0], want[0]) and torch.equal(pools[1], want[1])
    wpp.wpp_rope_append(ctx(), desc, q, k, v, None, *pools, turns, pos, slots_dev, interleaved=interleaved, status=status)       # queries in place
    assert torch.equal(packed[:, :Hq], q_want) and torch.equal(packed[:, Hq:], before[:, Hq:]) and int(status.item()) == 0


def test_rope_append_reports_slots_that_are_none():
    T, B = 20, 16
    q, k, v = _normal(1, T, 4, 64), _normal(2, T, 2, 64), _normal(3, T, 2, 64)
    turns, pos, out = wpp.wpp_rope_frequencies(64)[0].cuda(), _i32(range(T)), torch.empty_like(q)
    desc = wpp.make_desc(1, 4, 2, 64, B, 8, 8)
    for bad in (8 * B, -2, 2 ** 62, -2 ** 63):
        slots, status = torch.arange(T, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        slots[7] = bad
        pools = [torch.full((8, 2, B, 64), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        wpp.wpp_rope_append(ctx(), desc, q, k, v, out, *pools, turns, pos, slots, status=status)
        assert int(status.item()) == 3
        rows = pools[1].transpose(1, 2).flatten(0, 1)
        assert torch.equal(rows[:7], v[:7]) and torch.equal(rows[8:T], v[8:]) and (rows[7] == 3).all() and (rows[T:] == 3).all()


def test_rope_append_into_a_pool_with_strides_of_its_own_beyond_32_bits():
    T, B, Hkv, d, stride = 40, 16, 1, 64, 1 << 29
    big = torch.empty(9 * stride, dtype=torch.bfloat16, device="cuda")
    q, k, v = _normal(1, T, 4, d), _normal(2, T, Hkv, d), _normal(3, T, Hkv, d)
    turns, pos, status = wpp.wpp_rope_frequencies(64)[0].cuda(), _i32(range(T)), torch.zeros(1, dtype=torch.int32, device="cuda")
    desc = wpp.make_desc(1, 4, Hkv, d, B, 9, 9, kv_page_stride=stride, kv_token_stride=2 * d, kv_head_stride=2 * d * B)
    slots = torch.arange(T, device="cuda") + 6 * B
    wpp.wpp_rope_append(ctx(), desc, q, k, v, torch.empty_like(q), big, big[d:], turns, pos, slots, status=status)
    k_want = torch.empty_like(k)
    wpp.wpp_rope(ctx(), None, k, turns, pos, k_out=k_want)
    for t in range(T):
        at = (6 + t // B) * stride + t % B * 2 * d
        assert torch.equal(big[at:at + d], k_want[t, 0]) and torch.equal(big[at + d:at + 2 * d], v[t, 0])
    assert int(status.item()) == 0


def test_pages_with_a_cursor_apart_that_holds_anything():
    w = Pages([5, 0, 100], [3000, 9, 1], 32, seed=1, taken=2)          # (several CTAs)
    out, n = _i32([77, 78]), w.total
    for _ in range(2):                                                 # the second call takes what the first one did
        table, rows = _i32(w.table), torch.empty(4, dtype=torch.int64, device="cuda")
        positions, slots = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int64, device="cuda")
        cursor, status = _i32([w.taken, 5]), torch.zeros(1, dtype=torch.int32, device="cuda")
        wpp.wpp_assign_pages(ctx(), w.desc(), _i32(w.P), _i32(w.C), _i32(w.free), cursor, table, rows, positions, slots, cursor_out=out, status=status)
        want = opos.assign(w.P, w.C, w.free, w.taken, w.table, w.B, w.num_pages, n)
        assert np.array_equal(table.cpu().numpy(), want[0]) and np.array_equal(slots.cpu().numpy(), want[3])
        assert cursor.tolist() == [w.taken, 5] and out.tolist() == [want[4], 0] and int(status.item()) == 0
    both = _i32([0, 2, 9])                                             # the number is read where the zero would go
    with pytest.raises(wpp.WppError):
        wpp.wpp_assign_pages(ctx(), w.desc(), _i32(w.P), _i32(w.C), _i32(w.free), both[1:], table, rows, positions, slots, cursor_out=both[:2])
    assert both.tolist() == [0, 2, 9]


def test_pages_of_more_than_31_bits_count():
    """17 requests that want 2^27 pages each: nothing is written but the columns of the first 2^31 - 1."""
    R, most = 17, 1 << 27
    table = torch.full((R, most), -7, dtype=torch.int32, device="cuda")
    P, C, free = _i32([0] * R), _i32([2 ** 31 - 1] * R), _i32([4, 3, 9])
    cursor, rows, status = _i32([1, 0]), torch.empty(R + 1, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    wpp.wpp_assign_pages(ctx(), wpp.make_desc(R, 4, 2, 64, 16, most, 20), P, C, free, cursor, table, rows, status=status)
    assert rows.tolist() == [i * (2 ** 31 - 1) for i in range(R + 1)] and cursor.tolist() == [3, 0] and int(status.item()) == 3
    assert table[0, :3].tolist() == [3, 9, -1] and bool((table[1:15] == -1).all()) and table[15, -2:].tolist() == [-1, -7] and bool((table[16] == -7).all())


# ------------------------------------------------------------------------------------------------------- a wave of them all
@pytest.mark.parametrize("cache", [wpp.WPP_BF16, wpp.WPP_KV8, wpp.WPP_KV4])
@pytest.mark.parametrize("C", [[1, 1, 1], [40, 1, 150]])
def test_a_wave_from_lengths_to_attention(cache, C):
    """Pages and slots from the lengths, rotary positions, the append (fused where the cache is bf16) and attention, against 64 bits over the
    rows that the cache holds."""
    from oracle import kv4 as okv4, kv8 as okv8
    P, Hq, Hkv, d, B = [33, 0, 70], 8, 2, 128, 16
    w = Pages(P, C, B, seed=8)
    T = sum(C)
    block = {wpp.WPP_KV8: wpp.wpp_kv8_block_bytes(B, d), wpp.WPP_KV4: wpp.wpp_kv4_block_bytes(B, d)}.get(cache)
    desc = wpp.make_desc(3, Hq, Hkv, d, B, w.most, w.num_pages, dtype=cache)
    pools = [torch.zeros(w.num_pages, Hkv, block, dtype=torch.uint8, device="cuda") if block
             else torch.zeros(w.num_pages, Hkv, B, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    turns = wpp.wpp_rope_frequencies(d)[0].cuda()
    packed = [_normal(i, n, Hq + 2 * Hkv, d) for i, n in ((1, sum(P)), (2, T))]
    keys, values = [], []
    table, cursor = _i32(np.full_like(w.table, -1)), _i32([0, 0])
    free = _i32(np.random.default_rng(9).permutation(w.num_pages))
    ones = np.zeros(3, np.int32)
    for prefix, chunk, rows_in in ((ones, P, packed[0]), (np.array(P), C, packed[1])):         # the prefixes first, in a wave of their own
        n = int(np.sum(chunk))
        plan = wpp.wpp_plan_tiles(ctx(), desc, prefix, chunk).to_device()
        Pd, Cd, rows = _i32(prefix), _i32(chunk), torch.empty(4, dtype=torch.int64, device="cuda")
        positions, slots = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int64, device="cuda")
        wpp.wpp_assign_pages(ctx(), desc, Pd, Cd, free, cursor, table, rows, positions, slots, status=status)
        q, k, v = rows_in.split([Hq, Hkv, Hkv], 1)
        q_out, k_out = torch.empty(n, Hq, d, dtype=torch.bfloat16, device="cuda"), torch.empty(n, Hkv, d, dtype=torch.bfloat16, device="cuda")
        wpp.wpp_rope(ctx(), q, k, turns, positions, q_out=q_out, k_out=k_out)
        if cache == wpp.WPP_BF16:
            wpp.wpp_rope_append(ctx(), desc, q, k, v, q_out, *pools, turns, positions, slots, status=status)
        else:
            wpp.wpp_kv_append(ctx(), desc, k_out, v.contiguous(), *pools, table, Pd, Cd, plan, status=status)
        keys.append(k_out), values.append(v.contiguous())
        out, ws = torch.empty_like(q_out), torch.empty(int(plan.info.workspace_bytes), dtype=torch.uint8, device="cuda")
        wpp.wpp_prefill_attention_varlen(ctx(), desc, q_out, out, None, *pools, table, Pd, Cd, plan, workspace=ws, status=status)
    assert int(status.item()) == 0 and cursor.tolist()[1] == 0
    t = table.cpu().numpy()
    held = [t[i, :-(-(P[i] + C[i]) // B)] for i in range(3)]
    assert len(set(np.concatenate(held).tolist())) == cursor.tolist()[0] == sum(len(h) for h in held)
    at, row, starts = 0, 0, np.concatenate([[0], np.cumsum(P)])
    for i in range(3):
        n = P[i] + C[i]
        stand = []
        for pool, fresh in zip(pools, (keys, values)):
            x = pool.cpu().float().numpy() if not block else pool.cpu().numpy()
            if not block:                                              # what was put in stands there
                got = np.concatenate([x[p] for p in held[i]], 1)[:, :n].transpose(1, 0, 2)
                want = torch.cat([fresh[0][starts[i]:starts[i + 1]], fresh[1][row:row + C[i]]]).float().cpu().numpy()
                assert np.array_equal(got, want)
                stand.append(got.astype(np.float64))
            elif cache == wpp.WPP_KV8:
                stand.append(np.stack([okv8.rows_of(x, t[i], n, B, d, h)[0] for h in range(Hkv)], 1))
            else:
                stand.append(np.array([[okv4.read_row(x, t[i, j // B], h, j % B, B, d) for h in range(Hkv)] for j in range(n)]))
        K, V = stand
        qq = q_out[row:row + C[i]].double().cpu().numpy()
        for j in range(C[i]):
            m = P[i] + j + 1
            s = np.einsum("hgd,khd->hgk", qq[j].reshape(Hkv, -1, d), K[:m]) * d ** -0.5
            e = np.exp(s - s.max(-1, keepdims=True))
            e /= e.sum(-1, keepdims=True)
            o, spread = np.einsum("hgk,khd->hgd", e, V[:m]).reshape(Hq, d), np.einsum("hgk,khd->hgd", e, np.abs(V[:m])).reshape(Hq, d)
            got = out[row + j].double().cpu().numpy()
            # bf16 results and probabilities (the 4-bit cache's rows too, there, after K's scores): a step of 2^-8 each, and an eighth for the scores
            assert np.all(np.abs(got - o) <= 2.0 ** -8 * (np.abs(o) + 2.125 * spread) + 1e-5)
        row += C[i]


@pytest.mark.parametrize("outputs", ["positions", "slots", "neither"])
@pytest.mark.parametrize("case,status", [("nothing wrong", 0), ("short table", 3), ("short table, prefix alone", 3), ("bad page in a table", 3),
                                         ("page below zero in a table", 3), ("list runs out", 3), ("negative length", 1), ("empty chunk behind a bad page", 0)])
def test_pages_without_positions_or_slots_are_refused_alike(case, status, outputs):
    w = Pages([20, 0, 40, 7], [30, 100, 1, 60], 16, seed=4)
    if case == "short table":
        w.table, w.most = np.ascontiguousarray(w.table[:, :6]), 6                          # (request 1 needs 7)
    elif case == "short table, prefix alone":
        w.P[2], w.C[1], w.C[3], w.table, w.most = 90, 1, 1, np.ascontiguousarray(w.table[:, :5]), 5      # (request 2 holds 6)
    elif case in ("bad page in a table", "page below zero in a table"):
        w.table[0, 1] = w.num_pages if case.startswith("bad") else -1
    elif case == "list runs out":
        w.free = w.free[:6]
    elif case == "negative length":
        w.P[2] = -1
    elif case == "empty chunk behind a bad page":
        w.table[0, 1], w.C[0] = w.num_pages, 0
    w.total = int(np.maximum(w.C, 0).sum())
    table, cursor, bad = _i32(w.table), _i32([0, 0]), torch.zeros(1, dtype=torch.int32, device="cuda")
    rows, positions, slots = (torch.full((n,), -5, dtype=t, device="cuda") for n, t in ((5, torch.int64), (w.total, torch.int32), (w.total, torch.int64)))
    wpp.wpp_assign_pages(ctx(), w.desc(), _i32(w.P), _i32(w.C), _i32(w.free), cursor, table, rows, positions if outputs == "positions" else None,
                         slots if outputs == "slots" else None, status=bad)
    want = opos.assign(w.P, w.C, w.free, 0, w.table, w.B, w.num_pages, w.total)
    assert int(bad.item()) == status == want[5] and cursor.tolist() == [want[4], 0]
    assert np.array_equal(table.cpu().numpy(), want[0]) and np.array_equal(rows.cpu().numpy(), want[1])
    if outputs == "positions":
        assert np.array_equal(positions.cpu().numpy(), want[2])
    if outputs == "slots":
        assert np.array_equal(slots.cpu().numpy(), want[3])
