"""The oracle of the 4-bit cache against what its definition implies, and the library's refusals that need no GPU."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2609_35263_b200 as wpp
import paper_2609_35263_b200.binding as B
from oracle import kv4


def _rows(*rows):
    return kv4.bf16_bits(np.array(rows, np.float32))


def test_every_value_is_within_half_a_step():
    rng = np.random.default_rng(1)
    bits = kv4.bf16_bits((rng.standard_normal((500, 128)) * np.exp(rng.standard_normal((500, 1)) * 5)).astype(np.float32))
    codes, pairs = kv4.pack_rows(bits)
    x, least, scale = kv4.bf16_values(bits).astype(float), *np.moveaxis(kv4.bf16_values(pairs).astype(float), -1, 0)
    assert codes.max() == 15 and codes.min() == 0 and np.array_equal(least, x.min(-1))
    assert np.all(np.abs(least[:, None] + scale[:, None] * codes - x) <= scale[:, None] * (0.5 + 1e-6))


def test_quotients_round_as_rational_numbers_do():
    rng = np.random.default_rng(2)
    bits = kv4.bf16_bits(rng.integers(-64, 65, (40, 64)).astype(np.float32) / 8)           # many quotients lie on a half
    codes, pairs = kv4.pack_rows(bits)
    for r in range(40):
        x = [Fraction(float(v)) for v in kv4.bf16_values(bits[r])]
        least, scale = (Fraction(float(v)) for v in kv4.bf16_values(pairs[r]))
        assert [int(c) for c in codes[r]] == [round((v - least) / scale) for v in x]        # (Python rounds halves to even)


def test_rows_that_have_no_scale():
    nan, inf = np.float32("nan"), np.float32("inf")
    bits = _rows([3.0] * 64, [0.0] * 32 + [-0.0] * 32, [-0.0] * 64, [1e-38] + [0.0] * 63)
    codes, pairs = kv4.pack_rows(bits)
    assert not codes.any() and not pairs[:, 1].any() and list(kv4.bf16_values(pairs[:, 0])) == [3.0, 0.0, 0.0, 0.0]
    assert not pairs[1:, 0].any()                                                           # +0, never -0
    x = kv4.bf16_values(np.zeros((3, 64), np.uint16))
    x[0, 5], x[1, 9], x[2, 0], x[2, 1] = nan, -inf, 3.3e38, -3.3e38
    codes, pairs = kv4.pack_rows((np.ascontiguousarray(x).view(np.uint32) >> 16).astype(np.uint16))
    assert not codes.any() and np.array_equal(pairs, [[0x7FC0, 0]] * 3)


def test_append_and_read_back():
    rng = np.random.default_rng(3)
    new = kv4.bf16_bits(rng.standard_normal((5, 2, 64)).astype(np.float32))
    pool = rng.integers(0, 256, (4, 2, wpp.wpp_kv4_block_bytes(16, 64)), dtype=np.uint8)
    k, v = kv4.append(new, new, pool, pool, np.array([[2, 0]], np.int32), [14], [5], 16)
    assert np.array_equal(k, v) and np.array_equal(k[[1, 3]], pool[[1, 3]])
    codes, pairs = kv4.pack_rows(new)
    for t, (page, slot) in enumerate([(2, 14), (2, 15), (0, 0), (0, 1), (0, 2)]):
        for h in range(2):
            least, scale = kv4.bf16_values(pairs[t, h]).astype(float)
            assert np.array_equal(kv4.read_row(k, page, h, slot, 16, 64), least + scale * codes[t, h])
            k[page, h, slot * 32:(slot + 1) * 32] = pool[page, h, slot * 32:(slot + 1) * 32]
            k[page, h, 512 + 4 * slot:516 + 4 * slot] = pool[page, h, 512 + 4 * slot:516 + 4 * slot]
    assert np.array_equal(k, pool)                                                          # no other byte was written


def test_attention_of_one_key_and_of_equal_scores():
    from tests.kv4_harness import Wave
    w = Wave([0, 20], [1, 3], 4, 2, 64, 16, seed=4)
    out, lse, _ = w.reference()
    assert np.allclose(out[0, 0], kv4.read_row(w.v_pool, w.table[0, 0], 0, 0, 16, 64), rtol=1e-14)
    w.q[:] = 0
    out, lse, _ = w.reference()
    assert np.allclose(np.exp(lse), np.array([1, 21, 22, 23])[:, None])


# ------------------------------------------------------------------------------------------------------ the host's refusals
def test_block_bytes():
    for page in (16, 32, 64, 128):
        for d in (64, 128):
            assert wpp.wpp_kv4_block_bytes(page, d) == page * (d // 2 + 4) and wpp.wpp_kv4_block_bytes(page, d) % 16 == 0
    assert wpp.wpp_kv4_block_bytes(48, 128) == wpp.wpp_kv4_block_bytes(64, 96) == wpp.wpp_kv4_block_bytes(0, 0) == 0


@pytest.mark.parametrize("change,status", [
    (dict(kv_token_stride=64), 1), (dict(kv_head_stride=16), 1), (dict(kv_head_stride=64 * 36 + 8), 1), (dict(kv_page_stride=64 * 36 - 16), 1),
    (dict(q_token_stride=100), 1), (dict(dtype=3), 2), (dict(dtype=0), 2)])
def test_descriptions_that_are_refused(change, status):
    kw = dict(dtype=wpp.WPP_KV4)
    kw.update(change)
    with pytest.raises(wpp.WppError) as e:
        wpp.wpp_plan_tiles(None, wpp.make_desc(1, 8, 2, 64, 64, 4, 8, **kw), [10], [3], pin=False)
    assert e.value.status == status


def test_plans_of_the_two_kinds_of_cache_are_not_exchanged():
    lib = B.load_library()
    P, C = [100], [3]
    plan = wpp.wpp_plan_tiles(None, wpp.make_desc(1, 8, 2, 64, 64, 4, 8), P, C, pin=False)
    kv4_desc = wpp.make_desc(1, 8, 2, 64, 64, 4, 8, dtype=wpp.WPP_KV4)
    kv4_plan = wpp.wpp_plan_tiles(None, kv4_desc, P, C, pin=False)
    assert plan.info.shape in (1, 2) and kv4_plan.info.shape == 3
    fake = ctypes.create_string_buffer(1 << 16)               # (a context is only looked at behind the plan)
    for desc, host in ((kv4_desc, plan.host), (wpp.make_desc(1, 8, 2, 64, 64, 4, 8), kv4_plan.host)):
        assert lib.wpp_kv_append(fake, ctypes.byref(desc), *([None] * 7), host.data_ptr(), None, None, None) == 6
        assert lib.wpp_prefill_attention_varlen(fake, ctypes.byref(desc), *([None] * 8), host.data_ptr(), None, None, 0, None, None) == 6


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 64, 8), (64, 8, 8), (128, 40, 8), (128, 32, 1), (64, 20, 1), (128, 6, 2)])
@pytest.mark.parametrize("splits", [0, 1, 3, 64])
@pytest.mark.parametrize("shape", [0, 1, 2])
@pytest.mark.parametrize("P,C", [([0, 700, 5000, 64, 0, 131], [5, 1, 2, 0, 300, 129]), ([3, 9000], [700, 1]), ([20], [2])])
def test_plans_cover_every_visible_pair_once(d, Hq, Hkv, splits, shape, P, C):
    desc = wpp.make_desc(len(P), Hq, Hkv, d, 32, 400, 999, dtype=wpp.WPP_KV4)
    plan = wpp.wpp_plan_tiles(None, desc, P, C, opts=wpp.PlanOpts(0, 0, splits, 0, 0, shape), pin=False)
    raw = plan.host.numpy()[:plan.plan_bytes]
    assert np.array_equal(raw, wpp.wpp_plan_tiles(None, desc, P, C, opts=wpp.PlanOpts(0, 0, splits, 0, 0, shape), pin=False).host.numpy()[:plan.plan_bytes])
    check_cover(raw, P, C, Hq, Hkv)


def check_cover(raw, P, C, Hq, Hkv):
    """Every row of every head sees the key steps up to its end once, parts have places of their own and are combined once."""
    head = raw[:136].view(np.int32)
    n_units, n_combine, n_slots, off_units, off_combine, n_few = (int(head[i]) for i in (6, 7, 8, 24, 25, 30))
    units = raw[off_units:off_units + 48 * n_units].view(np.int32).reshape(-1, 12)
    combines = raw[off_combine:off_combine + 32 * n_combine].view(np.int32).reshape(-1, 8).tolist()
    seen, places = {}, {}
    for u, (req, a, b, slot, row0, row0b, rows, rowsb, h0, h1, _, pack) in enumerate(units.tolist()):
        if u < n_few:
            assert 0 < rows * rowsb <= 16
            pieces = [(h0 + k, row0, rows, row0b, h1 + k * rows) for k in range(rowsb)]
        else:
            G, rph = Hq // Hkv, 128 // pack
            pieces = [(h + k, r0, n, hf, k * rph) for hf, (h, r0, n) in enumerate([(h0, row0, rows), (h1, row0b, rowsb)]) if n
                      for k in range(min(pack, G))]
        for h, r0, n, hf, lane in pieces:
            assert 0 <= r0 and r0 + n <= C[req] and h < Hq and lane + n <= 128
            last = (P[req] + r0 + n + 127) // 128
            seen.setdefault((req, h), {}).setdefault((r0, n), []).append((a, min(b, last), slot, hf, lane))
            if slot >= 0:
                assert slot < n_slots
                for r in range(n):
                    assert (slot, hf, lane + r) not in places                            # nobody else writes there
                    places[slot, hf, lane + r] = u
    assert {(i, h) for i in range(len(C)) if C[i] for h in range(Hq)} == set(seen)
    by_row = {(c[0], c[1], c[3]): c for c in combines}
    assert len(by_row) == len(combines)
    for (req, h), blocks in seen.items():
        at = 0
        for (r0, n), parts in sorted(blocks.items()):
            assert r0 == at
            at += n
            cut = sorted(x for x in parts if x[0] < x[1])
            assert cut[0][0] == 0 and cut[-1][1] == (P[req] + r0 + n + 127) // 128
            assert all(x[1] == y[0] for x, y in zip(cut, cut[1:]))
            if parts[0][2] >= 0:
                c = by_row.pop((req, r0, h))
                assert c[2] == n and sorted(x[2] for x in parts) == list(range(c[4], c[4] + c[5]))
                assert {(x[3], x[4]) for x in parts} == {(c[6], c[7])}
            else:
                assert len(parts) == 1
        assert at == C[req]
    assert not by_row


@pytest.mark.parametrize("d,Hq,Hkv,P,C", [(128, 40, 8, [0] * 5, [9, 43, 26, 40, 31]), (128, 64, 8, [63] * 20, [2, 10] * 10), (128, 64, 8, [21] * 61, [1] * 30 + [2] * 31),
                                          (64, 8, 2, [700] * 64, [1] * 64), (128, 64, 8, list(range(255, 16384, 253)), [1] * 64)])
def test_few_row_blocks_are_dealt_out_evenly(d, Hq, Hkv, P, C):
    desc = wpp.make_desc(len(P), Hq, Hkv, d, 32, 600, 999, dtype=wpp.WPP_KV4)
    raw = wpp.wpp_plan_tiles(None, desc, P, C, opts=wpp.PlanOpts(0, 0, 0, 148, 0, 2), pin=False).host.numpy()
    head = raw[:136].view(np.int32)
    units = raw[head[24]:head[24] + 48 * head[6]].view(np.int32).reshape(-1, 12)
    first = raw[head[33]:head[33] + 4 * (head[32] + 1)].view(np.int32)
    assert first[0] == 0 and first[-1] == head[30] == len(units) and (np.diff(first) > 0).all() and head[32] <= 3 * 148
    cost = units[:, 2] - units[:, 1] + 3                   # what starting a block costs, in key steps
    assert np.add.reduceat(cost, first[:-1]).max() <= 1.25 * cost.sum() / (2 * 148) + cost.max()


def test_a_head_shard_of_a_cache_in_4_bits():
    from paper_2609_35263_b200.stages import head_shard
    pool = torch.zeros(9, 4, wpp.wpp_kv4_block_bytes(16, 64), dtype=torch.uint8)
    q, kv = torch.zeros(7, 8, 64, dtype=torch.bfloat16), torch.zeros(7, 4, 64, dtype=torch.bfloat16)
    desc, views = head_shard(1, 2, 1, 8, 4, 64, 16, 9, 9, q, q, kv, kv, pool, pool)
    assert desc.dtype == wpp.WPP_KV4 and desc.num_kv_heads == 2 and desc.num_q_heads == 4
    assert desc.kv_page_stride == 4 * 576 and desc.kv_head_stride == 576 and desc.kv_token_stride == 0
    assert views["k_pool"].data_ptr() == pool.data_ptr() + 2 * 576
    wpp.wpp_plan_tiles(None, desc, [100], [7], pin=False)


@pytest.mark.parametrize("P,C", [([0] * 40 + [200000], [900] * 40 + [128]), ([0] * 4 + [60000] * 4, [4000] * 8), (list(range(0, 64000, 2000)), [700] * 32)])
@pytest.mark.parametrize("d,Hq,Hkv", [(128, 64, 8), (64, 8, 8), (128, 40, 8)])
def test_tiles_that_fill_the_machine_take_no_more_scratch_than_the_built_in_array_has(d, Hq, Hkv, P, C):
    desc = wpp.make_desc(len(P), Hq, Hkv, d, 128, 1600, 99999, dtype=wpp.WPP_KV4)
    plan = wpp.wpp_plan_tiles(None, desc, P, C, opts=wpp.PlanOpts(0, 0, 0, 148), pin=False)
    raw = plan.host.numpy()
    check_cover(raw[:plan.plan_bytes], P, C, Hq, Hkv)
    if sum(-(-c // 256) for c in C) * Hq >= 148:
        assert plan.info.workspace_bytes <= wpp.wpp_static_scratch_bytes()
