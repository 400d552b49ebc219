"""The oracle of linear attention against its closed forms, and the library's refusals that need no GPU."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2609_35263_b200 as wpp
import paper_2609_35263_b200.binding as B
from oracle.linear import linear_chunk


def _inputs(T, H, d, seed=0):
    rng = np.random.default_rng(seed)
    return rng.standard_normal((T, H, d)), rng.standard_normal((T, H, d)), rng.standard_normal((T, H, d)), -np.exp(rng.uniform(-4, 1, (T, H)))


def test_the_recurrence_is_masked_attention_with_weights():
    q, k, v, g = _inputs(30, 2, 8)
    pool = np.random.default_rng(1).standard_normal((2, 2, 8, 8))
    start = pool[0].copy()
    o, _ = linear_chunk(q, k, v, g, [30], pool, [0], [1], scale=0.3)
    c = np.cumsum(g, 0)
    for h in range(2):
        w = np.exp(np.minimum(c[:, None, h] - c[None, :, h], 0)) * np.tril(np.ones((30, 30)))
        want = 0.3 * ((q[:, h] @ k[:, h].T * w) @ v[:, h] + np.exp(c[:, h])[:, None] * (q[:, h] @ start[h]))
        assert np.allclose(o[:, h], want, rtol=1e-10)
        assert np.allclose(pool[1, h], np.exp(c[-1, h]) * start[h] + (k[:, h] * np.exp(c[-1, h] - c[:, h])[:, None]).T @ v[:, h], rtol=1e-10)


def test_chunks_follow_one_another_and_snapshots_are_states_on_the_way():
    q, k, v, g = _inputs(50, 3, 4, seed=2)
    pool = np.zeros((4, 3, 4, 4))
    whole, _ = linear_chunk(q, k, v, g, [50], pool, [-1], [0], prefix_lens=[14], snap_interval=32, snap_slots=np.array([[1, 2]]))
    first, _ = linear_chunk(q[:18], k[:18], v[:18], g[:18], [18], pool, [-1], [3])
    assert np.array_equal(pool[1], pool[3]) and np.array_equal(first, whole[:18])
    rest, _ = linear_chunk(q[18:], k[18:], v[18:], g[18:], [32], pool, [3], [3])
    assert np.array_equal(rest, whole[18:]) and np.array_equal(pool[3], pool[0]) and np.array_equal(pool[2], pool[0])


def test_a_decay_of_minus_infinity_forgets():
    q, k, v, g = _inputs(9, 1, 4, seed=3)
    g[5] = -np.inf
    pool = np.ones((1, 1, 4, 4))
    o, _ = linear_chunk(q, k, v, g, [9], pool, [0], [0])
    again, _ = linear_chunk(q[5:], k[5:], v[5:], g[5:], [4], pool, [-1], [-1])
    assert np.array_equal(o[5:], again)


# ------------------------------------------------------------------------------------------------------ the host's refusals
def test_entry_point_rejects_without_touching_a_gpu():
    lib = B.load_library()
    desc = B.LinearDesc(1, 1, 128, 1, total_tokens=4)
    assert lib.wpp_linear_chunk(None, ctypes.byref(desc), *([None] * 12), 0, None, None) == 1
    fake = ctypes.create_string_buffer(1 << 16)

    def call(**kw):
        d = B.LinearDesc(1, 4, 128, 1, total_tokens=4)
        for n, v in kw.items():
            setattr(d, n, v)
        return lib.wpp_linear_chunk(fake, ctypes.byref(d), *([None] * 12), 0, None, None)
    for name in ("num_requests", "num_slots", "snap_interval", "max_snaps", "layout", "total_tokens", "q_token_stride", "decay_token_stride"):
        assert call(**{name: -1}) == 1, name
    assert call(num_heads=0) == 1 and call(layout=3) == 1 and call(scale=float("nan")) == 1 and call(scale=float("inf")) == 1
    assert call(head_dim=96) == 2 and call(num_requests=70000) == 2 and call(num_heads=70000) == 2
    assert call(num_requests=0) == 0


def test_workspace_bytes():
    assert wpp.wpp_linear_workspace_bytes(4, 8, 128, 1000) > 0
    assert wpp.wpp_linear_workspace_bytes(4, 8, 96, 1000) == wpp.wpp_linear_workspace_bytes(-1, 8, 128, 1000) == 0


class _NoContext:
    handle, device = ctypes.c_void_p(), 0


class _Stream:
    cuda_stream = 0


def _call(**kw):
    x, i = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int64)
    a = dict(q=x, k=x, v=x, log_decay=torch.zeros(4, 2), row_offsets=i, state_pool=torch.zeros(1, 2, 64, 64), state_in=i, state_out=i, out=x,
             stream=_Stream())
    a.update(kw)
    wpp.wpp_linear_chunk(_NoContext(), **a)


@pytest.mark.parametrize("kw", [
    {}, dict(k=torch.zeros(4, 2, 32)), dict(out=torch.zeros(3, 2, 64)), dict(log_decay=torch.zeros(3)), dict(log_decay=torch.zeros(4, 3)),
    dict(q=torch.zeros(4, 64, 2).transpose(1, 2)), dict(v=torch.zeros(2, 4, 64).transpose(0, 1)), dict(log_decay=torch.zeros(2, 4).t())])
def test_shapes_and_orders_that_are_refused(kw):
    with pytest.raises(wpp.WppError) as e:
        _call(**kw)
    assert e.value.status == 1


@pytest.mark.parametrize("name", ["state_in", "prefix_lens", "workspace", "status"])
def test_an_integer_is_no_memory(name):
    with pytest.raises(AttributeError):
        _call(**{name: 64})


# ----------------------------------------------------------------------------------- what the binding refuses before the library sees it
@pytest.fixture
def queued(monkeypatch):
    """The calls that would have reached the library."""
    B.load_library()
    calls = []

    class Calls:
        @staticmethod
        def linear_chunk(*a):
            calls.append(a)
            return 0
    monkeypatch.setattr(B, "_call", Calls)
    return calls


def test_a_call_that_is_right_is_queued(queued):
    _call()
    assert len(queued) == 1


@pytest.mark.parametrize("pool", [
    torch.zeros(3, 1, 64, 64), torch.zeros(3, 2, 64, 32), torch.zeros(3, 2, 32, 64), torch.zeros(3, 2, 64 * 64), torch.zeros(2, 64, 64),
    torch.zeros(3, 2, 64, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, 64, dtype=torch.float64), torch.zeros(3, 2, 64, 128)[..., ::2],
    torch.zeros(6, 2, 64, 64)[::2], torch.zeros(3, 2, 64, 64).transpose(2, 3)],
    ids=["a head too few", "half the width", "half the height", "flat", "no slots", "bf16", "fp64", "gaps in rows", "gaps between slots", "transposed"])
def test_a_pool_that_is_not_one_of_such_states_is_refused(queued, pool):
    """The kernels write whole slots: of a smaller pool they would write what lies behind it."""
    with pytest.raises(wpp.WppError) as e:
        _call(state_pool=pool)
    assert e.value.status == 1 and not queued


@pytest.mark.parametrize("name", ["q", "k", "v", "out"])
def test_one_row_for_all_tokens_is_refused(queued, name):
    """A broadcast row has a stride of 0, which the library takes for rows behind one another: it would read and write behind the row."""
    row = torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(wpp.WppError) as e:
        _call(**{name: row.expand(4, 2, 64)})
    assert e.value.status == 1 and not queued


def test_one_token_may_have_any_stride(queued):
    x = torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    _call(q=x.expand(1, 2, 64), k=x.as_strided((1, 2, 64), (0, 64, 1)), v=x, out=x, log_decay=torch.zeros(1, 2))
    assert queued[0][1].q_token_stride == queued[0][1].k_token_stride == 128


def test_one_row_of_decays_for_all_tokens_is_a_decay_per_head(queued):
    _call(log_decay=torch.zeros(2).expand(4, 2))
    assert queued[0][1].decay_token_stride == 0


_I32 = dict(dtype=torch.int32)


@pytest.mark.parametrize("kw", [
    dict(log_decay=torch.zeros(4, 2, dtype=torch.bfloat16)), dict(log_decay=torch.zeros(2, dtype=torch.float16)),
    dict(row_offsets=torch.zeros(2, **_I32)), dict(state_in=torch.zeros(0, **_I32)), dict(state_out=torch.zeros(0, **_I32)),
    dict(prefix_lens=torch.zeros(0, **_I32), snap_interval=2), dict(snap_slots=torch.zeros(2, **_I32)),
    dict(snap_slots=torch.zeros(0, 2, **_I32)), dict(snap_slots=torch.zeros(1, 4, **_I32)[:, ::2])],
    ids=["bf16 decays", "fp16 decays", "32-bit offsets", "no state_in", "no state_out", "no prefixes", "flat snapshots", "no snapshots", "gaps"])
def test_arrays_that_are_shorter_than_what_is_read_are_refused(queued, kw):
    with pytest.raises(wpp.WppError) as e:
        _call(**kw)
    assert e.value.status == 1 and not queued
