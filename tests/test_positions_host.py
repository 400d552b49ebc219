"""Pages from lengths and rotary positions: what the host computes and refuses (no GPU)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2609_35263_b200 as wpp
from oracle import positions as opos


@pytest.mark.parametrize("n", [16, 32, 64, 96, 128])
@pytest.mark.parametrize("scaling,kw", [("none", {}), ("linear", dict(factor=4.0)), ("base", dict(factor=8.0)),
                                        ("wavelength", dict(factor=8.0, original_context=8192)), ("turns", dict(factor=4.0, original_context=4096)),
                                        ("wavelength", dict(factor=2.0, original_context=500, low=0.5, high=6.0)),
                                        ("turns", dict(factor=16.0, original_context=32768, low=2.0, high=64.0)),
                                        ("turns", dict(factor=2.0, original_context=1, low=1.0, high=1.5))])
@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_frequencies(n, scaling, kw, base):
    turns, magnitude = wpp.wpp_rope_frequencies(n, base=base, scaling=scaling, **kw)
    want, m = opos.frequencies(n, base=base, scaling=scaling, **kw)
    got = np.array([int(x) for x in turns.tolist()], dtype=np.float64) / 2.0 ** 64 * 2 * np.pi
    # a few roundings of 64-bit powers and quotients (2^-53 each; a power's exponent adds up to 14 times that), and half of 2^-64 of a turn
    assert turns.dtype == torch.int64 and turns.shape == (n // 2,) and np.all(np.abs(got - want) <= 64 * 2.0 ** -53 * want + 2 * np.pi * 2.0 ** -64)
    assert abs(magnitude - m) <= 2.0 ** -23


def test_frequencies_that_are_refused():
    for n in (0, 8, 24, 130, 144, -16):
        with pytest.raises(wpp.WppError) as e:
            wpp.wpp_rope_frequencies(n)
        assert e.value.status == 2
    for kw in (dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")), dict(scaling="linear", factor=0.5), dict(scaling="linear", factor=float("nan")),
               dict(scaling="turns", factor=2.0), dict(scaling="wavelength", factor=2.0, original_context=8192, low=4.0, high=4.0),
               dict(scaling="wavelength", factor=2.0, original_context=8192, low=-1.0), dict(scaling="other")):
        with pytest.raises(wpp.WppError) as e:
            wpp.wpp_rope_frequencies(64, **kw)
        assert e.value.status == 1, kw


class _NoContext:
    handle, device = ctypes.c_void_p(), -1          # (tensors of the host say device -1)


class _Stream:
    cuda_stream = 0


def _bf(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16)


def _rope(ctx=_NoContext(), **kw):
    wpp.load_library()
    a = dict(q=_bf(5, 4, 64), k=_bf(5, 2, 64), turns=torch.zeros(32, dtype=torch.int64), positions=torch.zeros(5, dtype=torch.int32))
    a.update(kw)
    wpp.wpp_rope(ctx, **a, stream=_Stream())


def _append(ctx=_NoContext(), desc=None, **kw):
    wpp.load_library()
    a = dict(q=_bf(5, 4, 64), k_new=_bf(5, 2, 64), v_new=_bf(5, 2, 64), q_out=None, k_cache=_bf(8, 2, 16, 64), v_cache=_bf(8, 2, 16, 64),
             turns=torch.zeros(32, dtype=torch.int64), positions=torch.zeros(5, dtype=torch.int32), slots=torch.zeros(5, dtype=torch.int64))
    a.update(kw)
    wpp.wpp_rope_append(ctx, desc or wpp.make_desc(1, 4, 2, 64, 16, 4, 8), **a, stream=_Stream())


def _pages(ctx=_NoContext(), desc=None, **kw):
    wpp.load_library()
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)
    a = dict(prefix_lens=i32(3), chunk_lens=i32(3), free_pages=i32(9), cursor=i32(2), block_tables=i32(3, 4), row_offsets=torch.zeros(4, dtype=torch.int64),
             positions=i32(7), slots=torch.zeros(7, dtype=torch.int64))
    a.update(kw)
    wpp.wpp_assign_pages(ctx, desc or wpp.make_desc(3, 4, 2, 64, 16, 4, 8), **a, stream=_Stream())


@pytest.fixture
def reached(monkeypatch):
    """Calls that pass the binding reach a null context, which the library answers with WPP_ERR_INVALID_ARG: told apart by the library
    being asked at all."""
    lib = wpp.load_library()
    seen = []
    P = ctypes.c_void_p

    def stub(name, n):
        kind = ctypes.CFUNCTYPE(ctypes.c_int, *([P] * n))
        f = kind(lambda *a: seen.append((name, a)) or 0)
        return f
    from paper_2609_35263_b200 import binding
    stubs = [stub("rope", 9), stub("rope_append", 14), stub("pages", 15)]
    binding._call.init_tensors(*(ctypes.cast(f, P).value for f in stubs), torch.bfloat16, torch.int32, torch.int64)
    yield seen
    binding._call.init_tensors(*(ctypes.cast(f, P).value for f in (lib.wpp_rope, lib.wpp_rope_append, lib.wpp_assign_pages)), torch.bfloat16, torch.int32,
                               torch.int64)


def _refused(reached, call, **kw):
    n = len(reached)
    with pytest.raises(wpp.WppError) as e:
        call(**kw)
    assert e.value.status == 1 and len(reached) == n, kw


def test_what_rope_takes_and_refuses(reached):
    packed = _bf(5, 9, 80)
    for kw in (dict(), dict(q=None), dict(k=None), dict(q=packed[:, :4, :64], k=packed[:, 4:6, :64]), dict(q=_bf(1, 4, 64), k=_bf(1, 2, 64)),
               dict(q=_bf(0, 4, 64), k=_bf(0, 2, 64)), dict(q_out=_bf(5, 4, 64)), dict(positions=torch.zeros(9, dtype=torch.int32)), dict(interleaved=True)):
        n = len(reached)
        _rope(**kw)
        assert len(reached) == n + 1, kw
    for kw in (dict(q=_bf(5, 4, 64).float()), dict(q=_bf(5, 256)), dict(q=_bf(4, 4, 64)), dict(k=_bf(5, 2, 128)), dict(q=None, k=None),
               dict(q_out=_bf(5, 4, 32)), dict(q_out=_bf(5, 3, 64)), dict(k_out=_bf(4, 2, 64)), dict(q=_bf(5, 64, 4).transpose(1, 2)),
               dict(q=_bf(1, 4, 64).expand(5, 4, 64)), dict(k=_bf(5, 1, 64).expand(5, 2, 64)), dict(turns=torch.zeros(32)),
               dict(turns=torch.zeros(64, dtype=torch.int64)[::2]), dict(positions=torch.zeros(4, dtype=torch.int32)),
               dict(positions=torch.zeros(5, dtype=torch.int64)), dict(positions=torch.zeros(5, 2, dtype=torch.int32))):
        _refused(reached, _rope, **kw)
    ctx = _NoContext()
    ctx.device = 0                                   # tensors of another device than the context's
    _refused(reached, _rope, ctx=ctx)


def test_tensors_of_a_subclass_answer_for_themselves(reached):
    class Elsewhere(torch.Tensor):
        def get_device(self):
            return 7

    q, k = torch.nn.Parameter(_bf(5, 4, 64)), _bf(5, 2, 64)
    _rope(q=q, k=k)
    assert [x[0] for x in reached] == ["rope"] and reached[0][1][2] == q.data_ptr()      # (where it is, not a copy)
    _refused(reached, _rope, k=k.as_subclass(Elsewhere))
    with pytest.raises(AttributeError):
        _rope(q=7)
    with pytest.raises(AttributeError):
        _rope(turns=object())


def test_what_rope_append_takes_and_refuses(reached):
    for kw in (dict(), dict(q=None), dict(slots=torch.zeros(6, dtype=torch.int64)), dict(v_new=_bf(5, 3, 64)[:, :2])):
        n = len(reached)
        _append(**kw)
        assert len(reached) == n + 1, kw
    for kw in (dict(k_new=None), dict(v_new=_bf(5, 1, 64)), dict(v_new=_bf(6, 2, 64)), dict(slots=torch.zeros(4, dtype=torch.int64)),
               dict(slots=torch.zeros(5, dtype=torch.int32)), dict(q_out=_bf(5, 2, 64)), dict(v_new=_bf(5, 1, 64).expand(5, 2, 64))):
        _refused(reached, _append, **kw)


def test_what_assign_pages_takes_and_refuses(reached):
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)
    for kw in (dict(), dict(positions=None), dict(slots=None), dict(positions=None, slots=None), dict(free_pages=i32(0)), dict(cursor_out=i32(2)),
               dict(prefix_lens=i32(4)), dict(block_tables=i32(5, 4))):
        n = len(reached)
        _pages(**kw)
        assert len(reached) == n + 1, kw
    for kw in (dict(prefix_lens=i32(2)), dict(chunk_lens=torch.zeros(3, dtype=torch.int64)), dict(cursor=i32(1)), dict(cursor_out=i32(1)),
               dict(block_tables=i32(2, 4)), dict(block_tables=i32(3, 5)), dict(block_tables=i32(4, 3).t()), dict(block_tables=i32(6, 4)[::2]),
               dict(row_offsets=torch.zeros(3, dtype=torch.int64)), dict(row_offsets=i32(4)), dict(slots=i32(7)), dict(positions=i32(14)[::2])):
        _refused(reached, _pages, **kw)


def test_the_shorter_of_positions_and_slots_counts(reached):
    _pages(slots=torch.zeros(5, dtype=torch.int64))
    assert reached[-1][0] == "pages" and reached[-1][1][12] == 5


def test_a_null_context_reaches_the_library():
    for call in (_rope, _append, _pages):
        with pytest.raises(wpp.WppError) as e:
            call()
        assert e.value.status == 1


def test_structures_match_the_header():
    from . import test_abi_layout as abi
    import os
    import re
    import subprocess
    import tempfile
    from paper_2609_35263_b200 import binding as B
    hdr = open(os.path.join(abi.ROOT, "include", "wpp.h")).read()
    pairs = {"wpp_rope_scaling": B.RopeScaling, "wpp_rope_desc": B.RopeDesc, "wpp_linear_desc": B.LinearDesc}
    with tempfile.TemporaryDirectory() as tmp:
        src, exe = os.path.join(tmp, "abi.c"), os.path.join(tmp, "abi")
        lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "wpp.h"', "int main(void) {"]
        for name in pairs:
            lines.append(f'printf("{name} size %zu\\n", sizeof({name}));')
            lines += [f'printf("{name} {f} %zu\\n", offsetof({name}, {f}));' for f in abi._c_fields(name, hdr)]
        open(src, "w").write("\n".join(lines + ["return 0;", "}"]))
        subprocess.check_call(["gcc", "-I", os.path.join(abi.ROOT, "include"), src, "-o", exe])
        seen = {}
        for line in subprocess.check_output([exe], text=True).splitlines():
            name, field, value = line.split()
            seen.setdefault(name, {})[field] = int(value)
    for name, cls in pairs.items():
        assert {"size": ctypes.sizeof(cls), **{n: getattr(cls, n).offset for n, _ in cls._fields_}} == seen[name], name


def _desc(**kw):
    d = wpp.RopeDesc(4, 2, 64, 64, 0, 1.0, 5)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def test_what_the_library_refuses_before_it_looks_for_a_device():
    """(The context is only asked for not being null before the description and the pointers are looked at.)"""
    lib = wpp.load_library()
    fake, at = ctypes.c_void_p(256), [ctypes.c_void_p(4096 * (i + 1)) for i in range(8)]

    def rope(desc, q=at[0], q_out=at[0], k=at[1], k_out=at[1], turns=at[2], positions=at[3]):
        return lib.wpp_rope(fake, ctypes.byref(desc) if desc else None, q, q_out, k, k_out, turns, positions, None)
    assert rope(None) == 1
    for kw, st in ((dict(head_dim=96), 2), (dict(rot_dim=24), 2), (dict(rot_dim=80), 2), (dict(rot_dim=0), 2), (dict(interleaved=2), 1),
                   (dict(magnitude=float("nan")), 1), (dict(magnitude=float("inf")), 1), (dict(q_token_stride=60), 1), (dict(k_head_stride=68), 1),
                   (dict(total_tokens=-1), 1), (dict(num_q_heads=-1), 1), (dict(num_q_heads=70000), 2)):
        assert rope(_desc(**kw)) == st, kw
    assert rope(_desc(total_tokens=0), None, None, None, None, None, None) == 0
    for kw in (dict(q=None), dict(q_out=None), dict(k=None), dict(turns=None), dict(positions=None), dict(turns=ctypes.c_void_p(8)), dict(q=ctypes.c_void_p(4104))):
        assert rope(_desc(), **kw) == 1, kw
    assert rope(_desc(qo_token_stride=512)) == 1                       # in place, but with other strides

    def append(batch, desc):
        return lib.wpp_rope_append(fake, ctypes.byref(batch), ctypes.byref(desc), *at[:6], at[6], at[7], at[0], None, None)
    batch = lambda **kw: wpp.make_desc(1, 4, 2, 64, 16, 4, 8, **kw)
    assert append(batch(dtype=wpp.WPP_KV8), _desc()) == 2 and append(batch(dtype=wpp.WPP_KV4), _desc()) == 2
    assert append(batch(), _desc(num_k_heads=1)) == 1 and append(batch(), _desc(num_q_heads=8)) == 1 and append(batch(), _desc(head_dim=128)) == 1
    assert append(batch(), _desc(total_tokens=0)) == 0

    def pages(batch, num_free=4, most=8, **kw):
        a = dict(prefix=at[0], chunks=at[1], free=at[2], cursor=at[3], cursor_out=at[3], tables=at[4], rows=at[5], positions=at[6], slots=at[7])
        a.update(kw)
        return lib.wpp_assign_pages(fake, ctypes.byref(batch), a["prefix"], a["chunks"], a["free"], num_free, a["cursor"], a["cursor_out"], a["tables"],
                                    a["rows"], a["positions"], a["slots"], most, None, None)
    assert pages(batch(), num_free=-1) == pages(batch(), most=-1) == 1
    assert pages(wpp.make_desc(16385, 4, 2, 64, 16, 4, 8)) == 2
    for name in ("prefix", "chunks", "free", "cursor", "cursor_out", "tables", "rows"):
        assert pages(batch(), **{name: None}) == 1, name


def test_rope_append_looks_at_its_pools(reached):
    """Keys and values go to computed places of them: what is of another type or ends too early is refused."""
    both, kv = _bf(8, 2, 2, 16, 64), wpp.make_desc(1, 4, 2, 64, 16, 4, 8, kv_page_stride=2 * 2 * 16 * 64)
    packed = wpp.make_desc(1, 4, 2, 64, 16, 4, 8, kv_token_stride=128, kv_head_stride=128 * 16, kv_page_stride=128 * 32)
    for kw in (dict(), dict(k_cache=_bf(9, 2, 16, 64)), dict(k_cache=_bf(8 * 2 * 16 * 64)), dict(v_cache=_bf(4, 2, 2, 2, 16, 64)), dict(k_cache=both, v_cache=both[:, 1], desc=kv),
               dict(k_cache=both[:, 0], v_cache=both.view(-1)[2 * 16 * 64:], desc=kv), dict(k_cache=_bf(8, 2, 16, 128)[..., :64], v_cache=_bf(8, 2, 16, 128)[..., 64:], desc=packed),
               dict(k_cache=torch.nn.Parameter(_bf(8, 2, 16, 64))), dict(k_cache=None), dict(desc=wpp.make_desc(1, 4, 2, 64, 16, 4, 8, dtype=wpp.WPP_KV8), k_cache=_bf(1)),
               dict(q=_bf(0, 4, 64), k_new=_bf(0, 2, 64), v_new=_bf(0, 2, 64), k_cache=_bf(1)), dict(desc=wpp.make_desc(1, 4, 2, 64, 16, 4, 8, kv_page_stride=-8))):
        n = len(reached)
        _append(**kw)                                    # (the stub in the library's place takes everything)
        assert len(reached) == n + 1, kw
    for name in ("k_cache", "v_cache"):
        for pool in (_bf(7, 2, 16, 64), _bf(8, 1, 16, 64), _bf(8, 2, 16, 32), _bf(8, 2, 16, 64)[1:], _bf(8 * 2 * 16 * 64 - 1), _bf(0, 2, 16, 64), _bf(8, 2, 16, 64).float(),
                     _bf(8, 2, 16, 64).half(), torch.zeros(8, 2, 16 * 64 * 2, dtype=torch.uint8), _bf(1, 2, 16, 64).expand(8, 2, 16, 64)):
            _refused(reached, _append, **{name: pool})
        _refused(reached, _append, **{"k_cache": both[:, 0], "v_cache": both[:, 1], "desc": kv, name: _bf(8, 2, 16, 64)})
        _refused(reached, _append, **{"desc": wpp.make_desc(1, 4, 2, 64, 16, 4, 2 ** 31 - 1, kv_page_stride=2 ** 62), name: _bf(8, 2, 16, 64)})

    class Elsewhere(torch.Tensor):
        def get_device(self):
            return 7
    for name in ("k_cache", "v_cache"):
        _refused(reached, _append, **{name: _bf(8, 2, 16, 64).as_subclass(Elsewhere)})
        with pytest.raises(AttributeError):
            _append(**{name: 4096})
