"""dif_cache_append, dif_attention_paged and dif_attention_window on the host: every
documented refusal, before any device work, and the binding's own checks."""
import ctypes as C
import math

import pytest
import torch

from paper_2607_06631_amd import binding as B

ARG, SHAPE, UNSUPPORTED, WORKSPACE = -1, -2, -4, -5
P = 0x10000   # a pointer that is never used


def _cache(**kw):
    c = B.DifKvCache(P, P, 4 * 16 * 64, 16 * 64, 64, 8, 16, 4, 64, 2, 3, P, 3, P, P)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _append(cache=None, how=None, **kw):
    d = dict(dtype=0, k=P, ldk=256, v=P, ldv=256, q=P, ldq=512, q_out=P, ldqo=512, M=5, heads=8)
    d.update(kw)
    h = B.DifAppend(None, None, 0, 1e-6, 10000.0, 1, None, 1.0)
    for k, v in (how or {}).items():
        setattr(h, k, v)
    return B.lib().dif_cache_append(d["dtype"], C.byref(_cache(**(cache or {}))), d["k"], d["ldk"], d["v"], d["ldv"], d["q"],
                                    d["ldq"], d["q_out"], d["ldqo"], d["M"], d["heads"], C.byref(h), None)


def _paged(cache=None, seen=(1, 0, 0), **kw):
    d = dict(dtype=0, flags=0, q=P, ldq=512, out=P, ldo=512, M=5, heads=8, ws=None, n=0)
    d.update(kw)
    return B.lib().dif_attention_paged(d["dtype"], d["flags"], d["q"], d["ldq"], C.byref(_cache(**(cache or {}))), d["out"],
                                       d["ldo"], d["M"], d["heads"], C.byref(B.DifSeen(*seen)), d["ws"], d["n"], None)


def _window(seen=(1, 0, 0), **kw):
    d = dict(dtype=0, dh=64, flags=0, q=P, ldq=512, k=P, ldk=256, v=P, ldv=256, out=P, ldo=512, M=5, N=9, heads=8, kv=4,
             seqs=2, off=P, koff=P, ws=None, n=0)
    d.update(kw)
    return B.lib().dif_attention_window(d["dtype"], d["dh"], d["flags"], d["q"], d["ldq"], d["k"], d["ldk"], d["v"], d["ldv"],
                                        d["out"], d["ldo"], d["M"], d["N"], d["heads"], d["kv"], d["seqs"], d["off"],
                                        d["koff"], C.byref(B.DifSeen(*seen)), d["ws"], d["n"], None)


CACHE = [
    (dict(k=None), ARG), (dict(v=None), ARG), (dict(k=P + 8), ARG), (dict(v=P + 2), ARG), (dict(table=None), ARG),
    (dict(lengths=None), ARG), (dict(row_offsets=None), ARG), (dict(table=P + 2), ARG), (dict(lengths=P + 1), ARG),
    (dict(row_offsets=P + 3), ARG), (dict(n_pages=0), SHAPE), (dict(max_pages=0), SHAPE), (dict(n_kv_heads=0), SHAPE),
    (dict(page_size=8), SHAPE), (dict(page_size=48), SHAPE), (dict(page_size=1 << 17), SHAPE), (dict(page_size=-16), SHAPE),
    (dict(max_pages=1 << 27, ld_table=1 << 27), SHAPE), (dict(max_pages=(1 << 27) - 4000, ld_table=1 << 27), SHAPE), (dict(ld_table=2), SHAPE), (dict(ld_table=1 << 50), SHAPE),
    (dict(n_seqs=0), SHAPE), (dict(n_seqs=4097), SHAPE), (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=0), UNSUPPORTED),
    (dict(page_stride=-8), SHAPE), (dict(page_stride=4), SHAPE), (dict(page_stride=1 << 31), SHAPE),
    (dict(head_stride=8), SHAPE), (dict(head_stride=66), SHAPE), (dict(head_stride=1 << 50), SHAPE),
    (dict(slot_stride=56), SHAPE), (dict(slot_stride=65), SHAPE), (dict(slot_stride=1 << 24), SHAPE),
    (dict(slot_stride=1 << 23, page_size=128), SHAPE),
]


@pytest.mark.parametrize("kw,code", CACHE, ids=str)
def test_caches(kw, code):
    assert _append(kw) == code
    assert B.lib().dif_last_error()
    assert _paged(kw) == code


@pytest.mark.parametrize("kw,how,code", [
    (dict(dtype=2), {}, ARG), (dict(M=-1), {}, SHAPE), (dict(k=None), {}, ARG), (dict(v=P + 8), {}, ARG), (dict(q=P + 4), {}, ARG),
    (dict(q_out=None), {}, ARG), (dict(q=None), {}, ARG), (dict(ldk=255), {}, SHAPE), (dict(ldv=248), {}, SHAPE),
    (dict(ldq=511), {}, SHAPE), (dict(ldqo=500), {}, SHAPE), (dict(ldk=260), {}, SHAPE), (dict(ldk=1 << 24), {}, SHAPE),
    (dict(heads=6), {}, SHAPE), (dict(heads=0), {}, SHAPE), (dict(M=2 ** 31 - 1), {}, SHAPE),
    ({}, dict(axes=2), ARG), ({}, dict(axes=-1), ARG), ({}, dict(theta=0.0), ARG), ({}, dict(theta=-1.0), ARG),
    ({}, dict(theta=math.inf), ARG), ({}, dict(theta=math.nan), ARG), ({}, dict(axes=3), ARG),
    ({}, dict(axes=0, positions=P), ARG), ({}, dict(positions=P + 2), ARG), ({}, dict(gain_k=P + 4), ARG),
    ({}, dict(gain_q=P + 8), ARG), ({}, dict(gain_k=P, eps=0.0), ARG), ({}, dict(gain_q=P, eps=math.nan), ARG),
    ({}, dict(gain_k=P, norm_dim=-1), SHAPE), (dict(q=None, q_out=None), dict(gain_q=P), ARG),
    (dict(heads=132, ldq=132 * 64, ldqo=132 * 64), dict(gain_q=P), SHAPE),
], ids=str)
def test_appends(kw, how, code):
    assert _append(None, how, **kw) == code
    assert B.lib().dif_last_error()


ATTENTION = [
    (dict(dtype=2), ARG), (dict(flags=2), ARG), (dict(M=-1), SHAPE), (dict(q=None), ARG), (dict(out=None), ARG),
    (dict(q=P + 8), ARG), (dict(out=P + 2), ARG), (dict(ldq=504), SHAPE), (dict(ldo=511), SHAPE), (dict(ldq=516), SHAPE),
    (dict(ldq=1 << 24), SHAPE), (dict(heads=6), SHAPE), (dict(heads=0), SHAPE), (dict(seen=(-1, 0, 0)), SHAPE),
    (dict(seen=(1, -1, 0)), SHAPE), (dict(seen=(1, 4, -1)), SHAPE), (dict(seen=(1, 0, 3)), ARG),
    (dict(ws=P + 128, n=1 << 30), WORKSPACE), (dict(ws=P, n=1 << 20), WORKSPACE), (dict(M=2 ** 31 - 1), SHAPE),
]


@pytest.mark.parametrize("kw,code", ATTENTION, ids=str)
def test_attention(kw, code):
    assert _paged(**kw) == code
    assert B.lib().dif_last_error()
    assert _window(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(dh=32), UNSUPPORTED), (dict(N=-1), SHAPE), (dict(N=2 ** 31 - 1), SHAPE), (dict(k=None), ARG), (dict(v=P + 8), ARG), (dict(ldk=255), SHAPE),
    (dict(ldv=8), SHAPE), (dict(ldv=1 << 24), SHAPE), (dict(kv=0), SHAPE), (dict(kv=3), SHAPE), (dict(seqs=0), SHAPE),
    (dict(seqs=5000), SHAPE), (dict(off=None), ARG), (dict(off=P + 2), ARG), (dict(koff=P + 1), ARG), (dict(koff=None), SHAPE),
], ids=str)
def test_packed(kw, code):
    assert _window(**kw) == code
    assert B.lib().dif_last_error()


def test_null_structs_and_workspace():
    lib = B.lib()
    h, s = B.DifAppend(None, None, 0, 1e-6, 10000.0, 1, None, 1.0), B.DifSeen(1, 0, 0)
    assert lib.dif_cache_append(0, None, P, 256, P, 256, None, 0, None, 0, 5, 0, C.byref(h), None) == ARG
    assert lib.dif_cache_append(0, C.byref(_cache()), P, 256, P, 256, None, 0, None, 0, 5, 0, None, None) == ARG
    assert lib.dif_attention_paged(0, 0, P, 512, None, P, 512, 5, 8, C.byref(s), None, 0, None) == ARG
    assert lib.dif_attention_paged(0, 0, P, 512, C.byref(_cache()), P, 512, 5, 8, None, None, 0, None) == ARG
    assert lib.dif_attention_paged_bytes(64, None) == ARG
    n = C.c_size_t()
    assert lib.dif_attention_paged_bytes(96, C.byref(n)) == UNSUPPORTED
    assert 0 < B.dif_attention_paged_bytes(64) < B.dif_attention_paged_bytes(128) < 1 << 28


def test_calls_with_nothing_to_do_touch_nothing():
    assert _append(M=0, k=None, v=None, q=None, q_out=None, heads=0) == 0
    assert _paged(M=0, q=None, out=None) == 0
    assert _window(M=0, q=None, out=None, k=None, v=None) == 0


def test_binding_checks_tensors():
    t = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    c = dict(cache_k=t(4, 2, 16, 64), cache_v=t(4, 2, 16, 64), table=i(1, 3), lengths=i(1), row_offsets=i(2))
    with pytest.raises(ValueError, match="device memory"):
        B.dif_cache_append(**c, k=t(3, 2, 64), v=t(3, 2, 64))
    with pytest.raises(ValueError, match="device memory"):
        B.dif_attention_paged(t(3, 4, 64), *c.values(), t(3, 4, 64))
    with pytest.raises(ValueError, match="device memory"):
        B.dif_attention_window(t(3, 4, 64), t(3, 2, 64), t(3, 2, 64), i(2), t(3, 4, 64))


def test_the_packed_struct_is_the_declared_one():
    values = tuple(range(3, 3 + len(B.DifKvCache._fields_)))
    packed = B._CACHE.pack(*values)
    assert len(packed) == C.sizeof(B.DifKvCache)
    c = B.DifKvCache.from_buffer_copy(packed)
    assert tuple(getattr(c, n) for n, _ in B.DifKvCache._fields_) == values
