"""dif_gemm_grouped, dif_gemm_lora and dif_lora_workspace_bytes on the host: every
documented refusal, before any device work, and the binding's own checks."""
import ctypes as C

import pytest

from paper_2607_06631_amd import binding as B

ARG, SHAPE, UNSUPPORTED, WORKSPACE = -1, -2, -4, -5
P = 0x10000   # a pointer that is never used


def _groups(**kw):
    g = B.DifGroups(2, 2, P, None, None, None, 64 * 64, 64, 64)
    for k, v in kw.items():
        setattr(g, k, v)
    return g


def _lora(**kw):
    l = B.DifLora(2, 2, 8, P, P, None, None, P, 64, 8 * 64, P, 8, 64 * 8)
    for k, v in kw.items():
        setattr(l, k, v)
    return l


DEFAULT = dict(dtype=0, out=0, A=P, lda=64, B=P, ldb=64, C=P, ldc=64, M=4, N=64, K=64, epi=0, bias=None, gate0=None,
               gate1=None)


def _args(kw):
    d = dict(DEFAULT, **kw)
    return tuple(d[k] for k in ("dtype", "out", "A", "lda", "B", "ldb", "C", "ldc", "M", "N", "K", "epi", "bias", "gate0",
                                "gate1"))


def _grouped(groups=None, **kw):
    g = _groups() if groups is None else groups
    return B.lib().dif_gemm_grouped(*_args(kw), C.byref(g), None)


def _adapters(lora=None, groups=None, ws=P, ws_bytes=1 << 20, **kw):
    l = _lora() if lora is None else lora
    return B.lib().dif_gemm_lora(*_args(kw), None if groups is None else C.byref(groups), C.byref(l), ws, ws_bytes, None)


PRODUCT = [
    (dict(dtype=5), ARG), (dict(out=7), ARG), (dict(dtype=1, out=0), ARG), (dict(epi=3), ARG), (dict(epi=-1), ARG),
    (dict(M=-1), SHAPE), (dict(N=-1), SHAPE), (dict(K=-1), SHAPE),
    (dict(A=None), ARG), (dict(B=None), ARG), (dict(C=None), ARG),
    (dict(A=P + 8), ARG), (dict(B=P + 2), ARG), (dict(C=P + 1), ARG), (dict(dtype=1, out=1, C=P + 2), ARG),
    (dict(lda=56), SHAPE), (dict(ldb=63), SHAPE), (dict(ldc=63), SHAPE), (dict(lda=68), SHAPE), (dict(ldb=65), SHAPE),
    (dict(lda=1 << 22), SHAPE), (dict(ldb=1 << 22), SHAPE), (dict(ldc=1 << 22), SHAPE),
    (dict(gate0=P), ARG), (dict(epi=1, gate0=P), ARG), (dict(epi=2, gate1=P), ARG),
    (dict(bias=P + 2), ARG), (dict(epi=2, gate0=P + 1), ARG),
    (dict(M=2 ** 31 - 1), SHAPE), (dict(M=2 ** 26, N=2 ** 20, ldc=2 ** 20), SHAPE),
    (dict(M=2 ** 24, N=2 ** 17, ldc=2 ** 17), SHAPE),   # (more threads than a launch counts)
    (dict(lda=1 << 55), SHAPE), (dict(ldb=1 << 55), SHAPE), (dict(ldc=1 << 55), SHAPE), (dict(dtype=1, out=1, lda=1 << 54), SHAPE),
]


@pytest.mark.parametrize("kw,code", PRODUCT, ids=lambda x: str(x))
def test_products_refusals(kw, code):
    assert _grouped(**kw) == code
    assert B.lib().dif_last_error()
    assert _adapters(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(n_groups=0), SHAPE), (dict(n_groups=4097), SHAPE), (dict(n_weights=0), SHAPE), (dict(n_weights=1), SHAPE),
    (dict(row_offsets=None), ARG), (dict(row_offsets=P + 2), ARG), (dict(weight_index=P + 1), ARG),
    (dict(n_kept=P + 1), ARG), (dict(k_kept=P + 3), ARG), (dict(b_stride=-64), SHAPE), (dict(b_stride=4), SHAPE),
    (dict(bias_stride=-1), SHAPE), (dict(gate_stride=-1), SHAPE)], ids=lambda x: str(x))
def test_groups_refusals(kw, code):
    assert _grouped(_groups(**kw)) == code
    assert _adapters(groups=_groups(**kw)) == (UNSUPPORTED if "k_kept" in kw and code == SHAPE else code)


def test_null_tables():
    assert B.lib().dif_gemm_grouped(*_args({}), None, None) == ARG
    assert B.lib().dif_gemm_lora(*_args({}), None, None, P, 1 << 20, None) == ARG
    assert B.lib().dif_lora_workspace_bytes(4, 8, None) == ARG


@pytest.mark.parametrize("kw,code", [
    (dict(n_requests=0), SHAPE), (dict(n_requests=4097), SHAPE), (dict(n_adapters=-1), SHAPE), (dict(rank=0), SHAPE),
    (dict(rank=1025), SHAPE), (dict(row_offsets=None), ARG), (dict(adapter=None), ARG), (dict(row_offsets=P + 1), ARG),
    (dict(adapter=P + 2), ARG), (dict(ranks=P + 2), ARG), (dict(scales=P + 2), ARG), (dict(down=None), ARG),
    (dict(up=None), ARG), (dict(down=P + 8), ARG), (dict(up=P + 8), ARG), (dict(ld_down=56), SHAPE),
    (dict(ld_down=68), SHAPE), (dict(ld_up=7), SHAPE), (dict(ld_up=12), SHAPE), (dict(ld_up=1 << 22), SHAPE),
    (dict(ld_down=1 << 55), SHAPE), (dict(ld_up=1 << 55), SHAPE),
    (dict(down_stride=-8), SHAPE), (dict(up_stride=4), SHAPE)], ids=lambda x: str(x))
def test_adapters_refusals(kw, code):
    assert _adapters(_lora(**kw)) == code


def test_workspace_refusals():
    need = B.dif_lora_workspace_bytes(4, 8)
    assert need >= 4 * 8 * 4
    assert _adapters(ws=None) == WORKSPACE
    assert _adapters(ws=P + 128) == WORKSPACE
    assert _adapters(ws_bytes=need - 1) == WORKSPACE
    for M, rank in ((-1, 8), (4, 0), (4, 1025)):
        with pytest.raises(B.DifError):
            B.dif_lora_workspace_bytes(M, rank)
    sizes = [B.dif_lora_workspace_bytes(m, r) for m, r in ((0, 1), (1, 1), (40000, 16), (40000, 17), (40000, 1024))]
    assert sizes[0] == 0 and sizes[2] == 40000 * 16 * 4 and sizes[3] == 40000 * 24 * 4 and sizes[4] == 40000 * 4096


def test_adapters_beside_pruned_reductions_are_refused():
    assert _adapters(groups=_groups(k_kept=P)) == UNSUPPORTED
    assert b"reduction" in B.lib().dif_last_error()


def test_calls_with_nothing_to_do_touch_nothing():
    for kw in (dict(M=0), dict(N=0, ldc=0)):
        assert _grouped(A=None, B=None, C=None, **kw) == 0
        assert _adapters(A=None, B=None, C=None, ws=None, ws_bytes=0, **kw) == 0


def test_binding_checks_tensors():
    import torch
    t = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)
    off = torch.tensor([0, 2, 4], dtype=torch.int32)
    ok = dict(A=t(4, 64), B=t(2, 32, 64), C_out=t(4, 32), row_offsets=off)
    with pytest.raises(ValueError, match="device memory"):
        B.dif_gemm_grouped(**ok)
    with pytest.raises(ValueError, match="row_offsets"):
        B.dif_gemm_grouped(**dict(ok, row_offsets=None))
    with pytest.raises(ValueError, match="device memory"):
        B.dif_gemm_lora(t(4, 64), t(32, 64), t(4, 32), off, off[:2], t(1, 8, 64), t(1, 32, 8), None)


def test_every_kernel_the_host_registers_is_in_the_device_code():
    """The names under which the host launches kernels are those of the device images:
    a name that host and device mangle apart ends the process at its first launch."""
    import re
    data = open(B.LIB_PATH, "rb").read()
    device = set(re.findall(rb"(_ZN3dif[A-Za-z0-9_$]*kernel[A-Za-z0-9_$]*)\.kd", data))
    host = set(re.findall(rb"\x00(_ZN3dif[A-Za-z0-9_$]*kernel[A-Za-z0-9_$]*)(?=\x00)", data))
    assert len(device) > 200 and all(name in host for name in device)
    assert not [name for name in host if b"$_" in name]   # (unnamed types are numbered per compilation)
