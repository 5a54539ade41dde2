"""Every tile shape of the mixed-batch products through its launcher.

The estimate that picks a shape would leave some reached only at sizes no test has.
Here each is asked for, at row counts below, at and past its tile, reductions of
fewer, as many and more k-tiles than it keeps in flight and with a last chunk of any
length, and adapters whose runs begin and end inside tiles.  References as in
tests/mixed_batch.py; without adapters all shapes must give the same bits.
"""
import ctypes as C

import pytest

from paper_2607_06631_amd import binding as B
from tests.gpu_util import say
from tests.mixed_batch import GELU, RESIDUAL, STORE, Problem
from tests.test_gpu_gemm_instances import BF16, F32, _Params

pytestmark = pytest.mark.gpu

SMALLEST = 10


class _Batch(C.Structure):
    _fields_ = [("g", _Params), ("group_off", C.c_void_p), ("w_index", C.c_void_p), ("n_groups", C.c_int),
                ("n_weights", C.c_int), ("spread", C.c_int), ("n_kept", C.c_void_p), ("k_kept", C.c_void_p),
                ("b_stride", C.c_int64), ("bias_stride", C.c_int64), ("gate_stride", C.c_int64),
                ("request_off", C.c_void_p), ("adapter", C.c_void_p), ("n_requests", C.c_int), ("n_adapters", C.c_int),
                ("rank", C.c_int), ("ranks", C.c_void_p), ("scales", C.c_void_p), ("low", C.c_void_p),
                ("ld_low", C.c_int), ("low_parts", C.c_int), ("low_stride", C.c_int64), ("up", C.c_void_p),
                ("ld_up", C.c_int64), ("up_stride", C.c_int64), ("parts", C.c_int), ("k_part", C.c_int),
                ("c_part", C.c_int64)]


def _ptr(t):
    return None if t is None else t.data_ptr()


def _launch(p, shape, low=None):
    """Problem p in tiles of `shape`; low [parts, M, ld] where it has adapters."""
    import torch
    t, out = p.tables(), p.fresh()
    x = _Batch()
    g = x.g
    g.A, g.C, g.lda, g.ldb, g.ldc = p.A.data_ptr(), out.data_ptr(), p.A.stride(0), p.B.stride(1), out.stride(0)
    g.Bs[0], g.biases[0] = p.B.data_ptr(), _ptr(p.bias)
    g.M, g.N, g.K, g.nseg, g.gate0, g.gate1 = p.M, p.N, p.K, 1, _ptr(p.gate0), _ptr(p.gate1)
    g.vec4 = int(g.ldc % 4 == 0)
    off = t["group_offsets"] if p.lora else t["row_offsets"]
    x.group_off, x.n_groups = _ptr(off), 1 if off is None else off.numel() - 1
    x.w_index, x.n_weights = _ptr(t["weight_index"]), p.W
    x.n_kept, x.k_kept = _ptr(t["n_kept"]), _ptr(t.get("k_kept"))
    x.b_stride, x.bias_stride, x.gate_stride = p.B.stride(0), p.N, p.N
    if p.lora:
        x.request_off, x.adapter, x.n_requests = _ptr(t["row_offsets"]), _ptr(t["adapter"]), len(p.rows)
        x.n_adapters, x.rank, x.ranks, x.scales = p.adapters, p.rank, _ptr(t["ranks"]), _ptr(p.scales)
        x.low, x.ld_low, x.low_parts, x.low_stride = _ptr(low), low.shape[2], low.shape[0], low.stride(0)
        x.up, x.ld_up, x.up_stride = p.up.data_ptr(), p.up.stride(1), p.up.stride(0)
    stream = torch.cuda.current_stream().cuda_stream
    types = {"bf16bf16": "DF16bDF16b", "bf16f32": "DF16bf", "f32f32": "ff"}[p.dtype + p.out]
    if shape == 0:
        f = getattr(B.lib(), "_ZN3dif21launch_gemm_batch_256I%sEE10hipError_tRKNS_11BatchParamsIDF16bT_EEiP12ihipStream_t"
                    % ("DF16b" if p.out == "bf16" else "f"))
        f.restype, f.argtypes = C.c_int, [C.c_void_p, C.c_int, C.c_void_p]
        assert f(C.addressof(x), p.epi, stream) == 0
    else:
        f = getattr(B.lib(), f"_ZN3dif22launch_gemm_batch_ringI{types}EE10hipError_tiRKNS_11BatchParamsIT_T0_EEiP12ihipStream_t")
        f.restype, f.argtypes = C.c_int, [C.c_int, C.c_void_p, C.c_int, C.c_void_p]
        assert f(shape, C.addressof(x), p.epi, stream) == 0
    torch.cuda.synchronize()
    return out


def _low(p, parts):
    """The rows' products with their adapters' down matrices, in `parts` of the sum;
    entries that nothing may read are NaN."""
    import torch
    ld = -(-p.rank // 8) * 8
    low = torch.full((parts, p.M, ld), float("nan"), device="cuda")
    _, a = p.row_of()
    for i in range(p.adapters):
        r = (a == i).nonzero().flatten().to("cuda")
        j = min(max(p.ranks[i], 0), p.rank) if p.ranks is not None else p.rank
        if not r.numel():
            continue
        cut = [p.K * s // parts for s in range(parts + 1)]
        for s in range(parts):
            low[s, r, :j] = (p.A[r, cut[s]:cut[s + 1]].double() @ p.down[i, :j, cut[s]:cut[s + 1]].double().t()).float()
    return low


CASES = ([("bf16", "bf16", s) for s in BF16 if s != 12] + [("bf16", "f32", s) for s in BF16 if s != 12] +
         [("f32", "f32", s) for s in F32])


@pytest.mark.parametrize("dtype,out,shape", CASES)
def test_grouped_shapes(dtype, out, shape):
    import torch
    bm, bn, nst = (F32 if dtype == "f32" else BF16)[shape]
    kt, vec = (32, 4) if dtype == "f32" else (64, 8)
    for n, (K, epi) in enumerate(((kt - 1, STORE), (kt, GELU), (nst * kt + vec, RESIDUAL), ((nst + 1) * kt + 5, STORE),
                                  ((2 * nst - 1) * kt, GELU), (2 * nst * kt, RESIDUAL), (2 * nst * kt + 1, GELU),
                                  ((2 * nst + 1) * kt - vec, STORE), ((3 * nst + 2) * kt + 3 * vec + 2, RESIDUAL))):
        rows = [bm + 5, 1, 0, 2 * bm, 7]
        N = bn + (37 if n % 2 else 36)
        say(f"grouped tile shape={shape} {dtype}->{out} N={N} K={K} epi={epi}")
        p = Problem(rows, N, K, epi, dtype, out, weights=3, index=[0, 1, 2, 1, 0], n_kept=[N, bn + 1, 3],
                    k_kept=[K, max(K - vec - 1, 1), K // 2], pad=8 * (n % 2), seed=shape + n)
        c = _launch(p, shape)
        p.check(c)
        assert torch.equal(c, _launch(p, SMALLEST))


@pytest.mark.parametrize("dtype,out,shape", CASES)
def test_adapter_shapes(dtype, out, shape):
    bm, bn, _ = (F32 if dtype == "f32" else BF16)[shape]
    kt = 32 if dtype == "f32" else 64
    runs = ([bm + 5, 3, 2 * bm - 1], [1] * 21, [5, 1, 0, bm // 2, 9, 1, 1, 40], [2 * bm])
    for n, (rank, ranks, parts, epi) in enumerate(((1, None, 1, STORE), (kt // 2, None, 4, GELU),
                                                   (kt // 2 + 1, [kt // 2 + 1, 3, 0], 1, RESIDUAL),
                                                   (2 * kt + 7, [2 * kt + 7, kt, kt + 1], 12, STORE))):
        for rows in runs:
            N, K = bn + (37 if n % 2 else 36), 2 * kt
            say(f"adapter tile shape={shape} {dtype}->{out} rows={rows} rank={rank}")
            p = Problem(rows, N, K, epi, dtype, out, adapter=[(i * 2 + n) % 4 - 1 for i in range(len(rows))], rank=rank,
                        adapters=3, ranks=ranks, pad=8 * (n % 2), seed=shape + n)
            p.check(_launch(p, shape, _low(p, parts)))
