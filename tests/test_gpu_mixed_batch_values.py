"""dif_gemm_lora where factors are infinite or near the types' largest values: what
real arithmetic gives, in every way the term is computed (runs of rows through the
matrix cores, many short runs together, every tile shape)."""
import pytest

from tests.gpu_util import say
from tests.mixed_batch import STORE, Problem
from tests.test_gpu_mixed_batch import TYPES
from tests.test_gpu_mixed_batch_tiles import CASES, _launch, _low
from tests.test_gpu_gemm_instances import BF16, F32

pytestmark = pytest.mark.gpu

INF = float("inf")


def _signs(p, j):
    """What an infinite term j of adapter 1 leaves of its rows, given that entry j of
    their low-rank product is positive."""
    import torch
    return (p.up[1, :, j].double() * p.scales[1].double()).sign() * torch.inf


def _infinite_up(rows, N, types, low, seed, j=5):
    """Adapter 1's up column j infinite with both signs; the rows' factor beside it
    positive: of any value, exact in every type (powers of two, one of them small), or
    infinite."""
    import torch
    R = len(rows)
    p = Problem(rows, N, 160, STORE, *types, adapter=[i % 2 for i in range(R)], rank=12, adapters=2, seed=seed)
    p.A.copy_(p.A.abs() + 0.25)
    p.down[1, j] = p.down[1, j].abs() + 0.01
    if low in ("exact", "tiny"):
        p.A[:, 0] = 4.0 if low == "exact" else 2.0 ** -60
        p.down[1, j] = 0.0
        p.down[1, j, 0] = 0.5 if low == "exact" else 2.0 ** -40
        p.scales[1] = 2.0
    if low == "infinite":
        p.down[1, j] = INF
    p.up[1, :, j] = torch.where(torch.arange(N, device="cuda") % 3 == 0, -INF, INF)
    return p


@pytest.mark.parametrize("low", ["any", "exact", "tiny", "infinite"])
@pytest.mark.parametrize("types", TYPES, ids="_".join)
@pytest.mark.parametrize("rows", [[40, 24], [1, 1, 1, 1, 1, 1], [700, 600, 800]], ids=str)
def test_infinite_up_factors_stay_infinite(rows, types, low):
    import torch
    say(f"lora infinite up {rows} {types} low={low}")
    p = _infinite_up(rows, 300, types, low, len(rows))
    got = p.run().double()
    _, a = p.row_of()
    hit = (a == 1).to("cuda")
    assert bool(torch.isfinite(got[~hit]).all()) and torch.equal(got[hit], _signs(p, 5).expand(int(hit.sum()), -1))


@pytest.mark.parametrize("dtype,out,shape", CASES)
def test_infinite_up_factors_in_every_tile_shape(dtype, out, shape):
    import torch
    bm, bn, _ = (F32 if dtype == "f32" else BF16)[shape]
    for rows in ([bm + 5, 3, bm - 1, 7], [1] * 21):
        say(f"infinite up, shape={shape} {dtype}->{out} rows={rows[:4]}")
        for j in range(12):   # (every place in a chunk, the last part of one)
            p = _infinite_up(rows, bn + 37, (dtype, out), ("any", "exact")[j % 2], shape + j, j)
            got = _launch(p, shape, _low(p, 1)).double()
            _, a = p.row_of()
            hit = (a == 1).to("cuda")
            assert bool(torch.isfinite(got[~hit]).all())
            assert torch.equal(got[hit], _signs(p, j).expand(int(hit.sum()), -1))


def _near_the_largest(rows, N, types, seed):
    """Adapter 1's factor 5 finite, between bf16's largest number and float32's, beside
    small entries of up."""
    R = len(rows)
    p = Problem(rows, N, 160, STORE, *types, adapter=[1 - i % 2 for i in range(R)], rank=12, adapters=2, seed=seed)
    p.A[:, 0] = (2 - 2.0 ** -7) * 2.0 ** 127   # (the largest of bf16; half a step of it is 2^119)
    p.A[:, 1] = 1.5 * 2.0 ** 119
    p.B[:, :, :2] = 0.0
    p.down[:, :, :2] = 0.0
    p.down[1, 5] = 0.0
    p.down[1, 5, :2] = 1.0
    p.scales[1] = 1.0
    p.up[1, :, 5] *= 2.0 ** -126
    return p


@pytest.mark.parametrize("types", TYPES, ids="_".join)
@pytest.mark.parametrize("rows", [[40, 24], [1, 1, 1, 1, 1, 1], [700, 600, 800]], ids=str)
def test_finite_factors_past_the_largest_bf16_stay_finite(rows, types):
    say(f"lora factor near the largest {rows} {types}")
    p = _near_the_largest(rows, 300, types, len(rows))
    p.check(p.run())


@pytest.mark.parametrize("dtype,out,shape", CASES)
def test_finite_factors_past_the_largest_bf16_in_every_tile_shape(dtype, out, shape):
    bm, bn, _ = (F32 if dtype == "f32" else BF16)[shape]
    for rows in ([bm + 5, 3, bm - 1, 7], [1] * 21):
        say(f"factor near the largest, shape={shape} {dtype}->{out} rows={rows[:4]}")
        p = _near_the_largest(rows, bn + 37, (dtype, out), shape)
        p.check(_launch(p, shape, _low(p, 1)))
