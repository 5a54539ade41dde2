"""Root-mean-square errors of dif_gemm_grouped and dif_gemm_lora against float64, where
the entrywise bound of tests/mixed_batch.py, a worst case, is far above them.

With u = 2^-24, half a float32 step: rounding to the nearest is off by c u of the value
in the root mean square, c = sqrt(E[step^2] / 12 E[x^2]) / u = 0.39 for values spread
evenly over a binade's logarithm and at most 0.43.  A running sum of n random products
of equal size s has, after t of them, size s sqrt(t); rounded after every product its
error is c u s sqrt(sum_t t) = c u s n / sqrt(2), relative to the result s sqrt(n)
c u sqrt(n / 2); rounded after every fourth product half of that.

  sums of 768 products (24 k-tiles of 32 floats) set aside, n = 13105: 18 sums at
  c u s 768 / sqrt(2) each and their running sum give at most
  c u sqrt(18 * 768^2 / 2 + 768 * 18^2 / 2) / sqrt(13105) = 8.8 u rounded after every
  product; one running sum rounded only after every fourth gives 17 u: 12 u lies between.

  a low-rank term alone: 64 products for the factor and three times 32 for the term are
  off by 0.43 u sqrt(32 + 48) = 3.9 u at most with all 24 bits of the factor; with 16 of
  them its rounding alone is 0.3 * 2^-16 = 77 u: 16 u lies between.

  the same stored as bf16: its rounding, 0.39 to 0.43 of 2^-8, with 16 bits of the
  factor; with 8 of them twice the variance, 0.55 of 2^-8: 0.46 lies between.
"""
import math

import pytest

from tests.gpu_util import say
from tests.mixed_batch import STORE, Problem
from tests.test_gpu_mixed_batch_tiles import CASES, _launch, _low
from tests.test_gpu_gemm_instances import BF16, F32

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _rms(p, got, limit):
    import torch
    want, _ = p.reference()
    err = (got.double() - want).square().mean().sqrt().item() / want.square().mean().sqrt().item()
    say(f"  rms error {err:.3e}, limit {limit:.3e}")
    assert math.isfinite(err) and err <= limit


@pytest.mark.parametrize("rows", [[67], [1] * 8, [300, 21, 700], [2100]], ids=str)
def test_long_sums_of_float32(rows):
    say(f"precision of float32 sums of 13105 products, rows {rows}")
    p = Problem(rows, 819, 13105, STORE, "f32", weights=len(rows), bias=False, seed=len(rows))
    _rms(p, p.run(), 12 * U)


@pytest.mark.parametrize("shape", list(F32))
def test_long_sums_of_float32_in_every_tile_shape(shape):
    bm, bn, _ = F32[shape]
    say(f"precision of float32 sums of 13105 products, shape {shape}")
    p = Problem([bm + 5, 40], 2 * bn + 3, 13105, STORE, "f32", bias=False, seed=shape)
    _rms(p, _launch(p, shape), 12 * U)


@pytest.mark.parametrize("rows", [[67], [300, 21, 700], [2100, 500]], ids=str)
def test_long_sums_of_float32_factors(rows):
    """The adapters' own sums: nothing beside them."""
    say(f"precision of float32 factors, sums of 13105 products, rows {rows}")
    R = len(rows)
    p = Problem(rows, 200, 13105, STORE, "f32", adapter=list(range(R)), rank=16, adapters=R, scales=False, bias=False,
                seed=R)
    p.B.zero_()
    _rms(p, p.run(), 12 * U)


@pytest.mark.parametrize("rows", [[67], [300, 21, 700], [2100]], ids=str)
def test_long_sums_of_bf16_products_in_float32(rows):
    """Rounded after every product: 0.43 u sqrt(13105 / 2) = 34.8 u at most."""
    say(f"precision of bf16 sums of 13105 products, rows {rows}")
    p = Problem(rows, 819, 13105, STORE, "bf16", "f32", bias=False, seed=len(rows))
    _rms(p, p.run(), 36 * U)


def _term_alone(rows, N, types, rank, seed):
    p = Problem(rows, N, 64, STORE, *types, adapter=[i % 2 for i in range(len(rows))], rank=rank, adapters=2,
                scales=False, bias=False, seed=seed)
    p.B.zero_()
    return p


@pytest.mark.parametrize("dtype,out,shape", CASES)
def test_bits_of_the_factor_in_every_tile_shape(dtype, out, shape):
    bm, bn, _ = (F32 if dtype == "f32" else BF16)[shape]
    for rows in ([bm + 5, bm - 3], [1] * 21):
        for rank in (32, 27):
            say(f"precision of the low-rank term, shape={shape} {dtype}->{out} rows={rows[:2]} rank={rank}")
            p = _term_alone(rows, bn + 37, (dtype, out), rank, shape)
            _rms(p, _launch(p, shape, _low(p, 1)), 16 * U if out == "f32" else 0.46 * 2.0 ** -8)


@pytest.mark.parametrize("types", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")], ids="_".join)
@pytest.mark.parametrize("rows", [[64], [1] * 40, [700, 600, 800]], ids=str)
def test_bits_of_the_factor(rows, types):
    say(f"precision of the low-rank term {rows[:3]} {types}")
    p = _term_alone(rows, 300, types, 32, len(rows))
    _rms(p, p.run(), 16 * U if types[1] == "f32" else 0.46 * 2.0 ** -8)
