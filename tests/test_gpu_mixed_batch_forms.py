"""Forms of the mixed-batch calls beside the usual ones: residuals without gates, with
the layer's gate alone or a gate that all matrices share; kept widths and adapters in
one call, whose runs of rows cross each other.  References as in tests/mixed_batch.py."""
import pytest

from tests.gpu_util import say
from tests.mixed_batch import GELU, RESIDUAL, STORE, Problem
from tests.test_gpu_mixed_batch import TYPES
from tests.test_gpu_mixed_batch_tiles import CASES, _launch, _low
from tests.test_gpu_gemm_instances import BF16, F32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("types", TYPES, ids="_".join)
@pytest.mark.parametrize("gates", [0, 1])
@pytest.mark.parametrize("rows", [[1, 1, 1, 1], [60, 0, 7, 130], [700, 1, 1500, 99]], ids=str)
def test_residuals_of_fewer_gates(rows, gates, types):
    say(f"residual with {gates} gates, rows {rows} {types}")
    p = Problem(rows, 261, 200, RESIDUAL, *types, gates=gates, seed=gates, behind=3)
    p.check(p.run())
    q = Problem(rows, 261, 200, RESIDUAL, *types, gates=gates, adapter=[0, -1, 1, 0], rank=11, adapters=2, seed=gates)
    q.check(q.run())


@pytest.mark.parametrize("types", TYPES, ids="_".join)
def test_a_gate_and_a_bias_that_all_matrices_share(types):
    say(f"shared gate1 and bias {types}")
    p = Problem([60, 0, 7, 130], 261, 200, RESIDUAL, *types, seed=1)
    q = Problem([60, 0, 7, 130], 261, 200, RESIDUAL, *types, adapter=[0, -1, 1, 0], rank=11, adapters=2,
                groups=[67, 130], weights=2, seed=2)
    for x in (p, q):
        x.gate1[:] = x.gate1[0].clone()
        x.bias[:] = x.bias[0].clone()
        x.check(x.run(gate1=x.gate1[0].clone(), bias=x.bias[0].clone()))


@pytest.mark.parametrize("types", TYPES, ids="_".join)
def test_gates_and_biases_whose_rows_lie_apart(types):
    import torch
    say(f"gate1 and bias with gaps {types}")
    p = Problem([60, 0, 7, 130], 261, 200, RESIDUAL, *types, seed=3)
    room = torch.full((2, p.W, p.N + 5), float("nan"), device="cuda")
    room[0, :, :p.N], room[1, :, :p.N] = p.gate1, p.bias
    p.check(p.run(gate1=room[0, :, :p.N], bias=room[1, :, :p.N]))


# (rows of the requests, adapters, rows of the groups, matrices, kept columns)
BOTH = {
    "runs_cross_groups": ([50, 7, 33, 64], [0, 1, 1, -1], [30, 60, 64], [1, 0, 1], [130, 77]),
    "single_rows": ([1] * 40, [i % 4 - 1 for i in range(40)], [13, 1, 26], [0, 1, 0], [101, 17]),
    "nothing_kept": ([20, 20, 20], [0, 1, 2], [25, 10, 25], [0, 1, 0], [0, 130]),
    "bad_index": ([20, 20, 20], [0, 7, 2], [25, 10, 25], [0, 2, -1], [64, 130]),
    "groups_end_early": ([15, 30, 15], [2, 0, 1], [20, 20], [1, 0], [129, 64]),
    "empty_ones": ([0, 33, 0, 0, 40, 0], [0, 1, 2, -1, 0, 1], [0, 50, 0, 23, 0], [0, 1, 1, 0, 0], [130, 99]),
    "stills": ([1560, 390, 1, 900], [0, 1, 2, 0], [1560, 391, 900], [1, 0, 1], [130, 101]),
    "many": ([3] * 150, [i % 5 - 1 for i in range(150)], [i % 7 for i in range(150)], [i % 2 for i in range(150)],
             [130, 33]),
}


@pytest.mark.parametrize("types", TYPES, ids="_".join)
@pytest.mark.parametrize("epilogue", [STORE, GELU, RESIDUAL])
@pytest.mark.parametrize("case", BOTH)
def test_kept_widths_beside_adapters(case, epilogue, types):
    rows, adapter, groups, index, kept = BOTH[case]
    say(f"kept widths and adapters, {case} epilogue={epilogue} {types}")
    p = Problem(rows, 130, 192, epilogue, *types, adapter=adapter, rank=24, adapters=3, ranks=[24, 5, 17], groups=groups,
                weights=2, index=index, n_kept=kept, seed=len(case), behind=3)
    p.check(p.run())


@pytest.mark.parametrize("dtype,out,shape", CASES)
def test_kept_widths_beside_adapters_in_every_tile_shape(dtype, out, shape):
    bm, bn, _ = (F32 if dtype == "f32" else BF16)[shape]
    for n, (rows, groups) in enumerate((([bm + 5, 3, 2 * bm - 1], [bm, 2 * bm + 7]), ([1] * 21, [9, 12]),
                                        ([2 * bm, bm], [bm + 1, 2 * bm - 1]))):
        N = bn + 37
        say(f"kept widths and adapters, shape={shape} {dtype}->{out} rows={rows[:3]}")
        p = Problem(rows, N, 160, (STORE, GELU, RESIDUAL)[n], dtype, out, adapter=[i % 3 for i in range(len(rows))],
                    rank=20, adapters=3, ranks=[20, 0, 9], groups=groups, weights=2, index=[1, 0],
                    n_kept=[bn - 3, N - 2], seed=shape + n)
        p.check(_launch(p, shape, _low(p, 1 + n)))
