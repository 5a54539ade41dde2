"""dif_gemm_grouped and dif_gemm_lora through the C ABI against float64, entry by
entry within a bound that counts roundings (tests/mixed_batch.py)."""
import pytest

from tests.gpu_util import say
from tests.mixed_batch import GELU, RESIDUAL, STORE, Problem

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]

# (rows of the groups, N, K, more)
GROUPED = {
    "one_row": ([1], 1, 1, {}),
    "one_row_wide": ([1], 700, 512, {}),
    "single_rows": ([1, 0, 1, 1, 0, 0, 1], 320, 640, {}),
    "empty": ([0, 0, 0], 64, 64, dict(behind=5)),
    "k_zero": ([3, 5], 40, 0, {}),
    "odd": ([37, 1, 64, 0, 129], 77, 203, dict(behind=3, pad=24)),
    "k_below_a_tile": ([17, 40], 65, 24, {}),
    "k_ends_in_a_chunk": ([17, 40], 65, 129, {}),
    "shared_matrices": ([50, 7, 33, 64], 130, 192, dict(weights=2, index=[1, 0, 1, 1])),
    "bad_index": ([10, 20, 30], 48, 64, dict(weights=2, index=[0, -1, 2])),
    "kept": ([65, 65, 65, 65], 192, 320, dict(n_kept=[192, 1, 0, 101], k_kept=[320, 7, 64, 0])),
    "kept_beyond": ([9, 9], 33, 64, dict(n_kept=[99, -4], k_kept=[-1, 1 << 30])),
    "before_and_behind": ([100, 28], 96, 128, dict(before=11, behind=40)),
    "many_groups": ([(i * 7) % 4 for i in range(200)], 72, 96, dict(weights=5, index=[i % 5 for i in range(200)])),
    "tall": ([1500, 3, 997], 256, 256, {}),
    "wide": ([60, 200], 2100, 576, {}),
    "large_tiles": ([2100, 1999], 1280, 704, dict(pad=8)),
    "long_reduction": ([120, 33], 260, 4160, dict(k_kept=[4160, 4099])),
}


@pytest.mark.parametrize("types", TYPES, ids="_".join)
@pytest.mark.parametrize("epilogue", [STORE, GELU, RESIDUAL])
@pytest.mark.parametrize("case", GROUPED)
def test_grouped(case, epilogue, types):
    rows, N, K, more = GROUPED[case]
    say(f"grouped {case} epilogue={epilogue} {types}")
    p = Problem(rows, N, K, epilogue, *types, seed=len(case), **more)
    p.check(p.run())


# (rows of the requests, N, K, adapters of the requests, rank, adapters, more)
LORA = {
    "one_row": ([1], 5, 8, [0], 1, 1, {}),
    "single_rows": ([1] * 9, 320, 640, [3, 0, 1, -1, 2, 2, 0, 7, 1], 16, 4, {}),
    "no_adapters": ([5, 9], 64, 128, [-1, -1], 8, 2, {}),
    "none_at_all": ([5, 9], 64, 128, [0, 0], 8, 0, {}),
    "empty_requests": ([0, 4, 0, 0, 60, 0], 70, 96, [0, 1, 0, 2, 0, 1], 8, 3, {}),
    "odd": ([37, 1, 64, 0, 129], 77, 203, [0, 2, -1, 1, 2], 7, 3, dict(ranks=[7, 3, 5], behind=3, pad=24)),
    "ranks_to_zero": ([40, 40, 40], 80, 64, [0, 1, 2], 33, 3, dict(ranks=[0, -3, 400])),
    "rank_over_a_tile": ([40, 90], 130, 128, [1, 0], 100, 2, {}),
    "rank_200": ([200, 61], 256, 192, [0, 1], 200, 2, dict(ranks=[199, 65])),
    "no_scales": ([33, 20], 48, 64, [0, 1], 12, 2, dict(scales=False)),
    "k_zero": ([3, 5], 40, 0, [0, 1], 4, 2, {}),
    "before_and_behind": ([100, 28], 96, 128, [0, 1], 8, 2, dict(before=11, behind=40)),
    "many_requests": ([(i * 5) % 3 for i in range(300)], 72, 96, [i % 7 - 1 for i in range(300)], 8, 6, {}),
    "neighbours_share": ([10, 10, 10, 10, 10], 64, 64, [1, 1, 0, 0, 1], 8, 2, {}),
    "grouped_base": ([50, 7, 33, 64], 130, 192, [0, 1, 1, -1], 16, 2,
                     dict(groups=[30, 60, 64], weights=2, index=[1, 0, 1], n_kept=[130, 77])),
    "groups_end_early": ([50, 30], 65, 64, [0, 1], 8, 2, dict(groups=[20, 30], weights=2)),
    "large_tiles": ([2100, 1, 1998], 1280, 704, [1, 0, 1], 40, 2, dict(pad=8)),
    "wide": ([60, 200], 2100, 576, [0, 1], 64, 2, {}),
}


@pytest.mark.parametrize("types", TYPES, ids="_".join)
@pytest.mark.parametrize("epilogue", [STORE, GELU, RESIDUAL])
@pytest.mark.parametrize("case", LORA)
def test_lora(case, epilogue, types):
    rows, N, K, adapter, rank, adapters, more = LORA[case]
    say(f"lora {case} epilogue={epilogue} {types}")
    p = Problem(rows, N, K, epilogue, *types, adapter=adapter, rank=rank, adapters=adapters, seed=len(case), **more)
    p.check(p.run())
