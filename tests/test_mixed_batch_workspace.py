"""dif_lora_workspace_bytes: what one batch asks for serves every smaller one."""
import pytest

from paper_2607_06631_amd import binding as B

# around the row counts at which the down product takes fewer parts, and far from them
ROWS = sorted({0, 1, 2, 3, 7, 31, 4095, 4096, 8191, 8192, 8193, 40000, 1 << 20} |
              {m + d for m in (64, 128, 256, 512, 1024, 2048) for d in (-1, 0, 1)})


@pytest.mark.parametrize("rank", [1, 8, 9, 16, 17, 100, 1024])
def test_never_less_for_more_rows(rank):
    sizes = [B.dif_lora_workspace_bytes(m, rank) for m in ROWS]
    assert sizes == sorted(sizes), [x for x in zip(ROWS, sizes)]


@pytest.mark.parametrize("rows", ROWS)
def test_never_less_for_a_larger_rank(rows):
    sizes = [B.dif_lora_workspace_bytes(rows, r) for r in range(1, 1025)]
    assert sizes == sorted(sizes)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 100, 128, 500, 512, 513, 2048], ids=str)
def test_a_workspace_of_the_largest_batch_serves_smaller_ones(rows):
    """Its bits are those of a call with a workspace of its own size."""
    import torch

    from tests.gpu_util import say
    from tests.mixed_batch import Problem
    say(f"lora, {rows} rows in a workspace for 2049")
    p = Problem([rows], 96, 640, adapter=[0], rank=16, adapters=1, seed=rows)
    ws = torch.full((B.dif_lora_workspace_bytes(2049, 16),), 255, dtype=torch.uint8, device="cuda")
    C = p.run(ws=ws)
    p.check(C)
    assert torch.equal(C, p.run())
