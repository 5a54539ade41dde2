"""The binding's refusal of mixed-batch calls without their tables."""
import pytest

from paper_2607_06631_amd import binding as B


def test_adapters_without_tables_are_refused():
    import torch
    t = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    off, which = torch.tensor([0, 4], dtype=torch.int32), torch.tensor([0], dtype=torch.int32)
    call = lambda row_offsets, adapter: B.dif_gemm_lora(t(4, 64), t(32, 64), t(4, 32), row_offsets, adapter,
                                                        t(1, 8, 64), t(1, 32, 8), None)
    for bad in (None, torch.tensor(4, dtype=torch.int32)):
        with pytest.raises(ValueError, match="row_offsets"):
            call(bad, which)
    with pytest.raises(ValueError, match="adapter"):
        call(off, None)
    with pytest.raises(ValueError, match="device memory"):
        call(off, which)


def test_groups_without_a_table_of_rows_are_refused():
    import torch
    t = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    for bad in (None, torch.tensor(4, dtype=torch.int32)):
        with pytest.raises(ValueError, match="row_offsets"):
            B.dif_gemm_grouped(t(4, 64), t(1, 32, 64), t(4, 32), bad)
