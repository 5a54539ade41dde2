"""Streamed attention over batches of other kinds than its other tests: more items than 1024
(the launch then orders its workgroups in bands), cache layouts in every kernel, calls whose
tables hold much less or something else than their sizes allow."""
import math

import pytest
import torch

from paper_2607_06631_amd import binding as B
from tests import stream_ref as R
from tests.gpu_util import say
from tests.test_gpu_stream_attention import packed, paged

pytestmark = [pytest.mark.gpu]

BF, F32 = torch.bfloat16, torch.float32
TYPES = pytest.mark.parametrize("dtype", (BF, F32), ids=("bf16", "f32"))


@pytest.mark.parametrize("dtype,dh,room", ((BF, 128, 4096), (BF, 128, 0), (BF, 64, 0), (F32, 128, 0), (F32, 64, 0)))
@pytest.mark.parametrize("heads,kv", ((13, 13), (26, 13)))
def test_more_than_1024_items(dtype, dh, room, heads, kv):
    """Row tiles of many sequences (81 and more of 256 rows times 13 key heads), then of one."""
    rows = [300 - i % 7 for i in range(45)]
    paged(rows, [90 + i for i in range(45)], heads, kv, dh, 16, dtype, block=40, behind=3, room=room)
    paged([20700 // (heads // kv) + 5], [77], heads, kv, dh, 16, dtype, block=0, behind=3, room=room)


def test_more_than_1024_packed_items():
    rows = [300 - i % 7 for i in range(45)]
    packed(rows, [90 + i for i in range(45)], 26, 13, 128, BF, block=40, behind=3)
    packed([20705], [77], 13, 13, 64, F32, block=0, behind=3)
