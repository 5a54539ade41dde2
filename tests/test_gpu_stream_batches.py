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


def _laid_out(t, how):
    """The cache t [pages, heads, page, dh] in memory as `how` says, for keys and values alike."""
    p, h, s, d = t[0].shape
    if how == "nhd":            # a page's tokens, then heads
        return [x.transpose(1, 2).contiguous().cuda().transpose(1, 2) for x in t]
    if how == "beside":         # keys and values of a token beside each other, heads 8 elements apart
        both = torch.full((p, s, 2, h, d + 8), math.nan, dtype=t[0].dtype, device="cuda")
        out = [both[:, :, i, :, :d].transpose(1, 2) for i in (0, 1)]
    elif how == "heads first":  # a pool for each head
        both = torch.full((2, h, p + 1, s, d), math.nan, dtype=t[0].dtype, device="cuda")
        out = [both[i, :, 1:].transpose(0, 1) for i in (0, 1)]
    elif how == "apart":        # room behind tokens, heads and pages
        both = torch.full((2, p, h + 1, s + 3, d + 16), math.nan, dtype=t[0].dtype, device="cuda")
        out = [both[i, :, :h, :s, :d] for i in (0, 1)]
    for x, y in zip(out, t):
        x.copy_(y)
    return out


@pytest.mark.parametrize("dtype,dh,rows,lengths,room", (
    (BF, 128, [257, 130], [700, 300], 4096), (BF, 128, [257, 130], [700, 300], 0), (BF, 64, [140, 33, 1], [500, 90, 70], 0),
    (F32, 128, [140, 33, 1], [300, 90, 70], 0), (F32, 64, [140, 33, 1], [300, 90, 70], 0), (BF, 128, [1, 3, 1], [700, 90, 1], 0),
    (BF, 64, [1, 3, 1], [1700, 90, 1], 0), (F32, 128, [1, 3, 1], [700, 90, 1], 0), (F32, 64, [1, 3, 1], [1700, 90, 1], 0)))
@pytest.mark.parametrize("how", ("nhd", "beside", "heads first", "apart"))
@pytest.mark.parametrize("page,mask", ((16, (1, 0, 0)), (64, (1, 60, 5)), (32, (50, 20, 5)), (16, (0, 0, 0))))
def test_layouts(dtype, dh, rows, lengths, room, how, page, mask):
    """Every kernel, with what lies between the tokens full of NaN."""
    say(f"layout {how} {dtype} {dh} {rows} {lengths} room {room} page {page} {mask}")
    b = R.Batch(rows, lengths, 3, dh, page, dtype, fill=math.nan, max_pages=room // page or None)
    q, q0 = R.padded_rows(b.gen, sum(rows), 6, dh, dtype, 8)
    want, tol, r0 = [], [], 0
    for i, r in enumerate(rows):
        o, t = R.attend(q0[r0:r0 + r], b.keys(b.k, i), b.keys(b.v, i), R.seen(*mask, r, lengths[i]), dh ** -0.5, dtype)
        want.append(o)
        tol.append(t)
        r0 += r
    want, tol = torch.cat(want), torch.cat(tol)
    k, v = _laid_out((b.k, b.v), how)
    assert k.stride() == v.stride()
    for ws in (None, torch.full((B.dif_attention_paged_bytes(dh),), 255, dtype=torch.uint8, device="cuda")):
        out = torch.full_like(q, 3.0)
        B.dif_attention_paged(q, k, v, *b.cuda()[2:], out, block=mask[0], window=mask[1], sinks=mask[2], ws=ws)
        assert ((out.double().cpu() - want).abs() <= tol).all()


@TYPES
@pytest.mark.parametrize("dh", (64, 128))
def test_a_chunk_among_empty_slots(dtype, dh):
    """No more rows than sequences, nearly all of one sequence: taken for single tokens."""
    n = 1200
    rows = [0] * n
    rows[700], rows[3], rows[1199] = 1000, 1, 40
    paged(rows, [max(r, i % 3) for i, r in enumerate(rows)], 2, 2, dh, 16, dtype, behind=2)
    paged(rows, [max(r, 0) for r in rows], 4, 1, dh, 64, dtype, block=100, window=300, sinks=4)


@TYPES
@pytest.mark.parametrize("rows,lengths", (([1], [5003]), ([30], [5003]), ([1, 0, 2], [5003, 9, 3000])))
def test_few_rows_of_a_call_for_many(dtype, rows, lengths):
    """Room for rows behind the last sequence decides the kernel, and that nothing is split."""
    paged(rows, lengths, 2, 2, 64, 16, dtype, behind=5000)
    paged(rows, lengths, 2, 1, 128, 64, dtype, window=2000, sinks=70, behind=9000)


@TYPES
@pytest.mark.parametrize("at", (0, 64, 149))
def test_one_long_cache_beside_many_short_ones(dtype, at):
    lengths = [17 + i for i in range(150)]
    lengths[at] = 20011
    paged([1] * 150, lengths, 8, 8, 64, 16, dtype)


@TYPES
@pytest.mark.parametrize("streams,kv", ((127, 8), (128, 8), (150, 8), (250, 5)))
def test_one_long_cache_among_many_is_split(dtype, streams, kv):
    """On both sides of 1024 items: the workspace holds its pieces' sums."""
    dh, long = 64, 20011
    lengths = [17 + i % 100 for i in range(streams)]
    lengths[streams // 2] = long
    say(f"one long cache among {streams} {dtype}")
    b = R.Batch([1] * streams, lengths, kv, dh, 16, dtype)
    q, q0 = R.padded_rows(b.gen, streams, kv, dh, dtype, 0)
    ws = torch.full((B.dif_attention_paged_bytes(dh),), 255, dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(q)
    B.dif_attention_paged(q, *b.cuda(), out, ws=ws)
    assert int((ws != 255).sum()) > 20 * kv * dh * 4
    i = streams // 2
    want, tol = R.attend(q0[i:i + 1], b.keys(b.k, i), b.keys(b.v, i), R.seen(1, 0, 0, 1, long), dh ** -0.5, dtype)
    assert ((out[i:i + 1].double().cpu() - want).abs() <= tol).all()
