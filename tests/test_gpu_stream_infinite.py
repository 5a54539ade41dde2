"""Infinite values at tokens that rows see, against the definition: the infinity of their
sign, since a probability is above zero, and NaN where both signs meet.  Entries of other
dims and rows that do not see the token are as if it were not there."""
import math

import pytest
import torch

from paper_2607_06631_amd import binding as B
from tests import stream_ref as R
from tests.gpu_util import say

pytestmark = [pytest.mark.gpu]

BF, F32 = torch.bfloat16, torch.float32
TYPES = pytest.mark.parametrize("dtype", (BF, F32), ids=("bf16", "f32"))


def _run(rows, lengths, kv, group, dh, page, dtype, hits, block=1, window=0, sinks=0, room=0, seed=5):
    """hits: (sequence, token, +1 / -1 / 0), 0 an infinity of each sign in neighbouring dims."""
    say(f"infinite {rows[:4]} {lengths[:4]} {kv * group}/{kv}x{dh} page {page} {dtype} {hits} block {block} window {window} "
        f"sinks {sinks} room {room}")
    b = R.Batch(rows, lengths, kv, dh, page, dtype, seed=seed, max_pages=room // page or None)
    q, q0 = R.padded_rows(b.gen, sum(rows), kv * group, dh, dtype, 0, 0.5)
    v = b.v.clone()
    for i, j, sign in hits:
        pg, sl = b.place(i, j)
        v[pg, :, sl, 3::7] = sign * math.inf if sign else math.inf
        if not sign:
            v[pg, :, sl, 4::7] = -math.inf
    want, tol, r0 = [], [], 0
    for i, r in enumerate(rows):
        mask = R.seen(block, window, sinks, r, lengths[i])
        o, t = R.attend(q0[r0:r0 + r], b.keys(b.k, i), b.keys(b.v, i), mask, dh ** -0.5, dtype)
        vals = b.keys(v, i).double()
        for h in range(kv):   # the infinities that a row sees, with a probability above zero
            inf = torch.where(vals[:, h].isinf(), vals[:, h], 0.0)
            up = (mask.double() @ (inf > 0).double()) > 0
            down = (mask.double() @ (inf < 0).double()) > 0
            add = torch.where(up & down, math.nan, torch.where(up, math.inf, torch.where(down, -math.inf, 0.0)))
            o[:, h * group:(h + 1) * group] += add[:, None]
        want.append(o)
        tol.append(t)
        r0 += r
    want, tol = torch.cat(want), torch.cat(tol)
    assert not want.isfinite().all()
    dev = list(b.cuda())
    dev[1] = v.cuda()
    for ws in (None, torch.full((B.dif_attention_paged_bytes(dh),), 255, dtype=torch.uint8, device="cuda")):
        out = torch.zeros_like(q)
        B.dif_attention_paged(q, *dev, out, block=block, window=window, sinks=sinks, ws=ws)
        got = out.double().cpu()
        assert torch.equal(got.isnan(), want.isnan())
        assert torch.equal(torch.where(got.isinf(), got, 0.0), torch.where(want.isinf(), want, 0.0))
        fin = want.isfinite()
        assert ((got[fin] - want[fin]).abs() <= tol[fin]).all()


@TYPES
@pytest.mark.parametrize("dh", (64, 128))
@pytest.mark.parametrize("sign", (1, -1, 0))
def test_single_tokens(dtype, dh, sign):
    """In a whole tile, the last token of a tail, the only token."""
    _run([1, 1, 1], [100, 70, 1], 2, 2, dh, 16, dtype, [(0, 20, sign), (1, 69, sign), (2, 0, sign)])


@TYPES
@pytest.mark.parametrize("group", (1, 4, 16))
def test_every_place_of_a_tile(dtype, group):
    """A sequence for each token of two tiles, the second with a tail."""
    n = 45
    _run([1] * n, [n] * n, 1, group, 64, 16, dtype, [(i, i, 1 if i % 2 else -1) for i in range(n)])


@TYPES
def test_both_signs_in_one_dim(dtype):
    _run([1, 2], [90, 90], 1, 3, 64, 16, dtype, [(0, 3, 1), (0, 88, -1), (1, 4, 1), (1, 5, -1)])


@TYPES
@pytest.mark.parametrize("window,sinks", ((20, 0), (20, 5), (64, 33), (40, 100)))
def test_windows(dtype, window, sinks):
    """First and last tokens of the window and of the sinks."""
    n = 300
    hits = [n - window, n - 1] + ([0, sinks - 1] if sinks else [])
    _run([1] * len(hits), [n] * len(hits), 2, 4, 64, 16, dtype, [(i, j, 1) for i, j in enumerate(hits)], window=window,
         sinks=sinks)


@TYPES
@pytest.mark.parametrize("dh", (64, 128))
def test_split_caches(dtype, dh):
    _run([1], [5003], 2, 2, dh, 16, dtype, [(0, 5002, -1)])
    _run([1, 2], [5003, 3001], 2, 2, dh, 64, dtype, [(0, 17, 1), (1, 2990, -1), (1, 3000, 1)])


@TYPES
def test_few_rows_that_see_different_tokens(dtype):
    _run([12], [90], 2, 1, 64, 16, dtype, [(0, 85, 1)])
    _run([12], [90], 2, 1, 64, 16, dtype, [(0, 89, 1)])
    _run([5], [90], 2, 3, 128, 16, dtype, [(0, 66, 1), (0, 87, -1)], window=20)


@TYPES
@pytest.mark.parametrize("dh", (64, 128))
@pytest.mark.parametrize("room", (0, 4096))
def test_chunks(dtype, dh, room):
    _run([300], [800], 1, 1, dh, 16, dtype, [(0, 120, 1), (0, 700, -1), (0, 799, 1)], room=room)
    _run([300], [813], 1, 2, dh, 16, dtype, [(0, 10, 1), (0, 560, -1), (0, 812, 1)], block=0, room=room)
    _run([300, 40], [800, 70], 2, 1, dh, 16, dtype, [(0, 2, -1), (0, 600, 1), (1, 69, 1)], block=50, window=130, sinks=4,
         room=room)


@TYPES
@pytest.mark.parametrize("dh", (64, 128))
@pytest.mark.parametrize("rows,room", ((1, 0), (1, 4096), (300, 0), (300, 4096)))
def test_small_probabilities(dtype, dh, rows, room):
    """An infinity whose token has 2^-86 of the others' probability."""
    say(f"small probabilities {dtype} {dh} {rows} {room}")
    n, page = 500, 16
    b = R.Batch([rows], [n], 1, dh, page, dtype, max_pages=room // page or None)
    b.k *= 0.01
    pg, sl = b.place(0, 100)
    b.k[pg, :, sl] = -240 / dh ** 0.5          # a score of -60
    b.v[pg, :, sl, 3] = -math.inf
    q = torch.full((rows, 2, dh), 0.25, dtype=dtype, device="cuda")
    out = torch.zeros_like(q)
    B.dif_attention_paged(q, *b.cuda(), out)
    want, tol = R.attend(q.cpu(), b.keys(b.k, 0), b.keys(b.v, 0), R.seen(1, 0, 0, rows, n), dh ** -0.5, dtype)
    got = out.double().cpu()
    assert (got[..., 3] == -math.inf).all()
    rest = [i for i in range(dh) if i != 3]
    assert ((got - want).abs() <= tol)[..., rest].all()


@TYPES
@pytest.mark.parametrize("dh", (64, 128))
@pytest.mark.parametrize("rows,room", ((1, 0), (1, 5008), (300, 0), (300, 4096)))
def test_scores_of_minus_infinity(dtype, dh, rows, room):
    """They count for nothing beside others; a row that has no others is 0."""
    say(f"minus infinity {dtype} {dh} {rows} {room}")
    n, page = max(500, room - 1000 if rows == 1 else 500), 16
    b = R.Batch([rows], [n], 2, dh, page, dtype, max_pages=room // page or None)
    for j in range(n):
        pg, sl = b.place(0, j)
        b.k[pg, 0 if j % 3 else slice(None), sl, 5] = -math.inf   # head 0: every key, head 1: each third
    q, q0 = R.padded_rows(b.gen, rows, 2, dh, dtype, 0)
    q[:, :, 5], q0[:, :, 5] = 0.5, 0.5
    mask = R.seen(1, 0, 0, rows, n)
    mask[:, ::3] = False
    kept = b.keys(b.k, 0).clone()
    kept[:, 0] = 0.0
    want, tol = R.attend(q0, kept, b.keys(b.v, 0), mask, dh ** -0.5, dtype)
    want[:, 0] = tol[:, 0] = 0.0
    for ws in (None, torch.full((B.dif_attention_paged_bytes(dh),), 255, dtype=torch.uint8, device="cuda")):
        out = torch.full_like(q, 3.0)
        B.dif_attention_paged(q, *b.cuda(), out, ws=ws)
        assert ((out.double().cpu() - want).abs() <= tol).all()
