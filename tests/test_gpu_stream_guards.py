"""Tables that hold anything: nothing beside an operand is written, and where the tables,
limited to the call's sizes, still name rows and tokens, results are those of the limited
tables, bit for bit."""
import math

import pytest
import torch

from paper_2607_06631_amd import binding as B
from tests import stream_ref as R
from tests.gpu_util import say

pytestmark = [pytest.mark.gpu]

BF, F32 = torch.bfloat16, torch.float32
TYPES = pytest.mark.parametrize("dtype", (BF, F32), ids=("bf16", "f32"))
MOST, LEAST = 2 ** 31 - 1, -2 ** 31
GUARD = 4096   # elements on both sides


class Guarded:
    """Tensors in the middle of allocations full of one value."""

    def __init__(self):
        self.all = []

    def put(self, t, fill=5):
        """A copy of t (contiguous) between guards."""
        n = t.numel()
        whole = torch.full((n + 2 * GUARD,), fill, dtype=t.dtype, device="cuda")
        inner = whole[GUARD:GUARD + n].view(t.shape)
        inner.copy_(t)
        self.all.append((whole, n, fill))
        return inner

    def check(self):
        torch.cuda.synchronize()
        for whole, n, fill in self.all:
            assert (whole[:GUARD] == fill).all() and (whole[GUARD + n:] == fill).all()


def _i32(*v):
    return torch.tensor(v, dtype=torch.int32)


# what the tables may hold: (offsets, lengths, their limits for M rows and `most` keys)
WILD = (
    ((-5, 4, MOST), (40, 40), (0, 4, None), (40, 40)),
    ((LEAST, 3, 3), (MOST, -3), (0, 3, 3), (None, 0)),
    ((0, None, None), (LEAST, MOST), (0, None, None), (0, None)),
    ((MOST, MOST, MOST), (40, 40), (None, None, None), (40, 40)),
    ((3, 2, 6), (40, 40), None, None),          # not ascending: undefined rows
    ((MOST, LEAST, 7), (MOST, MOST), None, None),
    ((7, 0, MOST), (LEAST, 1000), None, None),
)


@TYPES
@pytest.mark.parametrize("dh", (64, 128))
@pytest.mark.parametrize("rows,room", ((4, 64), (4, 5000), (150, 400), (150, 4096)))
@pytest.mark.parametrize("mask", ((1, 0, 0), (1, 30, 3), (0, 0, 0), (50, 20, 5)))
def test_attention(dtype, dh, rows, room, mask):
    page, M = 16, 2 * rows
    g = Guarded()
    b = R.Batch([rows, rows], [40 + rows, 40 + rows], 1, dh, page, dtype, max_pages=-(-room // page))
    most = b.table.shape[1] * page
    b.table[b.table < 0] = torch.arange(int((b.table < 0).sum()), dtype=torch.int32) * 7919 - 2 ** 20   # pages anywhere
    b.table[0, 1], b.table[1, 0] = MOST, LEAST
    q = R.padded_rows(b.gen, M, 2, dh, dtype, 0)[0].contiguous()
    ck, cv = g.put(b.k.cuda()), g.put(b.v.cuda())
    table, qg = g.put(b.table.cuda()), g.put(q)
    kw = dict(block=mask[0], window=mask[1], sinks=mask[2])
    for off, lengths, lim_off, lim_len in WILD:
        whole = lambda v, top: _i32(*[top if x is None else x for x in v])
        for ws_on in (False, True):
            say(f"wild {dtype} {dh} rows {rows} room {room} {mask} offsets {off} lengths {lengths} ws {ws_on}")
            ws = g.put(torch.full((B.dif_attention_paged_bytes(dh),), 255, dtype=torch.uint8, device="cuda")) if ws_on else None
            out = g.put(torch.full_like(q, 3.0))
            B.dif_attention_paged(qg, ck, cv, table, g.put(whole(lengths, most)), g.put(whole(off, M)), out, ws=ws, **kw)
            g.check()
            assert torch.equal(ck.cpu(), b.k) and torch.equal(cv.cpu(), b.v)
            if lim_off is not None:
                ref = torch.full_like(q, 3.0)
                pages = table.clamp(0, ck.shape[0] - 1)   # (negative ones are the last)
                pages[table < 0] = ck.shape[0] - 1
                B.dif_attention_paged(qg, ck, cv, pages, whole(lim_len, most).cuda(), whole(lim_off, M).cuda(), ref, ws=ws, **kw)
                torch.cuda.synchronize()
                assert torch.equal(out.cpu(), ref.cpu())
            del g.all[-3 - ws_on:]


@TYPES
@pytest.mark.parametrize("dh", (64, 128))
@pytest.mark.parametrize("rows,keys", ((4, 60), (150, 300), (150, 2100)))
def test_packed_attention(dtype, dh, rows, keys):
    M = 2 * rows
    g = Guarded()
    gen = torch.Generator().manual_seed(4)
    q, k, v = (g.put(R.padded_rows(gen, n, h, dh, dtype, 0)[0].contiguous()) for n, h in ((M, 2), (keys, 1), (keys, 1)))
    wild = ((-5, 4, MOST), (LEAST, 3, 3), (MOST, MOST, MOST), (3, 2, 6), (MOST, LEAST, 7), (7, 0, MOST))
    for off in wild:
        for koff in wild:
            say(f"wild packed {dtype} {dh} rows {rows} keys {keys} {off} {koff}")
            out = g.put(torch.full_like(q, 3.0))
            B.dif_attention_window(q, k, v, g.put(_i32(*off)), out, key_offsets=g.put(_i32(*koff)))
            g.check()
            if list(off) == sorted(off) and list(koff) == sorted(koff):
                ref = torch.full_like(q, 3.0)
                cut = lambda o, n: _i32(*[min(max(x, 0), n) for x in o]).cuda()
                B.dif_attention_window(q, k, v, cut(off, M), ref, key_offsets=cut(koff, keys))
                torch.cuda.synchronize()
                assert torch.equal(out.cpu(), ref.cpu())
            del g.all[-3:]


@TYPES
@pytest.mark.parametrize("dh", (64, 128))
def test_append(dtype, dh):
    page, M, H, KV = 16, 8, 4, 2
    b = R.Batch([4, 4], [40, 40], KV, dh, page, dtype, max_pages=4)
    b.table[b.table < 0] = torch.tensor([LEAST, MOST], dtype=torch.int32)
    b.table[1, 1] = b.k.shape[0]
    q, k, v = (R.padded_rows(b.gen, M, h, dh, dtype, 0)[0].contiguous() for h in (H, KV, KV))
    most = 4 * page
    for off, lengths, lim_off, lim_len in WILD + (((0, 4, 8), (MOST, 2), (0, 4, 8), (MOST, 2)),):
        whole = lambda t, top: _i32(*[top if x is None else x for x in t])
        say(f"wild append {dtype} {dh} offsets {off} lengths {lengths}")
        g = Guarded()
        ck, cv, qo = g.put(b.k.cuda()), g.put(b.v.cuda()), g.put(torch.full_like(q, 3.0))
        o, n = whole(off, M), whole(lengths, most)
        B.dif_cache_append(ck, cv, g.put(b.table.cuda()), g.put(n), g.put(o), g.put(k), g.put(v), q=g.put(q), q_out=qo)
        g.check()
        if lim_off is None:
            continue
        wk, wv, wq = b.k.clone(), b.v.clone(), torch.full_like(q.cpu(), 3.0)
        lo, n = whole(lim_off, M).tolist(), n.tolist()   # (indexes count from the length as it is)
        for s in range(2):
            for r in range(lo[s], lo[s + 1]):
                wq[r] = q[r].cpu()
                at = n[s] - (lo[s + 1] - r)
                if 0 <= at < most and 0 <= int(b.table[s, at // page]) < b.k.shape[0]:
                    wk[b.table[s, at // page], :, at % page] = k[r].cpu()
                    wv[b.table[s, at // page], :, at % page] = v[r].cpu()
        assert torch.equal(ck.cpu(), wk) and torch.equal(cv.cpu(), wv) and torch.equal(qo.cpu(), wq)
