"""dif_attention_paged and dif_attention_window against float64."""
import math

import pytest
import torch

from paper_2607_06631_amd import binding as B
from tests import stream_ref as R
from tests.gpu_util import say

pytestmark = [pytest.mark.gpu]

BF, F32 = torch.bfloat16, torch.float32
TYPES = pytest.mark.parametrize("dtype", (BF, F32), ids=("bf16", "f32"))


def _ws(dh):
    return torch.full((B.dif_attention_paged_bytes(dh),), 255, dtype=torch.uint8, device="cuda")   # (NaNs)


def _check(out, want, tol, left, name):
    m = want.shape[0]
    got = out[:m].double().cpu()
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (f"{name}: {int(bad.sum())} of {bad.numel()} off, worst "
                           f"{float((got - want).abs().max()):.3e}, first {bad.nonzero()[0].tolist()}")
    assert torch.equal(out[m:].cpu(), left[m:]), f"{name}: rows behind the last sequence"


def paged(rows, lengths, heads, kv, dh, page, dtype, block=1, window=0, sinks=0, layout="hnd", pad=0, behind=0,
          scaled=False, fill=None, std=1.0, seed=1, change=None, split=True, room=0):
    say(f"paged {rows[:6]} {lengths[:6]} {heads}/{kv}x{dh} page {page} {dtype} block {block} window {window} sinks {sinks} "
        f"room {room}")
    b = R.Batch(rows, lengths, kv, dh, page, dtype, layout, fill=fill, seed=seed, max_pages=room // page or None)
    if change:
        change(b)
    scale = math.log(2.0) if scaled else dh ** -0.5
    q, q0 = R.padded_rows(b.gen, sum(rows) + behind, heads, dh, dtype, pad, std * (R.LOG2E * dh ** -0.5 if scaled else 1.0))
    want, tol, r0 = [], [], 0
    for i, r in enumerate(rows):
        o, t = R.attend(q0[r0:r0 + r], b.keys(b.k, i), b.keys(b.v, i), R.seen(block, window, sinks, r, lengths[i]), scale, dtype)
        want.append(o)
        tol.append(t)
        r0 += r
    left = torch.full((r0 + behind, heads, dh), 3.0, dtype=dtype)
    dev = b.cuda()
    for ws in (None, _ws(dh)) if split else (None,):
        out = left.cuda()
        B.dif_attention_paged(q, *dev, out, block=block, window=window, sinks=sinks,
                              flags=B.DIF_ATTN_Q_PRESCALED if scaled else 0, ws=ws)
        torch.cuda.synchronize()
        _check(out, torch.cat(want), torch.cat(tol), left, "split" if ws is not None else "whole")


def packed(rows, lengths, heads, kv, dh, dtype, block=1, window=0, sinks=0, pad=0, behind=0, scaled=False, seed=1):
    say(f"packed {rows[:6]} {lengths[:6]} {heads}/{kv}x{dh} {dtype} block {block} window {window} sinks {sinks}")
    gen = torch.Generator().manual_seed(seed)
    scale = math.log(2.0) if scaled else dh ** -0.5
    q, q0 = R.padded_rows(gen, sum(rows) + behind, heads, dh, dtype, pad, R.LOG2E * dh ** -0.5 if scaled else 1.0)
    k, k0 = R.padded_rows(gen, sum(lengths) + behind, kv, dh, dtype, pad)
    v, v0 = R.padded_rows(gen, sum(lengths) + behind, kv, dh, dtype, 2 * pad)
    want, tol, r0, n0 = [], [], 0, 0
    for r, n in zip(rows, lengths):
        o, t = R.attend(q0[r0:r0 + r], k0[n0:n0 + n], v0[n0:n0 + n], R.seen(block, window, sinks, r, n), scale, dtype)
        want.append(o)
        tol.append(t)
        r0, n0 = r0 + r, n0 + n
    offsets = lambda c: torch.tensor([sum(c[:i]) for i in range(len(c) + 1)], dtype=torch.int32).cuda()
    left = torch.full((r0 + behind, heads, dh), 3.0, dtype=dtype)
    same = rows == lengths and not behind
    for ws in (None, _ws(dh)):
        out = left.cuda()
        B.dif_attention_window(q, k, v, offsets(rows), out, key_offsets=None if same else offsets(lengths), block=block,
                               window=window, sinks=sinks, flags=B.DIF_ATTN_Q_PRESCALED if scaled else 0, ws=ws)
        torch.cuda.synchronize()
        _check(out, torch.cat(want), torch.cat(tol), left, "split" if ws is not None else "whole")


@TYPES
@pytest.mark.parametrize("dh", (64, 128))
@pytest.mark.parametrize("layout", ("hnd", "nhd"))
def test_single_tokens(dtype, dh, layout):
    paged([1, 1, 1, 0, 1], [1, 16, 257, 5, 700], 4, 2, dh, 16, dtype, layout=layout, pad=8, behind=2)


@TYPES
@pytest.mark.parametrize("dh", (64, 128))
@pytest.mark.parametrize("page", (16, 32, 64, 256))
def test_chunks(dtype, dh, page):
    paged([150, 1, 0, 33, 64], [333, 65, 7, 33, 128], 6, 2, dh, page, dtype, pad=8, behind=2)


@TYPES
@pytest.mark.parametrize("group", (1, 2, 3, 5, 8, 16, 20))
def test_shared_heads(dtype, group):
    paged([1, 3, 40], [77, 130, 40], 2 * group, 2, 64, 32, dtype)


@TYPES
@pytest.mark.parametrize("block", (0, 1, 7, 64, 100, 2 ** 31 - 1))
def test_blocks(dtype, block):
    paged([90, 5, 1], [260, 5, 131], 2, 2, 128, 16, dtype, block=block)


@TYPES
@pytest.mark.parametrize("window,sinks", ((1, 0), (1, 1), (20, 4), (64, 0), (64, 64), (100, 200), (2 ** 31 - 1, 2 ** 31 - 1),
                                          (33, 2 ** 31 - 1), (2 ** 31 - 1, 0)))
def test_windows(dtype, window, sinks):
    paged([90, 5, 1, 140], [260, 5, 531, 140], 4, 2, 64, 16, dtype, window=window, sinks=sinks)


@TYPES
@pytest.mark.parametrize("block,window,sinks", ((0, 30, 3), (50, 70, 10), (100, 10, 0), (100, 10, 5), (300, 1, 0)))
def test_windows_of_blocks(dtype, block, window, sinks):
    """Among them windows that lie behind the sequence's end: rows that see nothing, or
    the first keys alone."""
    paged([90, 5, 1, 1], [260, 5, 131, 20], 2, 1, 64, 16, dtype, block=block, window=window, sinks=sinks)


@TYPES
@pytest.mark.parametrize("scaled", (False, True))
@pytest.mark.parametrize("std", (0.01, 6.0, 60.0))
def test_scores_of_any_size(dtype, scaled, std):
    paged([70, 1], [200, 300], 2, 1, 128, 64, dtype, scaled=scaled, std=std)


@TYPES
@pytest.mark.parametrize("far", (-1.0, 1.0))
def test_scores_far_from_zero(dtype, far):
    """Every score of a row far above or below 0, the first key's most of all."""
    def change(b):
        b.k[..., 0] = far * 300
        b.k[int(b.table[0, 0]), :, 0, 0] = -far * 300
    paged([40, 1], [100, 90], 1, 1, 64, 16, dtype, std=8.0, change=change)


@TYPES
@pytest.mark.parametrize("rows", ([1, 1, 1], [130, 40, 3]))
@pytest.mark.parametrize("fill", (math.nan, math.inf, -math.inf))
def test_places_without_a_token_hold_anything(dtype, rows, fill):
    paged(rows, [200, 41, 16], 4, 2, 64, 16, dtype, fill=fill)
    paged(rows, [200, 41, 16], 4, 2, 128, 32, dtype, block=30, window=50, sinks=3, fill=fill)


@TYPES
@pytest.mark.parametrize("value", (math.nan, math.inf))
@pytest.mark.parametrize("heads", (2, 8))
def test_hidden_tokens_do_not_reach_a_row(dtype, value, heads):
    """Values and keys that are not finite at tokens which some rows see and others do
    not: rows that see them are not finite, the others as if they were not there."""
    rows, n, dh = 12, 90, 64
    b = R.Batch([rows], [n], 2, dh, 16, dtype)
    q, q0 = R.padded_rows(b.gen, rows, heads, dh, dtype, 0)
    for window, hit_at in ((0, n - 4), (20, n - 4), (20, n - rows - 12)):
        for what in ("k", "v"):
            k, v = b.k.clone(), b.v.clone()
            pg, sl = b.place(0, hit_at)
            (k if what == "k" else v)[pg, :, sl, 3::7] = value
            mask = R.seen(1, window, 0, rows, n)
            want, tol = R.attend(q0, b.keys(b.k, 0), b.keys(b.v, 0), mask, dh ** -0.5, dtype)
            clean = ~mask[:, hit_at]
            assert clean.any() and not clean.all()
            dev = list(b.cuda())
            dev[0], dev[1] = k.cuda(), v.cuda()
            for ws in (None, _ws(dh)):
                out = torch.zeros_like(q)
                B.dif_attention_paged(q, *dev, out, window=window, ws=ws)
                got = out.double().cpu()
                assert ((got[clean] - want[clean]).abs() <= tol[clean]).all()
                assert not torch.isfinite(got[~clean][:, :, 3]).all(-1).any() or what == "k"
                if what == "v":
                    hit = torch.arange(dh) % 7 == 3
                    assert not torch.isfinite(got[~clean][..., hit]).any()
                    assert ((got[~clean] - want[~clean]).abs() <= tol[~clean])[..., ~hit].all()


@TYPES
def test_pages_that_no_row_sees_are_not_read(dtype):
    """Their table entries name pages of NaN, or none at all."""
    def change(b):
        b.k = torch.cat((b.k, torch.full_like(b.k[:1], math.nan)))
        b.v = torch.cat((b.v, torch.full_like(b.v[:1], math.nan)))
        bad = [b.k.shape[0] - 1, -1, 2 ** 31 - 1, -2 ** 31]
        for i in range(2):
            for t in range(1, 9):   # between the first key and the windows
                b.table[i, t] = bad[t % 4]
    for rows in ([1, 1], [20, 7]):
        b = R.Batch(rows, [300, 290], 2, 64, 16, dtype)
        q, q0 = R.padded_rows(b.gen, sum(rows), 4, 64, dtype, 0)
        want, tol, r0 = [], [], 0
        for i, r in enumerate(rows):
            o, t = R.attend(q0[r0:r0 + r], b.keys(b.k, i), b.keys(b.v, i), R.seen(1, 90, 3, r, b.lengths[i]), 0.125, dtype)
            want.append(o)
            tol.append(t)
            r0 += r
        change(b)
        dev = b.cuda()
        for ws in (None, _ws(64)):
            out = torch.zeros_like(q)
            B.dif_attention_paged(q, *dev, out, window=90, sinks=3, ws=ws)
            torch.cuda.synchronize()
            _check(out, torch.cat(want), torch.cat(tol), out.cpu(), "unread pages")


@TYPES
def test_more_rows_than_keys(dtype):
    """Rows before a sequence's first token see nothing; without blocks, everything."""
    for block in (1, 3):
        paged([5, 4, 2], [3, 0, 2], 2, 2, 64, 16, dtype, block=block)
    b = R.Batch([5, 4, 1], [3, 1, 1], 2, 64, 16, dtype)
    paged([5, 4, 1], [3, 1, 1], 2, 2, 64, 16, dtype, block=0)
    packed([5, 0, 4], [3, 0, 0], 2, 2, 64, dtype, block=1)


@TYPES
@pytest.mark.parametrize("dh", (64, 128))
def test_packed_sequences(dtype, dh):
    packed([100, 1, 0, 37], [100, 1, 0, 37], 4, 2, dh, dtype)
    packed([100, 1, 0, 37], [150, 300, 5, 37], 4, 2, dh, dtype, pad=8, behind=3)
    packed([200, 9], [200, 130], 2, 2, dh, dtype, block=30, window=64, sinks=9, scaled=True)
    packed([1, 1, 1], [500, 1, 63], 8, 1, dh, dtype, window=100, sinks=1)


@TYPES
def test_many_sequences(dtype):
    rows = [i % 3 for i in range(700)]
    paged(rows, [max(r, (i * 13) % 50) for i, r in enumerate(rows)], 2, 1, 64, 16, dtype, behind=1)
    paged([1] * 130, [1 + 3 * i for i in range(130)], 2, 1, 64, 16, dtype)


@TYPES
@pytest.mark.parametrize("rows", ([1], [1, 2], [30], [3, 200]))
def test_long_caches(dtype, rows):
    """Key ranges that are split, at lengths that end inside a page."""
    paged(rows, [5003, 3001][:len(rows)], 4, 2, 64, 16, dtype)
    paged(rows, [5003, 3001][:len(rows)], 2, 2, 128, 64, dtype, window=2000, sinks=70)


def test_past_32_bits():
    """Pages 5 GiB into the cache."""
    P, H, S, dh = 5 * 2 ** 30 // (2 * 8 * 256 * 128) + 2, 8, 256, 128
    ck = torch.zeros((P, H, S, dh), dtype=BF, device="cuda")
    cv = torch.zeros((P, H, S, dh), dtype=BF, device="cuda")
    gen = torch.Generator().manual_seed(3)
    k, v = (torch.randn((H, S, dh), generator=gen).to(BF) for _ in range(2))
    ck[P - 1], cv[P - 1] = k.cuda(), v.cuda()
    table = torch.tensor([[P - 1]], dtype=torch.int32).cuda()
    lengths = torch.tensor([S], dtype=torch.int32).cuda()
    for r in (1, 100):
        q, q0 = R.padded_rows(gen, r, H, dh, BF, 0)
        out = torch.zeros_like(q)
        B.dif_attention_paged(q, ck, cv, table, lengths, torch.tensor([0, r], dtype=torch.int32).cuda(), out, ws=_ws(dh))
        torch.cuda.synchronize()
        want, tol = R.attend(q0, k.transpose(0, 1), v.transpose(0, 1), R.seen(1, 0, 0, r, S), dh ** -0.5, BF)
        _check(out, want, tol, out.cpu(), "far pages")


@TYPES
def test_tables_out_of_range_stay_inside(dtype):
    b = R.Batch([4, 4], [40, 40], 1, 64, 16, dtype)
    q, _ = R.padded_rows(b.gen, 8, 2, 64, dtype, 0)
    k, _ = R.padded_rows(b.gen, 8, 1, 64, dtype, 0)
    dev = list(b.cuda())
    wild = lambda *v: torch.tensor(v, dtype=torch.int32).cuda()
    for off in ((-5, 4, 100), (3, 2, 9), (2 ** 31 - 1, -2 ** 31, 7), (8, 8, 8)):
        for length in ((40, 40), (-3, 2 ** 31 - 1), (0, 1000)):
            for ws in (None, _ws(64)):
                B.dif_attention_paged(q, dev[0], dev[1], dev[2], wild(*length), wild(*off), torch.zeros_like(q), ws=ws)
            B.dif_attention_window(q, k, k, wild(*off), torch.zeros_like(q))
            B.dif_attention_window(q, k, k, wild(0, 4, 8), torch.zeros_like(q), key_offsets=wild(*off))
    torch.cuda.synchronize()


@TYPES
def test_streams_of_tokens(dtype):
    """The operators as they are used: a prompt and then single tokens, appended and
    attended to, against the packed attention of the whole sequence."""
    heads, kv, dh, page, lens = 4, 2, 64, 16, [37, 20]
    gen = torch.Generator().manual_seed(9)
    rows = [R.padded_rows(gen, n, heads + 2 * kv, dh, dtype, 0)[0] for n in lens]
    gq, gk = (1 + 0.1 * torch.randn(h * dh, generator=gen).cuda() for h in (heads, kv))
    P = 8
    ck, cv = (torch.full((P, kv, page, dh), math.nan, dtype=dtype, device="cuda") for _ in range(2))
    table = torch.tensor([[5, 0, 3], [7, 2, -1]], dtype=torch.int32).cuda()
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32).cuda()
    ws, got, held = _ws(dh), [[], []], [0, 0]
    for step in ([30, 11], [1, 1], [1, 0], [0, 3], [5, 5]):
        new = [torch.cat([r[h:h + s] for r, h, s in zip(rows, held, step)])][0]
        held = [h + s for h, s in zip(held, step)]
        q, k, v = new[:, :heads], new[:, heads:heads + kv], new[:, heads + kv:]
        args = (ck, cv, table, i32(*held), i32(0, step[0], sum(step)))
        qo, out = torch.empty(q.shape, dtype=dtype, device="cuda"), torch.empty(q.shape, dtype=dtype, device="cuda")
        B.dif_cache_append(*args, k, v, q=q, q_out=qo, gain_k=gk, gain_q=gq, theta=10000.0)
        B.dif_attention_paged(qo, *args, out, window=16, sinks=2, ws=ws)
        got[0].append(out[:step[0]])
        got[1].append(out[step[0]:])
    for i in range(2):
        n = held[i]
        assert n == lens[i]
        # the same tokens at once: appended to a cache of their own, whose rows are then packed
        c2k, c2v = (torch.zeros((3, kv, page, dh), dtype=dtype, device="cuda") for _ in range(2))
        q, k, v = rows[i][:, :heads], rows[i][:, heads:heads + kv], rows[i][:, heads + kv:]
        qo = torch.empty(q.shape, dtype=dtype, device="cuda")
        B.dif_cache_append(c2k, c2v, i32(0, 1, 2)[None], i32(n), i32(0, n), k, v, q=q, q_out=qo, gain_k=gk, gain_q=gq,
                           theta=10000.0)
        flat = lambda c: c.transpose(1, 2).reshape(3 * page, kv, dh)[:n].contiguous()
        out = torch.empty(q.shape, dtype=dtype, device="cuda")
        B.dif_attention_window(qo, flat(c2k), flat(c2v), i32(0, n), out, window=16, sinks=2)
        want, tol = R.attend(qo.cpu(), flat(c2k).cpu(), flat(c2v).cpu(), R.seen(1, 16, 2, n, n), dh ** -0.5, dtype)
        _check(out, want, tol, out.cpu(), "packed")
        _check(torch.cat(got[i]), want, tol, out.cpu(), "streamed")


def test_captured_with_tables_that_change():
    """A captured append and attention follow lengths, offsets, pages and queries."""
    heads, kv, dh, page, M = 4, 2, 128, 16, 6
    b = R.Batch([3, 3], [70, 35], kv, dh, page, BF, max_pages=8)
    free = [p for p in range(b.k.shape[0]) if p not in b.table.flatten().tolist()]
    dev = b.cuda()
    q, k, v = (R.padded_rows(b.gen, M, h, dh, BF, 0)[0].contiguous() for h in (heads, kv, kv))
    qo, out, ws = torch.zeros_like(q), torch.zeros_like(q), _ws(dh)

    def step():
        B.dif_cache_append(*dev, k, v, q=q, q_out=qo, theta=10000.0)
        B.dif_attention_paged(qo, *dev, out, ws=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn, (lengths, off) in enumerate((([70, 35], [0, 3, 6]), ([73, 36], [0, 5, 6]), ([73, 40], [0, 0, 4]))):
        dev[3].copy_(torch.tensor(lengths, dtype=torch.int32))
        dev[4].copy_(torch.tensor(off, dtype=torch.int32))
        q.copy_(torch.randn(q.shape, generator=b.gen).to(BF))
        keep = [t.clone() for t in dev[:2]]
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        first = out.clone()
        for t, s in zip(dev[:2], keep):
            t.copy_(s)
        out.fill_(9.0)
        step()
        torch.cuda.synchronize()
        assert torch.equal(first, out), f"replay {turn}"
        assert (out[off[2]:] == 9.0).all()
    assert free


def test_on_another_stream():
    b = R.Batch([3, 1], [70, 35], 2, 64, 16, BF)
    dev = b.cuda()
    q, _ = R.padded_rows(b.gen, 4, 4, 64, BF, 0)
    one, two = torch.zeros_like(q), torch.zeros_like(q)
    B.dif_attention_paged(q, *dev, one, ws=_ws(64))
    ws = _ws(64)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    B.dif_attention_paged(q, *dev, two, ws=ws, stream=s)
    s.synchronize()
    assert torch.equal(one, two)


WIDE = pytest.mark.parametrize("rows,lengths,heads,kv", (
    ([300], [300], 1, 1), ([257, 700], [900, 700], 2, 2), ([130, 40], [1500, 333], 8, 2), ([513], [4000], 1, 1)))


# (tokens that a sequence's pages may hold: tables with room for more than 2048 choose the kernel
# of long caches, however many there are)
ROOM = pytest.mark.parametrize("room", (0, 4096))


@ROOM
@WIDE
@pytest.mark.parametrize("block,window,sinks", ((1, 0, 0), (0, 0, 0), (100, 0, 0), (1, 150, 0), (1, 400, 70), (1, 3000, 300),
                                                (64, 128, 64), (1000, 700, 5), (4096, 10, 3)))
def test_long_chunks(rows, lengths, heads, kv, block, window, sinks, room):
    paged(rows, lengths, heads, kv, 128, 16 if window else 64, BF, block=block, window=window, sinks=sinks, pad=8, behind=3,
          scaled=block == 0 or window > 300, room=room)


@ROOM
@WIDE
def test_long_packed_chunks(rows, lengths, heads, kv, room):
    if room:   # a sequence of keys alone
        rows, lengths = [0] + rows, [2100] + lengths
    packed(rows, lengths, heads, kv, 128, BF, block=1, pad=8, behind=3)
    packed(rows, lengths, heads, kv, 128, BF, block=30, window=500, sinks=64, scaled=True)


@ROOM
@pytest.mark.parametrize("fill", (math.nan, math.inf, -math.inf))
def test_long_chunks_beside_places_without_a_token(fill, room):
    paged([300, 200], [1000, 203], 2, 2, 128, 16, BF, fill=fill, room=room)
    paged([300, 200], [1000, 203], 2, 2, 128, 32, BF, block=70, window=333, sinks=20, fill=fill, room=room)


@ROOM
def test_long_chunks_of_more_rows_than_keys(room):
    for lengths in ([0, 2500], [30, 0], [299, 64]):
        for block, window, sinks in ((1, 0, 0), (0, 0, 0), (16, 40, 3)):
            paged([300, 280], lengths, 2, 1, 128, 16, BF, block=block, window=window, sinks=sinks, behind=5, room=room)
    packed([300, 280], [2300, 0], 2, 1, 128, BF, block=1)
    packed([300, 280], [0, 2300], 2, 2, 128, BF, block=7, window=50, sinks=9)


@ROOM
@pytest.mark.parametrize("far", (-1.0, 1.0))
def test_long_chunks_of_scores_far_from_zero(far, room):
    def change(b):
        b.k[..., 0] = far * 300
        b.k[int(b.table[0, 0]), :, 0, 0] = -far * 300
    for scaled in (False, True):
        paged([400], [600], 1, 1, 128, 16, BF, std=8.0, change=change, scaled=scaled, room=room)
        paged([400], [600], 1, 1, 128, 16, BF, std=8.0, change=change, window=100, sinks=3, scaled=scaled, room=room)


@pytest.mark.parametrize("value", (math.nan, math.inf, -math.inf))
@pytest.mark.parametrize("dh,rows,room", ((128, 300, 0), (128, 300, 4096), (64, 300, 0), (128, 40, 0)))
def test_hidden_tokens_do_not_reach_the_rows_of_a_chunk(value, dh, rows, room):
    n = rows + 500
    b = R.Batch([rows], [n], 1, dh, 16, BF, max_pages=room // 16 or None)
    q, q0 = R.padded_rows(b.gen, rows, 2, dh, BF, 0)
    for window, hit_at in ((0, n - 20), (250, n - rows - 249 + rows // 2), (250, n - 30)):
        mask = R.seen(1, window, 0, rows, n)
        want, tol = R.attend(q0, b.keys(b.k, 0), b.keys(b.v, 0), mask, dh ** -0.5, BF)
        clean = ~mask[:, hit_at]
        assert clean.any() and not clean.all()
        for what in ("k", "v"):
            k, v = b.k.clone(), b.v.clone()
            pg, sl = b.place(0, hit_at)
            (k if what == "k" else v)[pg, :, sl, 3::7] = value
            dev = list(b.cuda())
            dev[0], dev[1] = k.cuda(), v.cuda()
            for ws in (None, _ws(dh)):
                out = torch.zeros_like(q)
                B.dif_attention_paged(q, *dev, out, window=window, ws=ws)
                got = out.double().cpu()
                assert ((got[clean] - want[clean]).abs() <= tol[clean]).all()
                if what == "v":
                    hit = torch.arange(dh) % 7 == 3
                    assert not torch.isfinite(got[~clean][..., hit]).any()
                    assert ((got[~clean] - want[~clean]).abs() <= tol[~clean])[..., ~hit].all()
                else:   # (an infinite key may also leave a row by the other side)
                    assert math.isinf(value) or not torch.isfinite(got[~clean]).any()


def test_long_chunks_of_tables_out_of_range_stay_inside():
    b = R.Batch([150, 150], [400, 400], 1, 128, 16, BF, max_pages=256)
    q, _ = R.padded_rows(b.gen, 300, 2, 128, BF, 0)
    dev = list(b.cuda())
    k = torch.zeros((2100, 1, 128), dtype=BF, device="cuda")
    wild = lambda *v: torch.tensor(v, dtype=torch.int32).cuda()
    for off in ((-5, 4, 1000), (3, 2, 9), (2 ** 31 - 1, -2 ** 31, 7), (300, 300, 300)):
        for length in ((400, 400), (-3, 2 ** 31 - 1), (0, 100000)):
            for ws in (None, _ws(128)):
                say(f"offsets {off} lengths {length}")
                B.dif_attention_paged(q, dev[0], dev[1], dev[2], wild(*length), wild(*off), torch.zeros_like(q), ws=ws)
            B.dif_attention_window(q, k, k, wild(*off), torch.zeros_like(q), key_offsets=wild(0, 4, 2100))
            B.dif_attention_window(q, k, k, wild(0, 200, 300), torch.zeros_like(q), key_offsets=wild(*off))
    torch.cuda.synchronize()


def test_long_chunks_captured_with_tables_that_change():
    """Whole and split, each replay against the eager call."""
    heads, kv, page, M = 2, 1, 16, 300
    b = R.Batch([150, 150], [1500, 900], kv, 128, page, BF, max_pages=256)
    dev, ws = b.cuda(), _ws(128)
    q = R.padded_rows(b.gen, M, heads, 128, BF, 0)[0].contiguous()
    out = torch.zeros_like(q)

    def step():
        B.dif_attention_paged(q, *dev, out, window=600, sinks=5, ws=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn, (lengths, off) in enumerate((([1500, 900], [0, 150, 300]), ([300, 900], [0, 299, 300]), ([1, 0], [0, 0, 0]),
                                           ([1400, 20], [0, 280, 290]))):
        dev[3].copy_(torch.tensor(lengths, dtype=torch.int32))
        dev[4].copy_(torch.tensor(off, dtype=torch.int32))
        q.copy_(torch.randn(q.shape, generator=b.gen).to(BF))
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        first = out.clone()
        out.fill_(9.0)
        step()
        torch.cuda.synchronize()
        assert torch.equal(first, out), f"replay {turn}"
        assert (out[off[2]:] == 9.0).all()


@TYPES
def test_chunks_beside_many_tokens(dtype):
    """Few rows on average: the single tokens and the chunks have launches of their own."""
    rows = [1] * 70 + [300, 0, 65, 64, 5] + [0] * 60
    lengths = [7 * i + 1 for i in range(70)] + [1500, 9, 65, 2000, 40] + [3] * 60
    paged(rows, lengths, 2, 2, 128, 64, dtype, behind=2)
    paged(rows, lengths, 4, 1, 64, 16, dtype, window=90, sinks=3)
    packed(rows, lengths, 2, 1, 128, dtype, block=50)


def test_most_sequences():
    n = 4096
    rows = [(i * 7) % 3 for i in range(n)]
    paged(rows, [max(r, i % 20) for i, r in enumerate(rows)], 1, 1, 64, 16, BF, behind=1)
    rows = [0] * n
    rows[4095], rows[17], rows[2000] = 300, 1, 2
    paged(rows, [max(r, i % 3) for i, r in enumerate(rows)], 2, 1, 128, 16, BF)
