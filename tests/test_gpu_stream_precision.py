"""bf16 single tokens keep 15 bits of a probability: a bound without its rounding to bf16, over
values whose sums nearly cancel, so that the output's own rounding does not hide it."""
import math

import pytest
import torch

from paper_2607_06631_amd import binding as B
from tests import stream_ref as R
from tests.gpu_util import say

BF, F32 = torch.bfloat16, torch.float32


def _bound(q, k, v, mask, scale):
    """The definition, and how far the kernel may be off: float32's bound, 2^-15 of every
    probability (two bf16 terms: the first leaves up to 2^-7, of which the second's rounding is
    half a step of 2^-8), the output's rounding."""
    o, t = R.attend(q, k, v, mask, scale, F32)
    a, _ = R.attend(q, k, v.abs(), mask, scale, F32)
    t = t + 1.01 * a * 2.0 ** -15
    return o, t + (o.abs() + t) * 2.0 ** -8


def _case(rows, lengths, kv, dh, seed):
    """Scores near 0, values +1 and -1 in turn (a dim for each of some phases)."""
    b = R.Batch(rows, lengths, kv, dh, 16, BF, seed=seed)
    for i, n in enumerate(lengths):
        for j in range(n):
            pg, sl = b.place(i, j)
            b.v[pg, :, sl] = torch.where((j // (1 + torch.arange(dh) % 5)) % 2 == 0, 1.0, -1.0).to(BF)
    return b


def _rounded(q, k, v, mask, scale):
    """The definition with probabilities (of the row's largest) rounded once to bf16."""
    s = torch.where(mask, q[:, 0].double() @ k[:, 0].double().t() * scale, -math.inf)
    p = torch.exp(s - s.amax(1, keepdim=True))
    return (p.to(BF).double() @ v[:, 0].double() / p.sum(1, keepdim=True)).to(BF).double()


@pytest.mark.parametrize("dh", (64, 128))
@pytest.mark.parametrize("n", (2, 4, 16, 33, 100, 600))
def test_the_bound_tells_one_rounding(dh, n):
    rows = 64   # single tokens that see the same cache
    b = _case([1], [n], 1, dh, n)
    gen = torch.Generator().manual_seed(n)
    q = (torch.randn((rows, 1, dh), generator=gen) * 0.3).to(BF)
    k, v, mask = b.keys(b.k, 0), b.keys(b.v, 0), R.seen(0, 0, 0, rows, n)
    o, t = _bound(q, k, v, mask, dh ** -0.5)
    assert ((o.to(BF).double() - o).abs() <= t).all()
    assert ((_rounded(q, k, v, mask, dh ** -0.5) - o[:, 0]).abs() > t[:, 0]).any()


@pytest.mark.gpu
@pytest.mark.parametrize("dh", (64, 128))
@pytest.mark.parametrize("rows,lengths", (
    ([1] * 6, [2, 4, 16, 33, 100, 600]), ([1] * 64, [2 + 9 * i for i in range(64)]), ([2, 3, 1, 4], [5, 40, 700, 64]),
    ([1, 1], [5003, 3001])))
@pytest.mark.parametrize("group", (1, 4))
def test_single_tokens(dh, rows, lengths, group):
    say(f"precision {dh} {rows[:4]} {lengths[:4]} {group}")
    b = _case(rows, lengths, 2, dh, 7)
    q, q0 = R.padded_rows(b.gen, sum(rows), 2 * group, dh, BF, 0, 0.3)
    want, tol, r0 = [], [], 0
    for i, r in enumerate(rows):
        o, t = _bound(q0[r0:r0 + r], b.keys(b.k, i), b.keys(b.v, i), R.seen(1, 0, 0, r, lengths[i]), dh ** -0.5)
        want.append(o)
        tol.append(t)
        r0 += r
    want, tol = torch.cat(want), torch.cat(tol)
    for ws in (None, torch.full((B.dif_attention_paged_bytes(dh),), 255, dtype=torch.uint8, device="cuda")):
        out = torch.zeros_like(q)
        B.dif_attention_paged(q, *b.cuda(), out, ws=ws)
        bad = ~((out.double().cpu() - want).abs() <= tol)
        assert not bad.any(), f"{int(bad.sum())} off, first {bad.nonzero()[0].tolist()}"
