"""Streamed generation in float64 from its definitions, one row's keys as a mask, with the
bounds that the kernels' roundings add up to; batches with pages in a mixed order."""
import math

import torch

LOG2E = 1.4426950408889634
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # half a step, relative


def seen(block, window, sinks, rows, n):
    """[rows, n]: the keys that the last `rows` positions of n keys see."""
    out = torch.zeros((rows, n), dtype=torch.bool)
    for i in range(rows):
        p = n - rows + i
        if block and p < 0:
            continue
        e = (p // block + 1) * block if block else n
        for j in range(max(0, e - window) if window else 0, min(e, n)):
            out[i, j] = True
        if window:
            out[i, :max(0, min(sinks, e, n))] = True
    return out


def attend(q, k, v, mask, scale, dtype):
    """softmax(q k^T scale) v of one sequence over what `mask` leaves, and how far a kernel
    in `dtype` may be off: q [r, H, dh], k and v [n, Hkv, dh].

    A probability is rounded once to dtype (its sum is not), the output once; scores are
    float32 sums of dh products, off by (dh + 8) 2^-24 of their absolute sum, and so
    are the probabilities' exponents (numerator and denominator: twice); sums over the
    keys are float32, n + 64 roundings at most; 2^-20 for exponential and reciprocal."""
    r, H, dh = q.shape
    n, kv = k.shape[:2]
    q, k, v = q.double(), k.double(), v.double()
    out, tol = torch.zeros(r, H, dh, dtype=torch.float64), torch.zeros(r, H, dh, dtype=torch.float64)
    if not n:
        return out, tol
    half = HALF[dtype]
    for h in range(H):
        kh, vh = k[:, h // (H // kv)], v[:, h // (H // kv)]
        s = torch.where(mask, q[:, h] @ torch.nan_to_num(kh, 0, 0, 0).t() * scale, -math.inf)
        top = s.amax(1, keepdim=True)
        p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
        total = p.sum(1, keepdim=True)
        p = torch.where(total > 0, p / total, 0.0)
        vh = torch.nan_to_num(vh, 0, 0, 0)
        o, a = p @ vh, p @ vh.abs()
        reach = torch.where(mask, q[:, h].abs() @ torch.nan_to_num(kh, 0, 0, 0).abs().t() * scale, 0.0).amax(1, keepdim=True)
        small = 2 * reach * (dh + 8) * 2.0 ** -24 + (n + 64) * 2.0 ** -24 + 2.0 ** -20
        out[:, h] = o
        tol[:, h] = a * (small + (half if dtype == torch.bfloat16 else 0.0)) * 1.01 + o.abs() * half + 1e-38
    return out, tol


class Batch:
    """A paged cache holding `lengths` tokens of each sequence, `rows` of them new."""

    def __init__(self, rows, lengths, kv, dh, page, dtype, layout="hnd", fill=None, seed=0, spare=2, max_pages=None):
        self.rows, self.lengths, self.page = rows, lengths, page
        gen = torch.Generator().manual_seed(seed)
        pages = [-(-n // page) for n in lengths]
        total = sum(pages) + spare
        order = torch.randperm(total, generator=gen).tolist()
        self.table = torch.full((len(rows), max_pages or max(1, *pages)), -7, dtype=torch.int32)
        for i, n in enumerate(pages):
            for t in range(n):
                self.table[i, t] = order.pop()
        shape = (total, kv, page, dh) if layout == "hnd" else (total, page, kv, dh)
        self.k = torch.randn(shape, generator=gen).to(dtype)
        self.v = torch.randn(shape, generator=gen).to(dtype)
        if layout == "nhd":
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        self.offsets = torch.tensor([sum(rows[:i]) for i in range(len(rows) + 1)], dtype=torch.int32)
        self.gen = gen
        if fill is not None:   # every place that holds no token
            for t in (self.k, self.v):
                used = torch.zeros((total, page), dtype=torch.bool)
                for i, n in enumerate(lengths):
                    j = torch.arange(n)
                    used[self.table[i].long()[j // page], j % page] = True
                t.transpose(1, 2)[~used] = fill

    def keys(self, t, i):
        """[n, kv, dh] of sequence i."""
        j = torch.arange(self.lengths[i])
        return t[self.table[i].long()[j // self.page], :, j % self.page]

    def place(self, i, j):
        return int(self.table[i, j // self.page]), j % self.page

    def cuda(self):
        """(cache_k, cache_v, table, lengths, row_offsets) on the device, layouts kept."""
        def up(t):
            return t.transpose(1, 2).contiguous().cuda().transpose(1, 2) if not t.is_contiguous() else t.cuda()
        return (up(self.k), up(self.v), self.table.cuda(), torch.tensor(self.lengths, dtype=torch.int32).cuda(),
                self.offsets.cuda())


def padded_rows(gen, m, heads, dh, dtype, pad, std=1.0):
    """[m, heads, dh] on the device with rows heads * dh + pad apart, and the same on the host."""
    t = (torch.randn((m, heads * dh + pad), generator=gen) * std).to(dtype)
    return t.cuda()[:, :heads * dh].unflatten(1, (heads, dh)), t[:, :heads * dh].unflatten(1, (heads, dh))


def turned(x, gain, norm_dim, eps, positions, theta, pairs, scale):
    """Norm, rotation and scale of rows x [m, heads, dh] in float64; positions [m, axes], pairs
    of each axis; and the bound of what float32 does to it, before the last rounding."""
    x = x.double()
    m, heads, dh = x.shape
    wide = heads * dh
    if gain is not None:
        x = x / torch.sqrt((x * x).sum((1, 2), keepdim=True) / (norm_dim or wide) + eps) * gain.double().view(heads, dh)
    y, reach = x.clone(), x.abs()
    if theta:
        angle = torch.cat([positions[:, a:a + 1].double() * theta ** (-torch.arange(n, dtype=torch.float64) / n)
                           for a, n in enumerate(pairs)], 1)[:, None]
        a, b = x[..., 0::2], x[..., 1::2]
        y = torch.stack((a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()), -1).flatten(2)
        reach = (a.abs() + b.abs()).repeat_interleave(2, -1)
    # sines to 2^-22 (angle, series, products), a sum of `wide` squares under a root, a few products
    return y * scale, reach * scale * (2.0 ** -21 + (wide * 2.0 ** -25 if gain is not None else 0.0))
