"""dif_cache_append against float64: every place of the cache, the rows it leaves, and
what it must not touch."""
import pytest
import torch

from paper_2607_06631_amd import binding as B
from tests import stream_ref as R
from tests.gpu_util import say

pytestmark = [pytest.mark.gpu]

BF, F32 = torch.bfloat16, torch.float32


def _bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == BF else torch.int32)


def _close(got, want, tol, name):
    got = got.double().cpu()
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), f"{name}: {int(bad.sum())} off, worst {float((got - want).abs().max()):.3e}"


def _run(rows, lengths, heads, kv, dh, page, dtype, layout="hnd", axes=1, norm=True, positions=None, norm_dim=0,
         scale=1.0, pad=0, behind=0, theta=10000.0, with_q=True, in_place=False, seed=1):
    say(f"append {rows} {lengths} {heads}/{kv}x{dh} page {page} {dtype} {layout} axes {axes}")
    b = R.Batch(rows, lengths, kv, dh, page, dtype, layout, seed=seed)
    m = sum(rows) + behind
    q, q0 = R.padded_rows(b.gen, m, heads, dh, dtype, pad, 0.8)
    k, k0 = R.padded_rows(b.gen, m, kv, dh, dtype, pad, 0.8)
    v, v0 = R.padded_rows(b.gen, m, kv, dh, dtype, pad)
    gq = 1 + 0.2 * torch.randn(heads * dh, generator=b.gen) if norm else None
    gk = 1 + 0.2 * torch.randn(kv * dh, generator=b.gen) if norm else None
    at = torch.cat([torch.arange(n - r, n) for r, n in zip(rows, lengths)] + [torch.zeros(behind, dtype=torch.long)])
    pos = None
    if positions is not None:
        pos = positions(at).int()
    out = q if in_place else torch.full((m, heads, dh), 7.0, dtype=dtype, device="cuda")
    dev = b.cuda()
    up = lambda t: None if t is None else t.cuda()
    B.dif_cache_append(*dev, k, v, q=q if with_q else None, q_out=out if with_q else None, gain_k=up(gk),
                       gain_q=up(gq) if with_q else None, norm_dim=norm_dim, theta=theta, axes=axes, positions=up(pos),
                       q_scale=scale)
    torch.cuda.synchronize()
    pairs = [dh // 2] if axes == 1 else [dh // 2 - 2 * (dh // 6), dh // 6, dh // 6]
    p64 = at[:, None] if pos is None else pos.view(m, -1)
    half = R.HALF[dtype]
    yk, tk = R.turned(k0, gk, norm_dim, 1e-6, p64, theta, pairs, 1.0)
    yq, tq = R.turned(q0, gq, norm_dim, 1e-6, p64, theta, pairs, scale)
    want_k, tol_k = b.k.double(), torch.zeros_like(b.k, dtype=torch.float64)
    want_v = b.v.clone()
    r0 = 0
    for i, (r, n) in enumerate(zip(rows, lengths)):
        for j in range(r):
            pg, sl = b.place(i, n - r + j)
            want_k[pg, :, sl], tol_k[pg, :, sl] = yk[r0], tk[r0] + yk[r0].abs() * half
            want_v[pg, :, sl] = v0[r0]
            r0 += 1
    _close(dev[0], want_k, tol_k, "keys")   # (a tolerance of 0 wherever nothing was appended)
    assert torch.equal(_bits(dev[1].cpu()), _bits(want_v))
    if with_q:
        _close(out[:r0], yq[:r0], tq[:r0] + yq[:r0].abs() * half, "queries")
        assert torch.equal(out[r0:].cpu(), (q0[r0:] if in_place else torch.full_like(q0[r0:], 7.0)))


@pytest.mark.parametrize("dtype", (BF, F32), ids=("bf16", "f32"))
@pytest.mark.parametrize("dh", (64, 128))
@pytest.mark.parametrize("layout", ("hnd", "nhd"))
def test_types_and_layouts(dtype, dh, layout):
    _run([5, 0, 1, 37], [9, 3, 100, 37], 6, 3, dh, 16, dtype, layout, pad=8, behind=3, scale=0.37)


@pytest.mark.parametrize("dtype", (BF, F32), ids=("bf16", "f32"))
@pytest.mark.parametrize("dh", (64, 128))
def test_three_axes(dtype, dh):
    grid = lambda at: torch.stack((at // 15 + 900, at // 5 % 3, at % 5), 1)
    _run([40, 1], [45, 31], 4, 4, dh, 32, dtype, axes=3, positions=grid, norm_dim=11 * dh)


@pytest.mark.parametrize("first", (0, -5, 1000003, 2 ** 31 - 60, -2 ** 31))
def test_far_positions(first):
    _run([50, 7], [50, 7], 2, 1, 128, 16, F32, norm=False, positions=lambda at: at + first)


@pytest.mark.parametrize("heads,kv", ((1, 1), (40, 40), (12, 12), (32, 8), (64, 2), (7, 1)))
def test_widths(heads, kv):
    _run([3, 1], [70, 65], heads, kv, 128, 64, BF, norm=True)


def test_widest_rows():
    _run([3], [3], 64, 64, 128, 16, BF, norm=True)
    _run([3], [3], 32, 32, 128, 16, F32, norm=True)
    _run([2], [2], 130, 65, 128, 16, BF, norm=False)    # more than a wave holds: in turns
    _run([2], [2], 99, 33, 64, 16, F32, norm=False)


def test_without_rotation_norm_or_queries():
    _run([4], [20], 4, 2, 64, 16, BF, norm=False, theta=0.0)
    _run([4], [20], 4, 2, 64, 16, BF, norm=True, theta=0.0)
    _run([4, 3], [20, 3], 4, 2, 64, 16, F32, with_q=False)
    _run([4, 3], [20, 3], 4, 2, 128, 16, BF, in_place=True, behind=2)


def test_many_sequences():
    rows = [i % 3 for i in range(1000)]
    _run(rows, [r + i % 40 for i, r in enumerate(rows)], 2, 1, 64, 16, BF, behind=1)
    _run([1] * 65, [1 + i for i in range(65)], 1, 1, 64, 16, F32)


def test_tokens_without_a_place_are_not_stored():
    b = R.Batch([3, 3, 3, 2], [3, 20, 31, 2], 2, 64, 16, F32, max_pages=2)
    m = 11
    q, _ = R.padded_rows(b.gen, m, 2, 64, F32, 0)
    k, k0 = R.padded_rows(b.gen, m, 2, 64, F32, 0)
    lengths = torch.tensor([1, 20, 34, 2], dtype=torch.int32)     # two indexes negative; two past two pages
    table = b.table.clone()
    table[1, 1], table[3, 0] = b.k.shape[0], -1                    # pages outside the cache
    dev = list(b.cuda())
    dev[2], dev[3] = table.cuda(), lengths.cuda()
    out = torch.zeros_like(q)
    B.dif_cache_append(*dev, k, k, q=q, q_out=out)
    torch.cuda.synchronize()
    want = b.k.clone()
    want[b.table[0, 0].long(), :, 0] = k0[2]
    want[b.table[2, 1].long(), :, 15] = k0[6]
    assert torch.equal(dev[0].cpu(), want)
    assert torch.equal(out, q)


def test_offsets_out_of_range_stay_inside():
    b = R.Batch([4, 4], [40, 40], 1, 64, 16, BF)
    k, _ = R.padded_rows(b.gen, 8, 1, 64, BF, 0)
    dev = list(b.cuda())
    for off in ([-5, 4, 100], [3, 2, 9], [2 ** 31 - 1, -2 ** 31, 7], [8, 8, 8]):
        dev[4] = torch.tensor(off, dtype=torch.int32).cuda()
        B.dif_cache_append(*dev, k, k)
    torch.cuda.synchronize()


def test_past_32_bits():
    """Pages 5 GiB into the cache."""
    P, H, S, dh = 5 * 2 ** 30 // (2 * 8 * 256 * 128) + 2, 8, 256, 128
    ck = torch.zeros((P, H, S, dh), dtype=BF, device="cuda")
    cv = torch.zeros((P, H, S, dh), dtype=BF, device="cuda")
    gen = torch.Generator().manual_seed(3)
    k, k0 = R.padded_rows(gen, 2, H, dh, BF, 0)
    table = torch.tensor([[P - 1], [0]], dtype=torch.int32).cuda()
    lengths = torch.tensor([S, 1], dtype=torch.int32).cuda()
    B.dif_cache_append(ck, cv, table, lengths, torch.tensor([0, 1, 2], dtype=torch.int32).cuda(), k, k)
    torch.cuda.synchronize()
    assert torch.equal(ck[P - 1, :, S - 1].cpu(), k0[0]) and torch.equal(cv[0, :, 0].cpu(), k0[1])
    assert int((ck != 0).any(-1).sum()) == 2 * H


@pytest.mark.parametrize("with_q", (True, False))
@pytest.mark.parametrize("m", (1, 2, 3, 5, 6, 7, 9))
def test_any_number_of_rows(m, with_q):
    """Waves left over in the last workgroup write nothing."""
    _run([m], [m + 3], 4, 2, 64, 16, BF, with_q=with_q)
