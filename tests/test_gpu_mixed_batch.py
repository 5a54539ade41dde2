"""dif_gemm_grouped and dif_gemm_lora through the C ABI against float64, entry by
entry within a bound that counts roundings (tests/mixed_batch.py)."""
import pytest

from tests.gpu_util import say
from tests.mixed_batch import GELU, RESIDUAL, STORE, Problem

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]

# (rows of the groups, N, K, more)
GROUPED = {
    "one_row": ([1], 1, 1, {}),
    "one_row_wide": ([1], 700, 512, {}),
    "single_rows": ([1, 0, 1, 1, 0, 0, 1], 320, 640, {}),
    "empty": ([0, 0, 0], 64, 64, dict(behind=5)),
    "k_zero": ([3, 5], 40, 0, {}),
    "odd": ([37, 1, 64, 0, 129], 77, 203, dict(behind=3, pad=24)),
    "k_below_a_tile": ([17, 40], 65, 24, {}),
    "k_ends_in_a_chunk": ([17, 40], 65, 129, {}),
    "shared_matrices": ([50, 7, 33, 64], 130, 192, dict(weights=2, index=[1, 0, 1, 1])),
    "bad_index": ([10, 20, 30], 48, 64, dict(weights=2, index=[0, -1, 2])),
    "kept": ([65, 65, 65, 65], 192, 320, dict(n_kept=[192, 1, 0, 101], k_kept=[320, 7, 64, 0])),
    "kept_beyond": ([9, 9], 33, 64, dict(n_kept=[99, -4], k_kept=[-1, 1 << 30])),
    "before_and_behind": ([100, 28], 96, 128, dict(before=11, behind=40)),
    "many_groups": ([(i * 7) % 4 for i in range(200)], 72, 96, dict(weights=5, index=[i % 5 for i in range(200)])),
    "tall": ([1500, 3, 997], 256, 256, {}),
    "wide": ([60, 200], 2100, 576, {}),
    "large_tiles": ([2100, 1999], 1280, 704, dict(pad=8)),
    "long_reduction": ([120, 33], 260, 4160, dict(k_kept=[4160, 4099])),
}


@pytest.mark.parametrize("types", TYPES, ids="_".join)
@pytest.mark.parametrize("epilogue", [STORE, GELU, RESIDUAL])
@pytest.mark.parametrize("case", GROUPED)
def test_grouped(case, epilogue, types):
    rows, N, K, more = GROUPED[case]
    say(f"grouped {case} epilogue={epilogue} {types}")
    p = Problem(rows, N, K, epilogue, *types, seed=len(case), **more)
    p.check(p.run())


# (rows of the requests, N, K, adapters of the requests, rank, adapters, more)
LORA = {
    "one_row": ([1], 5, 8, [0], 1, 1, {}),
    "single_rows": ([1] * 9, 320, 640, [3, 0, 1, -1, 2, 2, 0, 7, 1], 16, 4, {}),
    "no_adapters": ([5, 9], 64, 128, [-1, -1], 8, 2, {}),
    "none_at_all": ([5, 9], 64, 128, [0, 0], 8, 0, {}),
    "empty_requests": ([0, 4, 0, 0, 60, 0], 70, 96, [0, 1, 0, 2, 0, 1], 8, 3, {}),
    "odd": ([37, 1, 64, 0, 129], 77, 203, [0, 2, -1, 1, 2], 7, 3, dict(ranks=[7, 3, 5], behind=3, pad=24)),
    "ranks_to_zero": ([40, 40, 40], 80, 64, [0, 1, 2], 33, 3, dict(ranks=[0, -3, 400])),
    "rank_over_a_tile": ([40, 90], 130, 128, [1, 0], 100, 2, {}),
    "rank_200": ([200, 61], 256, 192, [0, 1], 200, 2, dict(ranks=[199, 65])),
    "no_scales": ([33, 20], 48, 64, [0, 1], 12, 2, dict(scales=False)),
    "k_zero": ([3, 5], 40, 0, [0, 1], 4, 2, {}),
    "before_and_behind": ([100, 28], 96, 128, [0, 1], 8, 2, dict(before=11, behind=40)),
    "decode_256": ([1] * 256, 1280, 640, [i % 7 - 1 for i in range(256)], 16, 6, {}),
    "short_1024": ([4] * 256, 1280, 640, [i % 5 for i in range(256)], 40, 5, {}),
    "many_requests": ([(i * 5) % 3 for i in range(300)], 72, 96, [i % 7 - 1 for i in range(300)], 8, 6, {}),
    "neighbours_share": ([10, 10, 10, 10, 10], 64, 64, [1, 1, 0, 0, 1], 8, 2, {}),
    "grouped_base": ([50, 7, 33, 64], 130, 192, [0, 1, 1, -1], 16, 2,
                     dict(groups=[30, 60, 64], weights=2, index=[1, 0, 1], n_kept=[130, 77])),
    "groups_end_early": ([50, 30], 65, 64, [0, 1], 8, 2, dict(groups=[20, 30], weights=2)),
    "large_tiles": ([2100, 1, 1998], 1280, 704, [1, 0, 1], 40, 2, dict(pad=8)),
    "wide": ([60, 200], 2100, 576, [0, 1], 64, 2, {}),
}


@pytest.mark.parametrize("types", TYPES, ids="_".join)
@pytest.mark.parametrize("epilogue", [STORE, GELU, RESIDUAL])
@pytest.mark.parametrize("case", LORA)
def test_lora(case, epilogue, types):
    rows, N, K, adapter, rank, adapters, more = LORA[case]
    say(f"lora {case} epilogue={epilogue} {types}")
    p = Problem(rows, N, K, epilogue, *types, adapter=adapter, rank=rank, adapters=adapters, seed=len(case), **more)
    p.check(p.run())


# ---------------------------------------------------------------------------
# what must not depend on how a launch is cut
# ---------------------------------------------------------------------------

def _with(p, **kw):
    import copy
    q = copy.copy(p)
    for k, v in kw.items():
        setattr(q, k, v)
    return q


@pytest.mark.parametrize("types", TYPES, ids="_".join)
def test_a_rows_bits_do_not_depend_on_its_batch(types):
    """The same 21 rows alone, in a batch of 5000 and in one of 40: other tiles, the
    same bits."""
    import torch
    say(f"grouped invariance {types}")
    for K in (64, 203, 1096):
        big = Problem([700, 21, 4279], 700, K, GELU, *types, weights=2, index=[0, 1, 0], seed=K)
        C = big.run()
        rows = big.A[700:721]
        for counts, at in (([21], 0), ([19, 21], 19)):
            q = Problem(counts, 700, K, GELU, *types, weights=2, index=[1] if at == 0 else [0, 1], seed=1)
            q.A[at:at + 21] = rows
            q = _with(q, B=big.B, bias=big.bias)
            assert torch.equal(q.run()[at:at + 21], C[700:721])


def test_one_group_gives_the_plain_products_bits():
    import torch

    from paper_2607_06631_amd import binding as B
    for M, N, K in ((5, 320, 640), (900, 1024, 512), (4100, 2048, 640)):
        say(f"grouped against dif_gemm {M} x {N} x {K}")
        p = Problem([M], N, K, GELU, seed=M)
        want = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
        B.dif_gemm(p.A, p.B[0], want, GELU, p.bias[0])
        assert torch.equal(p.run(), want)


# ---------------------------------------------------------------------------
# what must stay apart
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("types", TYPES, ids="_".join)
@pytest.mark.parametrize("rows", [[40, 24, 200, 24], [1, 1, 1, 1, 1, 1], [700, 600, 800]], ids=str)
def test_non_finite_adapters_stay_with_their_requests(rows, types):
    import torch
    say(f"lora non-finite {rows} {types}")
    R = len(rows)
    p = Problem(rows, 300, 160, STORE, *types, adapter=[i % 3 for i in range(R)], rank=12, adapters=3, seed=R)
    clean = p.run()
    for value in (float("nan"), float("inf")):
        for name in ("up", "down"):
            old = getattr(p, name)[1].clone()
            getattr(p, name)[1] = value
            got = p.run()
            getattr(p, name)[1] = old
            _, a = p.row_of()
            hit = (a == 1).to("cuda")
            assert torch.equal(got[~hit], clean[~hit])
            assert not bool(torch.isfinite(got[hit].float()).all(dim=1).any())


@pytest.mark.parametrize("types", TYPES, ids="_".join)
@pytest.mark.parametrize("rows", [[40, 24], [1, 1, 1, 1, 1, 1], [700, 600, 800]], ids=str)
def test_infinite_low_rank_factors_stay_infinite(rows, types):
    """One infinite entry among the factors of a row: infinities of the other factor's
    signs, as in real arithmetic, no NaN."""
    import torch
    say(f"lora infinite factors {rows} {types}")
    R = len(rows)
    p = Problem(rows, 300, 160, STORE, *types, adapter=[i % 2 for i in range(R)], rank=12, adapters=2, seed=R)
    p.A.copy_(p.A.abs() + 0.25)
    p.down[1, 5] = float("inf")
    p.up[1, :, 5] = torch.where(p.up[1, :, 5] < 0, -0.5, 0.5)
    got = p.run().double()
    _, a = p.row_of()
    hit = (a == 1).to("cuda")
    want = (p.up[1, :, 5].double() * p.scales[1].double()).sign() * float("inf")
    assert bool(torch.isfinite(got[~hit]).all()) and torch.equal(got[hit], want.expand(int(hit.sum()), -1))


@pytest.mark.parametrize("types", TYPES, ids="_".join)
def test_non_finite_rows_and_widths_past_the_kept_ones(types):
    """A row of NaN stays that row; what lies past a matrix's kept widths is not used."""
    import torch
    say(f"grouped non-finite {types}")
    p = Problem([65, 30, 200], 192, 328, RESIDUAL, *types, n_kept=[192, 50, 131], k_kept=[328, 64, 203], seed=3)
    want = p.run()
    at = 0
    for g, m in enumerate(p.rows):
        p.A[at:at + m, p.k_kept[g]:] = float("nan")
        p.B[g, :, p.k_kept[g]:] = float("inf")
        p.B[g, p.n_kept[g]:] = float("nan")
        p.bias[g, p.n_kept[g]:] = float("nan")
        at += m
    p.A[70] = float("inf")
    got = p.run()
    rows = torch.ones(p.M, dtype=torch.bool, device="cuda")
    rows[70] = False
    assert torch.equal(got[rows], want[rows])
    assert not bool(torch.isfinite(got[70, :50]).any()) and torch.equal(got[70, 50:], want[70, 50:])


# ---------------------------------------------------------------------------
# layouts and sizes
# ---------------------------------------------------------------------------

def test_offsets_past_32_bits():
    """Rows, matrices and adapters more than 2^31 elements apart."""
    import torch

    from paper_2607_06631_amd import binding as B
    say("grouped and lora, more than 2^31 elements apart")
    M, N, K, ld = 66000, 96, 64, 33000
    big = lambda: torch.empty(M, ld, dtype=torch.bfloat16, device="cuda")
    p = Problem([5, M - 12, 7], N, K, seed=9, weights=3)
    A, C = big()[:, :K], big()[:, 16:16 + N]
    A.copy_(p.A)
    C.copy_(p.C0)
    far = torch.empty(3, 1100000000, dtype=torch.bfloat16, device="cuda")   # matrices 1.1e9 elements apart
    W = far[:, :N * K].unflatten(1, (N, K))
    W.copy_(p.B)
    want = p.run()
    B.dif_gemm_grouped(A, W, C, p.tables()["row_offsets"], bias=p.bias)
    assert torch.equal(C, want)
    q = Problem([5, M - 12, 7], N, K, adapter=[2, 0, 1], rank=16, adapters=3, seed=10)
    A.copy_(q.A)
    C.copy_(q.C0)
    down, up = far[:, :16 * K].unflatten(1, (16, K)), far[:, 8192:8192 + N * 16].unflatten(1, (N, 16))
    down.copy_(q.down)
    up.copy_(q.up)
    want = q.run()
    ws = torch.empty(B.dif_lora_workspace_bytes(M, 16), dtype=torch.uint8, device="cuda")
    t = q.tables()
    B.dif_gemm_lora(A, q.B[0], C, t["row_offsets"], t["adapter"], down, up, ws, bias=q.bias, scales=q.scales)
    assert torch.equal(C, want)


def test_strided_operands():
    """Rows, matrices and adapters with gaps, output columns at an odd offset, vectors
    shared by all matrices."""
    import torch

    from paper_2607_06631_amd import binding as B
    say("grouped strided")
    p = Problem([30, 50], 100, 72, seed=4, weights=2)
    A = torch.zeros(80, 3, 96, dtype=torch.bfloat16, device="cuda")[:, 1, 8:80]
    W = torch.zeros(2, 2, 100, 88, dtype=torch.bfloat16, device="cuda")[:, 1, :, 16:88]
    room = torch.zeros(80, 211, dtype=torch.bfloat16, device="cuda")
    C = room[:, 7:107]
    A.copy_(p.A)
    W.copy_(p.B)
    C.copy_(p.C0)
    p.bias[1] = p.bias[0]
    B.dif_gemm_grouped(A, W, C, p.tables()["row_offsets"], bias=p.bias[0])
    assert torch.equal(C, p.run())
    assert bool((room[:, :7] == 0).all()) and bool((room[:, 107:] == 0).all())


@pytest.mark.parametrize("table", [[-5, 10, 3, 1 << 30, 40], [1 << 30, -7, 90, 20, 20], [60, 50, 40, 30, 20],
                                   [0, 90, 0, 90, 0], [-(1 << 31), (1 << 31) - 1, -1, 5, 1 << 20]], ids=str)
def test_tables_that_are_not_ascending_stay_inside_the_operands(table):
    """Every access is clamped to the operands: whatever the rows then hold, nothing
    around C changes, and the next call is right."""
    import torch

    from paper_2607_06631_amd import binding as B
    say(f"bad offsets {table}")
    p = Problem([30, 20, 20, 20], 70, 96, seed=11, weights=2, index=[0, 1, 1, 0], n_kept=[70, -3], k_kept=[1 << 30, 40])
    q = Problem([30, 20, 20, 20], 70, 96, adapter=[0, 7, -9, 1], rank=9, adapters=2, ranks=[1 << 30, -4], seed=12)
    off = torch.tensor(table, dtype=torch.int32, device="cuda")
    for x in (p, q):
        room = torch.full((x.M + 40, 90), 3.0, dtype=torch.bfloat16, device="cuda")
        x.run(C=room[20:-20, 10:80], row_offsets=off)
        edge = room.clone()
        edge[20:-20, 10:80] = 3.0
        assert bool((edge == 3.0).all())
        x.check(x.run())


def test_most_groups():
    say("4096 groups and requests")
    rows = [(i * 13) % 4 for i in range(4096)]
    p = Problem(rows, 40, 64, weights=7, index=[i % 7 for i in range(4096)], seed=6)
    p.check(p.run())
    q = Problem(rows, 40, 64, adapter=[i % 9 - 1 for i in range(4096)], rank=8, adapters=8, seed=7)
    q.check(q.run())


def test_more_small_tiles_than_a_launch_holds():
    """4096 groups of a row each on 131,100 columns: 2^24 tiles of 32 x 32 would be
    2^32 threads."""
    import torch

    from paper_2607_06631_amd import binding as B
    say("grouped, 4096 x 131100 in 4096 groups")
    M, N, K = 4096, 131100, 64
    a = torch.randn(M, K, device="cuda").bfloat16()
    w = torch.randn(1, N, K, device="cuda").bfloat16()
    got, want = (torch.zeros(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.dif_gemm_grouped(a, w, got, torch.arange(M + 1, dtype=torch.int32, device="cuda"),
                       weight_index=torch.zeros(M, dtype=torch.int32, device="cuda"))
    B.dif_gemm(a, w[0], want)
    assert torch.equal(got, want)


def test_empty_calls():
    import torch
    for M, N in ((0, 64), (5, 0)):
        say(f"grouped empty {M} x {N}")
        p = Problem([M], N, 64, weights=1, seed=1)
        assert p.run().shape == (M, N)
    q = Problem([0], 64, 64, adapter=[0], rank=8, adapters=1, seed=1)
    assert q.run(ws=torch.empty(0, dtype=torch.uint8, device="cuda")).shape == (0, 64)


# ---------------------------------------------------------------------------
# streams, graphs, a batch as it is served
# ---------------------------------------------------------------------------

def test_two_streams_with_their_own_workspaces():
    import torch

    from paper_2607_06631_amd import binding as B
    say("lora on two streams")
    p = Problem([300, 200, 77], 512, 320, GELU, adapter=[0, 1, 2], rank=16, adapters=3, seed=1)
    q = Problem([1] * 20, 512, 4096, RESIDUAL, adapter=[i % 3 for i in range(20)], rank=16, adapters=3, seed=2)
    want = [x.run() for x in (p, q)]
    # everything the calls read stands, and is kept, before the streams begin
    calls = []
    for x in (p, q):
        ws = torch.full((B.dif_lora_workspace_bytes(x.M, x.rank),), 255, dtype=torch.uint8, device="cuda")
        calls.append((x, ws, x.tables(), [x.fresh() for _ in range(6)], torch.cuda.Stream()))
    torch.cuda.synchronize()
    for i in range(6):
        for x, ws, tables, outs, stream in calls:
            B.dif_gemm_lora(x.A, x.B, outs[i], down=x.down, up=x.up, ws=ws, scales=x.scales, bias=x.bias, gate0=x.gate0,
                            gate1=x.gate1, epilogue=x.epi, stream=stream, **tables)
    torch.cuda.synchronize()
    for (x, _, _, outs, _), y in zip(calls, want):
        assert all(torch.equal(C, y) for C in outs)


def test_captured_calls_follow_their_tables():
    """A graph of both calls, replayed with other splits, adapters and widths in the
    tables, other inputs, and eager work in between."""
    import torch

    from paper_2607_06631_amd import binding as B
    say("mixed batch under graph capture")
    M, N, K, R = 640, 384, 200, 5
    g = Problem([128] * 5, N, K, GELU, weights=3, index=[0, 1, 2, 0, 1], n_kept=[N] * 3, k_kept=[K] * 3, seed=1)
    l = Problem([128] * 5, N, K, RESIDUAL, adapter=[0, 1, 2, 3, -1], rank=20, adapters=4, ranks=[20] * 4, seed=2)
    gt, lt = g.tables(), l.tables()
    Cg, Cl = g.fresh(), l.fresh()
    ws = torch.empty(B.dif_lora_workspace_bytes(M, 20), dtype=torch.uint8, device="cuda")
    gk = dict(gt, epilogue=GELU, bias=g.bias)
    lk = dict(adapter=lt["adapter"], ranks=lt["ranks"], scales=l.scales, epilogue=RESIDUAL, bias=l.bias, gate0=l.gate0,
              gate1=l.gate1)

    def both():
        B.dif_gemm_grouped(g.A, g.B, Cg, **gk)
        B.dif_gemm_lora(l.A, l.B, Cl, lt["row_offsets"], down=l.down, up=l.up, ws=ws, **lk)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for i, rows in enumerate(([128] * 5, [1, 0, 600, 20, 3], [0, 0, 0, 0, 0], [640, 0, 0, 0, 0], [200, 100, 50, 25, 12])):
        n_kept, k_kept = [N, 7 * i + 1, N - i], [K, K - 3 * i, 64 + i]
        index, adapter, ranks = [(i + j) % 3 for j in range(5)], [(i * j) % 6 - 1 for j in range(5)], [20, i, 3 * i, 8]
        off = torch.tensor([0] + [sum(rows[:j + 1]) for j in range(5)], dtype=torch.int32, device="cuda")
        gt["row_offsets"].copy_(off)
        lt["row_offsets"].copy_(off)
        for t, v in ((gt["n_kept"], n_kept), (gt["k_kept"], k_kept), (gt["weight_index"], index),
                     (lt["adapter"], adapter), (lt["ranks"], ranks)):
            t.copy_(torch.tensor(v, dtype=torch.int32, device="cuda"))
        g.A.copy_(g.rand((M, K)))
        l.A.copy_(l.rand((M, K)))
        Cg.copy_(g.C0)
        Cl.copy_(l.C0)
        graph.replay()
        torch.cuda.synchronize()
        gq = _with(g, rows=rows, groups=rows, index=index, n_kept=n_kept, k_kept=k_kept)
        lq = _with(l, rows=rows, adapter=adapter, ranks=ranks)
        gq.check(Cg)
        lq.check(Cl)
        eager_g, eager_l = gq.run(), lq.run()
        torch.cuda.synchronize()
        assert torch.equal(Cg, eager_g) and torch.equal(Cl, eager_l)


def test_an_ffn_of_requests_at_three_steps_with_adapters():
    """The two products of a block's FFN as a mixed batch runs them: rows grouped by
    step, whose structures keep their own channels, and each request's adapter beside
    the first; against float64 on the values in between as they are stored."""
    import torch

    from paper_2607_06631_amd import binding as B
    say("mixed batch FFN")
    D, F, kept = 256, 1024, [1024, 640, 413]
    rows, steps = [128, 77, 1, 200], [128 + 77, 1, 200]
    up = Problem(rows, F, D, GELU, adapter=[0, -1, 1, 0], rank=8, adapters=2, groups=steps, weights=3,
                 index=[2, 0, 1], n_kept=kept, seed=5)
    h = up.run()
    up.check(h)
    down = Problem(steps, D, F, RESIDUAL, weights=3, index=[2, 0, 1], k_kept=kept, seed=6)
    x = torch.randn(sum(rows), D, device="cuda").bfloat16()
    down = _with(down, A=h, C0=x)
    y = x.clone()
    B.dif_gemm_grouped(h, down.B, y, down.tables()["row_offsets"], RESIDUAL, bias=down.bias, gate0=down.gate0,
                       gate1=down.gate1, weight_index=down.tables()["weight_index"], k_kept=down.tables()["k_kept"])
    down.check(y)
