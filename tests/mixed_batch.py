"""Problems, float64 references and error bounds of the mixed-batch products.

The bound counts roundings.  A float32 sum of n products is off by at most n + 2
roundings of half a step, 2^-24 each, relative to the sum of the magnitudes; 2^-23
is taken, since the matrix cores do not promise round-to-nearest inside an
instruction.  The low-rank factor enters as two bf16 terms (three for float32
output), which leave at most 2^-16 (2^-24) of it.  GELU's slope is at most 1.13 and
its exponential and reciprocal cost a few 2^-22 of the value.  The last rounding is
half a step of the output type, 2^-8 (bf16) or 2^-24 relative.
"""
import math

import torch

U32 = 2.0 ** -23
STORE, GELU, RESIDUAL = 0, 1, 2


def dtype_of(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def offsets(counts, device):
    o = [0]
    for c in counts:
        o.append(o[-1] + c)
    return torch.tensor(o, dtype=torch.int32, device=device)


class Problem:
    """rows: of groups (grouped) or of requests (lora); `behind` rows follow.  All
    matrices are views of larger, NaN-filled storage: reading beyond them shows."""

    def __init__(self, rows, N, K, epilogue=STORE, dtype="bf16", out=None, weights=None, index=None, n_kept=None,
                 k_kept=None, adapter=None, rank=0, adapters=0, ranks=None, scales=True, groups=None, behind=0,
                 before=0, pad=0, bias=True, gates=2, seed=0, device="cuda"):
        self.rows, self.N, self.K, self.epi, self.dtype, self.out = rows, N, K, epilogue, dtype, out or dtype
        self.before, self.device = before, device
        self.M = before + sum(rows) + behind
        self.lora = adapter is not None
        self.groups = groups if self.lora else rows
        self.W = weights or (len(self.groups) if self.groups is not None else 1)
        self.index, self.n_kept, self.k_kept = index, n_kept, k_kept
        self.adapter, self.rank, self.adapters, self.ranks = adapter, rank, adapters, ranks
        self.gen = torch.Generator(device=device).manual_seed(1000 + seed)
        T, O = dtype_of(dtype), dtype_of(self.out)
        self.A = self.matrix((self.M, K), 1.0, T, pad)
        self.B = self.matrix((self.W, N, K), 1.0 / math.sqrt(max(K, 1)), T, pad)
        self.bias = self.rand((self.W, N)) if bias else None
        self.gate0 = self.rand((N,)) if epilogue == RESIDUAL and gates > 0 else None
        self.gate1 = self.rand((self.W, N)) if epilogue == RESIDUAL and gates > 1 else None
        self.C0 = self.matrix((self.M, N), 1.0, O, pad + 1 if pad else 0, align=1)
        if self.lora:
            self.down = self.matrix((adapters, rank, K), 1.0 / math.sqrt(max(K, 1)), T, pad)
            self.up = self.matrix((adapters, N, rank), 1.0 / math.sqrt(rank), T, pad)
            self.scales = self.rand((adapters,)) if scales else None

    def rand(self, shape):
        return torch.randn(shape, generator=self.gen, device=self.device)

    def matrix(self, shape, std, dtype, pad, align=None):
        vec = align or 16 // torch.empty(0, dtype=dtype).element_size()
        width = shape[-1]
        ld = max(vec, -(-(width + pad) // vec) * vec)
        t = torch.full((*shape[:-1], ld), float("nan"), dtype=dtype, device=self.device)
        t[..., :width] = self.rand(shape).mul_(std).to(dtype)
        return t[..., :width]

    # what row r is: (matrix or -1, adapter or -1)
    def row_of(self):
        w, a = [-1] * self.M, [-1] * self.M
        requests = [False] * self.M
        groups = self.groups if self.groups is not None else [self.M - self.before]
        at = self.before
        for g, m in enumerate(groups):
            wi = self.index[g] if self.index is not None else g
            for r in range(at, at + m):
                w[r] = wi if 0 <= wi < self.W else -1
            at += m
        if self.lora:
            at = self.before
            for q, m in enumerate(self.rows):
                ai = self.adapter[q]
                for r in range(at, at + m):
                    a[r] = ai if 0 <= ai < self.adapters else -1
                    requests[r] = True
                at += m
            w = [x if y else -1 for x, y in zip(w, requests)]
        return torch.tensor(w), torch.tensor(a)

    def reference(self):
        """(value, bound) in float64; rows and columns left alone keep C0, bound 0."""
        ref, bound = self.C0.double().clone(), torch.zeros_like(self.C0, dtype=torch.float64)
        ws, as_ = self.row_of()
        half = 2.0 ** -8 if self.out == "bf16" else 2.0 ** -24
        kept_bits = 2.0 ** -16 if self.out == "bf16" else 2.0 ** -24
        for w in range(self.W):
            n = min(max(self.n_kept[w], 0), self.N) if self.n_kept is not None else self.N
            k = min(max(self.k_kept[w], 0), self.K) if self.k_kept is not None else self.K
            bt = self.B[w, :n, :k].double().t().contiguous()
            for a in range(-1, self.adapters):
                r = ((ws == w) & (as_ == a)).nonzero().flatten().to(self.device)
                if not r.numel() or not n:
                    continue
                x = self.A[r][:, :k].double()
                y, s = x @ bt, x.abs() @ bt.abs()
                err = U32 * (k + 2) * s
                if a >= 0:
                    j = min(max(self.ranks[a], 0), self.rank) if self.ranks is not None else self.rank
                    sc = self.scales[a].double() if self.scales is not None else 1.0
                    d, u = self.down[a, :j].double().t().contiguous(), self.up[a, :n, :j].double().t().contiguous()
                    low, mag = x @ d * sc, x.abs() @ d.abs() * abs(sc)
                    elow = U32 * (k + 3) * mag + kept_bits * low.abs() if self.dtype == "bf16" else U32 * (k + 3) * mag
                    t = low.abs() @ u.abs()
                    y, s = y + low @ u, s + t
                    err += elow @ u.abs() + U32 * (j + 3) * t
                b = self.bias[w, :n].double() if self.bias is not None else torch.zeros(n, dtype=torch.float64,
                                                                                        device=self.device)
                y = y + b
                err += U32 * (s + b.abs())
                if self.epi == GELU:
                    inner = math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)
                    err = 1.13 * err + 2.0 ** -18 * y.abs()
                    y = 0.5 * y * (1 + torch.tanh(inner))
                if self.epi == RESIDUAL:
                    g = torch.ones(n, dtype=torch.float64, device=self.device)
                    if self.gate0 is not None:
                        g = self.gate0[:n].double()
                        if self.gate1 is not None:
                            g = g + self.gate1[w, :n].double()
                    gm = self.gate0[:n].double().abs() + (self.gate1[w, :n].double().abs() if self.gate1 is not None
                                                          else 0) if self.gate0 is not None else g
                    err = g.abs() * err + U32 * (gm * y.abs() + g.abs() * y.abs())
                    y = self.C0[r][:, :n].double() + g * y
                    err += U32 * y.abs()
                ref[r, :n] = y
                bound[r, :n] = err + half * (y.abs() + err)
        return ref, bound

    def tables(self):
        d = self.device
        t = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device=d)
        shift = lambda o: o + self.before
        k = dict(weight_index=t(self.index), n_kept=t(self.n_kept))
        if not self.lora:
            k.update(row_offsets=shift(offsets(self.rows, d)), k_kept=t(self.k_kept))
        else:
            k.update(row_offsets=shift(offsets(self.rows, d)), adapter=t(self.adapter), ranks=t(self.ranks),
                     group_offsets=None if self.groups is None else shift(offsets(self.groups, d)))
        return k

    def run(self, C=None, ws=None, stream=None, **replace):
        """One call through the public entry point; returns the output tensor."""
        from paper_2607_06631_amd import binding as B
        if C is None:
            C = self.fresh()
        k = dict(self.tables(), bias=self.bias, gate0=self.gate0, gate1=self.gate1, epilogue=self.epi, stream=stream)
        k.update(replace)
        if not self.lora:
            B.dif_gemm_grouped(self.A, self.B, C, **k)
        else:
            if ws is None:
                ws = torch.full((B.dif_lora_workspace_bytes(self.M, self.rank),), 255, dtype=torch.uint8,
                                device=self.device)
            B.dif_gemm_lora(self.A, self.B, C, down=self.down, up=self.up, ws=ws, scales=self.scales, **k)
        return C

    def fresh(self):
        C = torch.empty_strided(self.C0.shape, self.C0.stride(), dtype=self.C0.dtype, device=self.device)
        return C.copy_(self.C0)

    def check(self, C, ref=None):
        value, bound = ref if ref is not None else self.reference()
        got = C.double()
        assert bool(torch.isfinite(got).all())
        left = bound == 0
        assert torch.equal(got[left], value[left]), "left-alone entries changed"
        over = (got - value).abs() - bound
        worst = over.max().item() if over.numel() else 0.0
        assert worst <= 0.0, (worst, (got - value).abs().max().item(), bound.max().item())
