"""The products of a mixed batch: what a server needs once the rows of one launch
no longer share one matrix.

Requests of a batch stand at different sampler steps, whose structures keep
different heads and channels, and bring adapters of their own.  Two operators
cover that, both beside the plain product:

  grouped  rows in groups, a matrix (of its own kept widths) per group
  lora     a low-rank term per request beside the product that all share,
           or beside a grouped one

  listed()            the named cases
  draw(rng)           one more case of the same ranges
  prepare(case, seed) what a program holds before the call
  run(state)          one pass; returns its outputs
  work(case)          bytes and flops one pass cannot do without
  exact(case, seed)   what run() returns, in float64

Lists inside a case are texts of whole numbers with commas between them.
"""
import math

import torch

own = False

STORE, GELU, RESIDUAL = 0, 1, 2


def _ints(text):
    return [int(x) for x in text.split(",")] if text else []


def _text(values):
    return ",".join(str(int(v)) for v in values)


def _grouped(name, rows, n, k, epilogue=STORE, dtype="bf16", out=None, weights=None, index="", n_kept="",
             k_kept="", behind=0, pad=0):
    """rows: of each group; index: each group's matrix (its own number by default);
    n_kept, k_kept: each matrix's widths; behind: rows after the last group; pad:
    elements between the rows of A, of the matrices and of C beyond their widths."""
    c = dict(kind="grouped", rows=rows, n=n, k=k, epilogue=epilogue, dtype=dtype, out=out or dtype,
             weights=weights or len(_ints(rows)), index=index, n_kept=n_kept, k_kept=k_kept, behind=behind, pad=pad)
    if name:
        c["name"] = name
    return c


def _lora(name, rows, n, k, adapter, rank, adapters, ranks="", epilogue=STORE, dtype="bf16", out=None, behind=0,
          pad=0, groups="", weights=1, index=""):
    """rows: of each request; adapter: each request's (-1: none); ranks: each
    adapter's rank (all `rank` by default); groups: rows of each group where the
    base product is a grouped one, with index as above."""
    c = dict(kind="lora", rows=rows, n=n, k=k, adapter=adapter, rank=rank, adapters=adapters, ranks=ranks,
             epilogue=epilogue, dtype=dtype, out=out or dtype, behind=behind, pad=pad, groups=groups,
             weights=weights, index=index)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # The tiny float32 stack, a request at each of the four steps, FFN's first
        # half with the steps' own channels: launch and latency only.
        _grouped("grouped_tiny_f32", "128,128,128,128", 1024, 256, GELU, dtype="f32", n_kept="1024,768,640,512"),
        # Single rows: 24 tokens routed to 16 matrices of the 1.3B FFN, three of them
        # without any.  Reading the matrices is all there is.
        _grouped("grouped_single_rows", "1,2,0,1,3,1,1,0,4,1,2,1,0,3,2,2", 8960, 1536),
        # q, k and v of still pictures (1560 tokens) at the 1.3B width, five requests
        # at four steps whose structures keep 12, 10, 9 and 7 of the 12 heads.
        _grouped("grouped_qkv_1.3b_stills", "1560,1560,1560,1560,1560", 4608, 1536, weights=4, index="0,1,1,2,3",
                 n_kept="4608,3840,3456,2688"),
        # FFN's first half at the 14B width, stills at four steps: per-channel kept
        # counts, which are no multiple of anything.
        _grouped("grouped_ffn1_14b_stills", "1560,1560,1560,1560", 13824, 5120, GELU,
                 n_kept="13824,11059,9677,8294"),
        # Its second half: the same counts shorten the reduction; gated residual.
        _grouped("grouped_ffn2_14b_stills", "1560,1560,1560,1560", 5120, 13824, RESIDUAL,
                 k_kept="13824,11059,9677,8294"),
        # Two 480x832, 81-frame videos at two steps, attention output projection at
        # the 14B width (40 and 32 heads).  The largest case.
        _grouped("grouped_out_14b_480p", "32760,32760", 5120, 5120, k_kept="5120,4096"),
        # Odd in everything: ragged groups (one empty, one of a single row), widths,
        # padded rows, rows behind the last group, float32 output.
        _grouped("grouped_ragged", "777,1,0,2049,390", 1999, 1543, out="f32", n_kept="1999,1500,7,1811,1024",
                 k_kept="1543,64,1500,1001,1543", behind=37, pad=24),
        # One row of each of 16 requests, each with its own rank-16 adapter, beside
        # a 14B projection: the single-token form.
        _lora("lora_single_rows", _text([1] * 16), 5120, 5120, _text(range(16)), 16, 16),
        # The tiny float32 stack with odd ranks, a request without adapter.
        _lora("lora_tiny_f32", "128,77,1,128", 768, 256, "0,-1,2,1", 7, 3, ranks="7,4,5", dtype="f32"),
        # Stills, thumbnails and odd crops of eight requests beside the shared q
        # projection at the 14B width; ranks 8 to 64, two requests share an adapter,
        # two have none.
        _lora("lora_q_14b_stills", "1560,390,1560,0,391,1,1560,780", 5120, 5120, "0,1,-1,2,3,3,1,-1", 64, 4,
              ranks="64,16,8,32", behind=20),
        # FFN's second half at the 14B width for a 480p clip of nine frames and a
        # still, gated residual, rank 32.
        _lora("lora_ffn2_14b_clip", "14040,1560", 5120, 13824, "0,1", 32, 2, epilogue=RESIDUAL),
        # Both at once: FFN's first half at the 1.3B width, stills at three steps
        # with a matrix each and five requests' adapters, GELU behind the sum.
        _lora("lora_grouped_ffn1_1.3b", "1560,1560,390,1560,1171", 8960, 1536, "2,0,1,-1,0", 24, 3, epilogue=GELU,
              groups="3120,390,2731", weights=3, index="1,2,0"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _split(rng, total, parts):
    """`total` rows in `parts` uneven runs, some of them empty or of one row."""
    left, out = total, []
    for i in range(parts - 1):
        u = rng.random()
        r = 0 if u < 0.12 else 1 if u < 0.24 else int(left * rng.random() * 2.0 / (parts - i))
        r = min(r, left)
        out.append(r)
        left -= r
    out.append(left)
    rng.shuffle(out)
    return out


MOST = {"bf16": 3.0e12, "f32": 3.0e11}   # flops of a drawn case


def draw(rng):
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    out = rng.choice((dtype, dtype, "f32"))
    epilogue = rng.choice((STORE, GELU, RESIDUAL))
    while True:
        n, k = _log_int(rng, 48, 13824), _log_int(rng, 48, 13824)
        if rng.random() < 0.6:
            n, k = max(64, n // 64 * 64), max(64, k // 64 * 64)
        total = _log_int(rng, 1, 40000)
        if 2.0 * total * n * k <= MOST[dtype] / 4:
            break
    behind, pad = rng.choice((0, 0, rng.randint(1, 60))), rng.choice((0, 0, 8, 40))
    parts = rng.randint(1, 16)
    rows = _text(_split(rng, total, parts))
    if rng.random() < 0.5:
        weights = rng.choice((parts, parts, rng.randint(1, 8)))
        index = "" if weights == parts else _text(rng.randrange(weights) for _ in range(parts))
        kept = lambda full: _text(rng.randint(max(1, full // 3), full) for _ in range(weights))
        return _grouped(None, rows, n, k, epilogue, dtype, out, weights, index,
                        kept(n) if rng.random() < 0.5 else "", kept(k) if rng.random() < 0.5 else "", behind, pad)
    adapters, rank = rng.randint(1, 8), _log_int(rng, 1, 128)
    adapter = _text(rng.randint(-1, adapters - 1) for _ in range(parts))
    ranks = _text(rng.randint(max(1, rank // 4), rank) for _ in range(adapters)) if rng.random() < 0.5 else ""
    groups, weights, index = "", 1, ""
    if rng.random() < 0.3:
        runs, weights = rng.randint(1, 4), rng.randint(1, 4)
        groups, index = _text(_split(rng, total, runs)), _text(rng.randrange(weights) for _ in range(runs))
    return _lora(None, rows, n, k, adapter, rank, adapters, ranks, epilogue, dtype, out, behind, pad, groups,
                 weights, index)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


class _Draws:
    """Seeded tensors on the GPU, each from a stream of its own."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.seed, self.n = seed, 0

    def __call__(self, shape, std=1.0, dtype=torch.float32, pad=0):
        """pad: the last dimension's rows lie that many elements further apart, up
        to whole 16-byte pieces."""
        self.gen.manual_seed(self.seed * 1000003 + self.n)
        self.n += 1
        width, vec = shape[-1], 16 // torch.empty(0, dtype=dtype).element_size()
        ld = -(-(width + pad) // vec) * vec
        t = torch.empty((*shape[:-1], ld), dtype=dtype, device="cuda")
        if t.dim() == 3:   # (matrix by matrix: the float32 numbers before the rounding are large)
            for m in t:
                m.copy_(torch.randn(m.shape, generator=self.gen, device="cuda").mul_(std))
        else:
            t.copy_(torch.randn(t.shape, generator=self.gen, device="cuda").mul_(std))
        return t[..., :width]


def _offsets(counts):
    out = [0]
    for c in counts:
        out.append(out[-1] + c)
    return out


def _table(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda") if len(values) else None


def _inputs(c, seed):
    """Activations as a norm leaves them (unit scale), matrices as in the models'
    initialisation, adapters whose term is a tenth to a half of the product."""
    draws, d = _Draws(seed), _dtype(c["dtype"])
    rows, n, k = _ints(c["rows"]), c["n"], c["k"]
    m = sum(rows) + c["behind"]
    s = {"case": c, "rows": rows}
    s["a"] = draws((m, k), dtype=d, pad=c["pad"])
    s["b"] = draws((c["weights"], n, k), 0.02, dtype=d, pad=c["pad"])
    s["bias"] = draws((c["weights"], n), 0.02).contiguous()
    if c["epilogue"] == RESIDUAL:
        s["gate0"], s["gate1"] = draws((n,), 0.1).contiguous(), draws((c["weights"], n), 0.5).contiguous()
    else:
        s["gate0"] = s["gate1"] = None
    s["c0"] = draws((m, n), dtype=_dtype(c["out"]), pad=c["pad"])
    if c["kind"] == "lora":
        s["down"] = draws((c["adapters"], c["rank"], k), 1.0 / math.sqrt(k), dtype=d)
        s["up"] = draws((c["adapters"], n, c["rank"]), 0.05, dtype=d)
        s["scales"] = (0.5 + draws((c["adapters"],)).abs()).contiguous()
    return s


def _plan(c):
    """What a program knows of its batch on the host: each group's first and last
    row, matrix and kept widths; each request's rows, adapter and rank."""
    if c["kind"] == "grouped":
        off = _offsets(_ints(c["rows"]))
        index = _ints(c["index"]) or list(range(len(off) - 1))
    else:
        off = _offsets(_ints(c["groups"]) or [sum(_ints(c["rows"]))])
        index = _ints(c["index"]) or list(range(len(off) - 1))
    nk = _ints(c.get("n_kept", "")) or [c["n"]] * c["weights"]
    kk = _ints(c.get("k_kept", "")) or [c["k"]] * c["weights"]
    groups = [(off[i], off[i + 1], w, nk[w], kk[w]) for i, w in enumerate(index)]
    requests = []
    if c["kind"] == "lora":
        off = _offsets(_ints(c["rows"]))
        ranks = _ints(c["ranks"]) or [c["rank"]] * c["adapters"]
        requests = [(off[i], off[i + 1], a, ranks[a] if a >= 0 else 0) for i, a in enumerate(_ints(c["adapter"]))]
    return groups, requests


def prepare(c, seed):
    s = _inputs(c, seed)
    s["groups"], s["requests"] = _plan(c)
    s["c"] = s["c0"].clone() if not c["pad"] else torch.empty_strided(
        s["c0"].shape, s["c0"].stride(), dtype=s["c0"].dtype, device="cuda").copy_(s["c0"])
    # the same tables on the device
    s["offsets"] = _table(_offsets(s["rows"]))
    s["index"] = _table(_ints(c["index"]))
    s["n_kept"], s["k_kept"] = _table(_ints(c.get("n_kept", ""))), _table(_ints(c.get("k_kept", "")))
    if c["kind"] == "lora":
        s["adapter"], s["ranks"] = _table(_ints(c["adapter"])), _table(_ints(c["ranks"]))
        s["group_offsets"] = _table(_offsets(_ints(c["groups"]))) if c["groups"] else None
        if own:
            from paper_2607_06631_amd import binding as B
            s["ws"] = torch.empty(B.dif_lora_workspace_bytes(s["a"].shape[0], c["rank"]), dtype=torch.uint8,
                                  device="cuda")
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    c = s["case"]
    if c["epilogue"] == RESIDUAL:   # updates its output in place
        s["c"].copy_(s["c0"])
    if own:
        return _run_own(s, c)
    out = s["c"]
    for lo, hi, w, n, k in s["groups"]:
        if lo == hi:
            continue
        x = s["a"][lo:hi, :k].float()
        y = x @ s["b"][w, :n, :k].float().t()
        for qlo, qhi, a, r in s["requests"]:
            qlo, qhi = max(qlo, lo), min(qhi, hi)
            if a < 0 or qlo >= qhi:
                continue
            t = x[qlo - lo:qhi - lo] @ s["down"][a, :r].float().t()
            y[qlo - lo:qhi - lo] += (t * s["scales"][a]) @ s["up"][a, :, :r].float().t()
        y += s["bias"][w, :n]
        if c["epilogue"] == GELU:
            y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
        if c["epilogue"] == RESIDUAL:
            y = out[lo:hi, :n].float() + (s["gate0"][:n] + s["gate1"][w, :n]) * y
        out[lo:hi, :n] = y.to(out.dtype)
    return out


def _run_own(s, c):
    from paper_2607_06631_amd import binding as B
    if c["kind"] == "grouped":
        B.dif_gemm_grouped(s["a"], s["b"], s["c"], s["offsets"], c["epilogue"], bias=s["bias"], gate0=s["gate0"],
                           gate1=s["gate1"], weight_index=s["index"], n_kept=s["n_kept"], k_kept=s["k_kept"])
    else:
        B.dif_gemm_lora(s["a"], s["b"], s["c"], s["offsets"], s["adapter"], s["down"], s["up"], s["ws"],
                        c["epilogue"], bias=s["bias"], gate0=s["gate0"], gate1=s["gate1"], ranks=s["ranks"],
                        scales=s["scales"], group_offsets=s["group_offsets"], weight_index=s["index"])
    return s["c"]


# ---------------------------------------------------------------------------
# accounting
# ---------------------------------------------------------------------------

def work(c):
    es, eo = (2 if c["dtype"] == "bf16" else 4), (2 if c["out"] == "bf16" else 4)
    groups, requests = _plan(c)
    by = fl = 0.0
    seen = {}
    for lo, hi, w, n, k in groups:
        m = hi - lo
        if not m:
            continue
        fl += 2.0 * m * n * k
        by += es * m * k + eo * m * n * (2 if c["epilogue"] == RESIDUAL else 1)
        seen[w] = es * n * k + 4.0 * n * (2 if c["epilogue"] == RESIDUAL else 1)
    by += sum(seen.values())
    used = {}
    for lo, hi, a, r in requests:
        if a >= 0 and hi > lo:
            fl += 2.0 * (hi - lo) * r * (c["k"] + c["n"])
            used[a] = es * r * (c["k"] + c["n"])
    return {"bytes": by + sum(used.values()), "flops": fl}


# ---------------------------------------------------------------------------
# the same in float64, row block by row block from the definition
# ---------------------------------------------------------------------------

def exact(c, seed):
    s = _inputs(c, seed)
    out = s["c0"].double()
    rank_of = _ints(c.get("ranks", ""))
    if c["kind"] == "grouped":
        runs, adapter_of = _ints(c["rows"]), None
    else:
        runs, adapter_of = _ints(c["groups"]) or [sum(_ints(c["rows"]))], []
        for q, a in zip(_ints(c["rows"]), _ints(c["adapter"])):
            adapter_of += [a] * q
        adapter_of = torch.tensor(adapter_of + [-1] * c["behind"], device="cuda")
    which, n_of, k_of = _ints(c["index"]), _ints(c.get("n_kept", "")), _ints(c.get("k_kept", ""))
    at = 0
    for g, m in enumerate(runs):
        w = which[g] if which else g
        n, k = n_of[w] if n_of else c["n"], k_of[w] if k_of else c["k"]
        bt = s["b"][w].double()[:n, :k].t().contiguous()
        for r0 in range(at, at + m, 8192):
            r1 = min(r0 + 8192, at + m)
            xs = s["a"][r0:r1, :k].double()
            acc = torch.mm(xs, bt)
            if adapter_of is not None:
                for a in range(c["adapters"]):
                    mine = (adapter_of[r0:r1] == a).nonzero().flatten()
                    if mine.numel():
                        r = rank_of[a] if rank_of else c["rank"]
                        low = torch.mm(xs[mine], s["down"][a, :r].double().t().contiguous())
                        low = torch.mm(low, s["up"][a, :, :r].double().t().contiguous())
                        acc[mine] += low * s["scales"][a].double()
            acc += s["bias"][w, :n].double()
            if c["epilogue"] == GELU:
                acc = acc / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (acc + 0.044715 * acc ** 3)))
            if c["epilogue"] == RESIDUAL:
                acc = out[r0:r1, :n] + (s["gate0"][:n].double() + s["gate1"][w, :n].double()) * acc
            out[r0:r1, :n] = acc
        at += m
    return out
