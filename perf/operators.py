"""Timed calls of the operators that read and write 4-bit codes, with their inputs, work and plain forms.

A case is a dict of plain values: its "kind" names the operator, the rest its sizes and types.
listed() gives twelve of them, draw() more of the same ranges; prepare() makes what a program
has in hand before the call, run() is one call, exact() the same outputs from the definitions
in 64 bits.  Where `own` is false run() computes them from elementary torch operations in 32 bits.

matvec  y = x W^T, W[n, k] = scale[n, k div group] * levels[code[n, k]], 4-bit codes
attend  attention of one new token a sequence over a paged cache of plain or coded rows
write   stochastic rounding of new cache rows to 4 bits with a codebook a row, into the pages
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "f16": 2, "bf16": 2}
GAMMA, MUL1, MUL2 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB  # SplitMix64


def listed():
    return [
        # A small projection of one token: launch and latency.
        dict(name="matvec_1024x1024_b1_bf16", kind="matvec", n=1024, k=1024, b=1, group=128, dtype="bf16", scales="f32"),
        # One token through a square projection, fine groups.
        dict(name="matvec_8192x8192_b1_f16", kind="matvec", n=8192, k=8192, b=1, group=64, dtype="f16", scales="f16"),
        # Ragged matrix, a few sequences decoded together, the finest groups; a last group that is cut short.
        dict(name="matvec_5003x4097_b5_bf16", kind="matvec", n=5003, k=4097, b=5, group=32, dtype="bf16", scales="bf16"),
        # Single-precision activations, as the solver's own vectors are; a group size that is no power of two.
        dict(name="matvec_2999x2050_b3_f32", kind="matvec", n=2999, k=2050, b=3, group=96, dtype="f32", scales="f32"),
        # The largest: a wide projection for a batch of eight.
        dict(name="matvec_28672x8192_b8_bf16", kind="matvec", n=28672, k=8192, b=8, group=128, dtype="bf16", scales="f32"),
        # One chat at its beginning, every query head with keys of its own.
        dict(name="attend_b1_1000_bf16", kind="attend", b=1, hkv=8, g=1, d=128, length=1000, least=1000, window=0,
             page=16, levels=0, order="nhd", dtype="bf16"),
        # A served batch of unequal lengths, one of them empty, eight query heads to a key head.
        dict(name="attend_b32_8192_bf16", kind="attend", b=32, hkv=8, g=8, d=128, length=8192, least=0, window=0,
             page=16, levels=0, order="nhd", dtype="bf16"),
        # Long documents over rows coded with the eight-level codebooks of the solver's cache-row workload.
        dict(name="attend_b16_32768_coded8_f16", kind="attend", b=16, hkv=8, g=4, d=128, length=32768, least=32768,
             window=0, page=64, levels=8, order="hnd", dtype="f16"),
        # One long sequence alone over sixteen-level rows, wide heads, odd page: all of the card for one token.
        dict(name="attend_b1_70001_coded16_bf16", kind="attend", b=1, hkv=4, g=5, d=256, length=70001, least=70001,
             window=0, page=24, levels=16, order="nhd", dtype="bf16"),
        # Single precision, narrow heads, odd pages, a sliding window that hides the beginning.
        dict(name="attend_b3_5001_f32", kind="attend", b=3, hkv=4, g=3, d=64, length=5001, least=700, window=1500,
             page=7, levels=0, order="hnd", dtype="f32"),
        # The new rows of one decoding step of 32 sequences.
        dict(name="write_32x8x128_f32", kind="write", n=32, hkv=8, d=128, page=16, levels=8, order="nhd", dtype="f16",
             x="f32"),
        # The rows of a prompt.
        dict(name="write_8191x8x128_bf16", kind="write", n=8191, hkv=8, d=128, page=64, levels=16, order="hnd",
             dtype="bf16", x="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("matvec", "attend", "attend", "write"))
    dtype = rng.choice(("f16", "bf16"))
    if kind == "matvec":
        dtype = rng.choice(("f16", "bf16", "bf16", "f32"))
        n, k = _log_int(rng, 256, 28672), _log_int(rng, 256, 16384)
        if rng.random() < 0.5:  # half of the matrices have whole 64-column blocks, the others any size
            n, k = 64 * max(4, n // 64) + 8, 64 * max(4, k // 64)
        n, k = n + (n == 3072), k + 64 * (k == 3072)
        return dict(kind=kind, n=n, k=k, b=rng.randint(1, 8), group=rng.choice((32, 64, 96, 128, 256)), dtype=dtype,
                    scales=rng.choice((dtype, "f32")))
    levels = rng.choice((0, 8, 16))
    hkv, page, order = rng.choice((1, 2, 3, 4, 8)), rng.choice((1, 5, 16, 24, 32, 64, 128)), rng.choice(("nhd", "hnd"))
    if kind == "write":
        return dict(kind=kind, n=_log_int(rng, 1, 8191), hkv=hkv, d=rng.choice((64, 96, 128, 256)), page=page,
                    levels=levels or 8, order=order, dtype=dtype, x=rng.choice(("f32", dtype)))
    if not levels:
        dtype = rng.choice(("f16", "bf16", "f32"))
    d = rng.choice((64, 96, 128, 256)) if levels else rng.choice((40, 64, 72, 80, 96, 128, 192, 256))
    b, g = _log_int(rng, 1, 32), rng.choice((1, 2, 3, 4, 6, 8, 12))
    most = min(70001, (1 << 28) // (b * hkv * d))  # values of the keys
    length = _log_int(rng, 1, most)
    length += length == 3072
    return dict(kind=kind, b=b, hkv=hkv, g=g, d=d, length=length, least=rng.choice((0, length)),
                window=rng.choice((0, 0, 0, max(1, length // 3))), page=page, levels=levels, order=order, dtype=dtype)


def _lengths(case):
    """Each sequence's length: the first has the longest, the others spread between `least` and that."""
    lo, hi = case["least"], case["length"]
    return [hi] + [lo + int((hi - lo) * ((i * 0.6180339887) % 1.0)) if i > 1 else lo for i in range(1, case["b"])]


def _ranges(case):
    """(first key, end) of each sequence."""
    return [(max(0, n - case["window"]) if case["window"] else 0, n) for n in _lengths(case)]


def work(case):
    if case["kind"] == "matvec":
        n, k, b, e = case["n"], case["k"], case["b"], SIZES[case["dtype"]]
        weights = n * ((k + 1) // 2) + n * (-(-k // case["group"])) * SIZES[case["scales"]] + 16 * e
        return {"bytes": weights + (b * k + b * n) * e, "flops": 2 * b * n * k}
    if case["kind"] == "write":
        rows, d, levels = case["n"] * case["hkv"], case["d"], case["levels"]
        return {"bytes": rows * (d * SIZES[case["x"]] + 4 * levels + 4 + d // 2 + 2 * levels) + 8 * case["n"],
                "flops": rows * d * 3}
    keys = sum(e - s for s, e in _ranges(case))
    d, hq = case["d"], case["hkv"] * case["g"]
    row = d // 2 + 2 * case["levels"] if case["levels"] else d * SIZES[case["dtype"]]
    return {"bytes": 2 * keys * case["hkv"] * row + case["b"] * hq * (2 * d * SIZES[case["dtype"]] + 4),
            "flops": 4 * keys * hq * d}


# ------------------------------------------------------------------ inputs

def _rows(gen, rows, d):
    """Cache-like rows: a spread of its own for each, one entry in a hundred an outlier of eight spreads."""
    spread = 0.1 + 3.9 * torch.rand(rows, 1, generator=gen, device="cuda")
    x = torch.randn(rows, d, generator=gen, device="cuda")
    big = torch.rand(rows, d, generator=gen, device="cuda") < 0.01
    return torch.where(big, torch.sign(x) * 8.0, x) * spread


def _pages(shape, order):
    """A tensor seen as [pages, slots, heads, row] whose memory has the heads inside the slots or the slots inside the heads."""
    pages, slots, heads, row = shape
    if order == "nhd":
        return lambda make: make((pages, slots, heads, row))
    return lambda make: make((pages, heads, slots, row)).transpose(1, 2)


def _coded_cache(gen, pages, page, hkv, d, levels, order, dtype):
    """Coded rows: per row equally spaced levels over its range, each entry its nearest level's code."""
    heads_first = (pages, page, hkv) if order == "nhd" else (pages, hkv, page)
    rows = pages * page * hkv
    x = _rows(gen, rows, d)
    lo, hi = torch.aminmax(x, dim=1, keepdim=True)
    step = (hi - lo) / (levels - 1)
    code = ((x - lo) / step).add_(0.5).to(torch.uint8).clamp_(max=levels - 1)
    codes = (code[:, 0::2] | (code[:, 1::2] << 4)).view(*heads_first, d // 2)
    table = (lo + step * torch.arange(levels, device="cuda")).to(DTYPES[dtype]).view(*heads_first, levels)
    return (codes, table) if order == "nhd" else (codes.transpose(1, 2), table.transpose(1, 2))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    if case["kind"] == "matvec":
        n, k, b, group = case["n"], case["k"], case["b"], case["group"]
        # Normalised weights are spread normally over +-1: the codes of a codebook fitted to them crowd in the middle.
        wide = -(-k // 128) * 128
        idx = (torch.randn(n, wide, generator=gen, device="cuda") * 2.6 + 8.0).clamp_(0, 15).to(torch.uint8)
        idx[:, k:] = 0
        # Blocks of 128 columns, sixteen words of eight codes each, the words of a block stored as a transposed 4 x 4 square.
        codes = (idx[:, 0::2] | (idx[:, 1::2] << 4)).view(n, wide // 128, 4, 4, 4).transpose(2, 3).reshape(n, wide // 2)
        levels = torch.linspace(-1, 1, 16, device="cuda") ** 3 * 0.6 + torch.linspace(-0.4, 0.4, 16, device="cuda")
        scales = (torch.rand(n, -(-k // group), generator=gen, device="cuda") + 0.5) / math.sqrt(k)
        x = torch.randn(b, k, generator=gen, device="cuda")
        return dict(case=case, x=x.to(dt), codes=codes, levels=levels.to(dt), scales=scales.to(DTYPES[case["scales"]]))
    page, hkv, d, order, levels = case["page"], case["hkv"], case["d"], case["order"], case["levels"]
    if case["kind"] == "write":
        n = case["n"]
        pages = -(-n // page) + 3
        x = _rows(gen, n * hkv, d).to(DTYPES[case["x"]])
        lo, hi = torch.aminmax(x.float(), dim=1, keepdim=True)
        m = levels - torch.randint(0, 3, (n * hkv, 1), generator=gen, device="cuda")  # "at most s" values are found
        at = torch.arange(levels, device="cuda")
        book = torch.where(at == m - 1, hi, torch.where(at < m, lo + (hi - lo) * at / (m - 1), 0.0))
        slots = torch.randperm(pages * page, generator=gen, device="cuda")[:n]
        view = _pages((pages, page, hkv, d // 2), order)
        codes = view(lambda s: torch.zeros(s, dtype=torch.uint8, device="cuda"))
        view = _pages((pages, page, hkv, levels), order)
        table = view(lambda s: torch.zeros(s, dtype=dt, device="cuda"))
        return dict(case=case, x=x.view(n, hkv, d), book=book, m=m.view(-1).to(torch.int32), slots=slots, codes=codes,
                    table=table, seed=int(seed) * 7919 + 1)
    b, g = case["b"], case["g"]
    per = -(-case["length"] // page)
    pages = b * per + 2
    if levels:
        k, kt = _coded_cache(gen, pages, page, hkv, d, levels, order, case["dtype"])
        v, vt = _coded_cache(gen, pages, page, hkv, d, levels, order, case["dtype"])
    else:
        kt = vt = None
        view = _pages((pages, page, hkv, d), order)
        k = view(lambda s: torch.randn(s, generator=gen, device="cuda").to(dt))
        v = view(lambda s: torch.randn(s, generator=gen, device="cuda").to(dt))
    # The queries are a part of one fused projection's output.
    qkv = torch.randn(b, (g + 2) * hkv, d, generator=gen, device="cuda").to(dt)
    span = _ranges(case)
    tensor = lambda at: torch.tensor([s[at] for s in span], dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.randperm(pages, generator=gen, device="cuda")[:b * per].view(b, per).to(torch.int32)
    return dict(case=case, q=qkv[:, :g * hkv], k=k, v=v, kt=kt, vt=vt, table=table, lengths=tensor(1),
                starts=tensor(0) if case["window"] else None, scale=1.0 / math.sqrt(d) / (2.0 if levels else 1.0))


# --------------------------------------------------------------- plain forms

def _unpack(codes, k):
    return torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2)[..., :k].long()


def _plain_matvec(s):
    case = s["case"]
    k, group = case["k"], case["group"]
    codes = s["codes"].view(case["n"], -1, 4, 4, 4).transpose(2, 3).flatten(1)
    w = s["levels"].float()[_unpack(codes, k)]
    w = w * s["scales"].float().repeat_interleave(group, dim=1)[:, :k]
    return (s["x"].float() @ w.T).to(s["x"].dtype)


def _gathered(rows, levels, table):
    """[b, keys, heads, d] in 32 bits: the rows of each sequence's pages in order."""
    picked = rows[table.long()].flatten(1, 2)
    if levels is None:
        return picked.float()
    return levels[table.long()].flatten(1, 2).float().gather(-1, _unpack(picked, 2 * picked.shape[-1]))


def _plain_attend(s):
    case = s["case"]
    b, hkv, g, d = case["b"], case["hkv"], case["g"], case["d"]
    k = _gathered(s["k"], s["kt"], s["table"]).transpose(1, 2)  # [b, hkv, keys, d]
    at = torch.arange(k.shape[2], device="cuda")
    seen = at < s["lengths"][:, None]
    if s["starts"] is not None:
        seen = seen & (at >= s["starts"][:, None])
    seen = seen[:, None, None, :]
    q = s["q"].float().reshape(b, hkv, g, d)
    score = torch.where(seen, q @ k.transpose(2, 3) * s["scale"], -math.inf)
    del k
    top = score.amax(dim=-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(score - top)
    total = p.sum(dim=-1, keepdim=True)
    v = torch.where(seen.transpose(2, 3), _gathered(s["v"], s["vt"], s["table"]).transpose(1, 2), 0.0)
    out = (p @ v) / torch.where(total == 0, 1.0, total)
    lse = (torch.log(total) + top).view(b, hkv * g)
    return out.reshape(b, hkv * g, d).to(s["q"].dtype), lse


def _plain_write(s):
    case = s["case"]
    n, hkv, d, levels = case["n"], case["hkv"], case["d"], case["levels"]
    dt = DTYPES[case["dtype"]]
    x = s["x"].reshape(n * hkv, d).float()
    m = s["m"].long()[:, None]
    at = torch.arange(levels, device="cuda")
    book = s["book"].to(dt)
    book = torch.where(at < m, book, book.gather(1, m - 1))
    r = book.float()
    t = ((r[:, None, :] <= x[:, :, None]) & (at < m)[:, None, :]).sum(-1) - 1  # 16 comparisons an entry
    t = t.clamp_(min=0)
    signed = lambda z: z - (1 << 64) if z >= 1 << 63 else z  # noqa: E731
    z = (torch.arange(1, n * hkv * d + 1, device="cuda") * signed(GAMMA) + s["seed"]).view(n * hkv, d)
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * signed(MUL1)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * signed(MUL2)
    draw24 = ((z >> 40) & 0xFFFFFF).float() * 2.0 ** -24
    low = r.gather(1, t)
    high = r.gather(1, (t + 1).clamp_(max=levels - 1))
    up = (t < m - 1) & (low != x) & (draw24 * (high - low) < x - low)
    code = (t + up).to(torch.uint8).view(n, hkv, d)
    page, slot = s["slots"] // case["page"], s["slots"] % case["page"]
    s["codes"][page, slot] = code[..., 0::2] | (code[..., 1::2] << 4)
    s["table"][page, slot] = book.view(n, hkv, levels)
    return s["codes"], s["table"]


def run(state):
    kind = state["case"]["kind"]
    if not own:
        return {"matvec": _plain_matvec, "attend": _plain_attend, "write": _plain_write}[kind](state)
    import paper_2608_18147_gb300 as E

    if kind == "matvec":
        return E.ecasq_matvec(state["x"], state["codes"], state["levels"], state["scales"], state["case"]["group"])
    if kind == "write":
        return E.ecasq_cache_write(state["x"], state["book"], state["m"], state["slots"], state["codes"],
                                   state["table"], seed=state["seed"])
    if "ws" not in state:
        case = state["case"]
        state["ws"] = E.workspace_attend(case["b"], case["hkv"] * case["g"], case["hkv"], case["d"], case["length"])
    return E.ecasq_attend(state["q"], state["k"], state["v"], state["table"], state["lengths"], scale=state["scale"],
                          starts=state["starts"], k_levels=state["kt"], v_levels=state["vt"],
                          max_len=state["case"]["length"], ws=state["ws"])


# ------------------------------------------------------- definitions in 64 bits

def _exact_matvec(s, case):
    """Column by column of the batch, the scales folded into the activations of each group."""
    n, k, b, group = case["n"], case["k"], case["b"], case["group"]
    y = torch.zeros(b, n, dtype=torch.float64, device="cuda")
    col = torch.arange(k, device="cuda")
    word = col % 128 // 8
    byte = col // 128 * 64 + (word % 4 * 4 + word // 4) * 4 + col % 8 // 2
    for at in range(0, n, 4096):
        c = s["codes"][at:at + 4096][:, byte].int() // torch.where(col % 2 == 1, 16, 1).int() % 16
        w = s["levels"].double()[c]
        for i in range(-(-k // group)):
            part = slice(i * group, min(k, (i + 1) * group))
            y[:, at:at + 4096] += s["x"][:, part].double() @ w[:, part].T * s["scales"][at:at + 4096, i].double()
    return y


def _exact_attend(s, case):
    """One sequence and key head at a time, its keys looked up slot by slot."""
    hkv, g, d = case["hkv"], case["g"], case["d"]
    out = torch.zeros(case["b"], hkv * g, d, dtype=torch.float64, device="cuda")
    lse = torch.full((case["b"], hkv * g), -math.inf, dtype=torch.float64, device="cuda")

    def values(rows, levels, page, slot, h):
        r = rows[page, slot, h]
        if levels is None:
            return r.double()
        t = levels[page, slot, h].double()
        x = torch.empty(r.shape[0], d, dtype=torch.float64, device="cuda")
        x[:, 0::2] = torch.gather(t, 1, (r % 16).long())
        x[:, 1::2] = torch.gather(t, 1, (r // 16).long())
        return x

    for i, (first, end) in enumerate(_ranges(case)):
        if end <= first:
            continue
        t = torch.arange(first, end, device="cuda")
        page, slot = s["table"][i][t // case["page"]].long(), t % case["page"]
        for h in range(hkv):
            q = s["q"][i, h * g:(h + 1) * g].double()
            w = (values(s["k"], s["kt"], page, slot, h) @ q.T * s["scale"]).T
            lse[i, h * g:(h + 1) * g] = torch.logsumexp(w, dim=1)
            out[i, h * g:(h + 1) * g] = torch.softmax(w, dim=1) @ values(s["v"], s["vt"], page, slot, h)
    return out, lse


def _exact_write(s, case):
    """The levels before they are rounded; the codes are whole numbers that the rounding rule fixes."""
    m = s["m"].long()[:, None]
    at = torch.minimum(torch.arange(case["levels"], device="cuda")[None], m - 1)
    book = torch.gather(s["book"].double(), 1, at).view(case["n"], case["hkv"], case["levels"])
    table = torch.zeros(s["table"].shape, dtype=torch.float64, device="cuda")
    table[s["slots"] // case["page"], s["slots"] % case["page"]] = book
    return None, table


def exact(case, seed):
    s = prepare(case, seed)
    return {"matvec": _exact_matvec, "attend": _exact_attend, "write": _exact_write}[case["kind"]](s, case)
