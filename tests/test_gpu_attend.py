"""Attention of one new token over a paged cache (ecasq_attend) against a plain implementation in 64 bits.

Tolerances.  A score is an fp32 sum of d products and a few scalings: within e = (d / 8 + 16) 2^-23 scale sum |q k| of the
exact one, plus 2^-21 |s| for the change to base 2.  Scores that are all off by at most e move the weighted mean of
the values by at most 2 e sum p |v| (to first order; e is below 1e-2 here, and twice that is allowed) and the
logarithm of the sum by at most e.  Weights are kept to 16 bits or more and sums over n keys in fp32: (2^-15 + (n + 64) 2^-23) sum p |v|.
The result is rounded once, by u |out|.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
KINDS = [("f32", 0), ("f16", 0), ("bf16", 0), ("f16", 8), ("bf16", 8), ("f16", 16), ("bf16", 16)]


def dt(name):
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


class Side:
    """One side of a cache: the tensors of the call and the values that they stand for, in binary64."""

    def __init__(self, gen, pages, page, hkv, d, dtype, levels, order):
        shape = (pages, page, hkv) if order == "nhd" else (pages, hkv, page)
        turn = (lambda t: t) if order == "nhd" else (lambda t: t.transpose(1, 2))
        if not levels:
            self.rows = turn(torch.randn(*shape, d, generator=gen, device="cuda").to(dt(dtype)))
            self.levels = None
            return
        code = torch.randint(0, levels, (*shape, d), generator=gen, device="cuda", dtype=torch.uint8)
        self.rows = turn(code[..., 0::2] | (code[..., 1::2] << 4))
        self.levels = turn(torch.sort(torch.randn(*shape, levels, generator=gen, device="cuda")).values.to(dt(dtype)))

    def values(self, page, slot, h):
        r = self.rows[page, slot, h]
        if self.levels is None:
            return r.double().cpu().numpy()
        r = r.cpu().numpy()
        t = self.levels[page, slot, h].double().cpu().numpy()
        code = np.stack((r & 15, r >> 4), axis=-1).reshape(r.shape[0], -1).astype(np.int64)
        return np.take_along_axis(t, code, axis=1)


def make(lengths, hkv, g, d, page, dtype, levels, order="nhd", seed=0, starts=None, spare=3, max_len=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    b = len(lengths)
    per = max(1, -(-max(max(lengths), max_len or 0) // page))
    pages = b * per + spare
    k = Side(gen, pages, page, hkv, d, dtype, levels, order)
    v = Side(gen, pages, page, hkv, d, dtype, levels, order)
    q = torch.randn(b, hkv * g, d, generator=gen, device="cuda").to(dt(dtype))
    table = torch.randperm(pages, generator=gen, device="cuda")[:b * per].view(b, per).to(torch.int32)
    return dict(q=q, k=k, v=v, table=table, lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"),
                starts=None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda"), page=page,
                hkv=hkv, g=g, d=d, dtype=dtype)


def call(c, **kw):
    import paper_2608_18147_gb300 as E
    args = dict(k_levels=c["k"].levels, v_levels=c["v"].levels, starts=c["starts"])
    args.update(kw)
    return E.ecasq_attend(c["q"], c["k"].rows, c["v"].rows, c["table"], c["lengths"], **args)


def reference(c, scale=None, leave=None):
    """out, its tolerance, lse, its tolerance.  leave: (sequence, key) pairs to leave out."""
    b, hq, d = c["q"].shape
    scale = d ** -0.5 if scale is None else scale
    out, tol = np.zeros((b, hq, d)), np.zeros((b, hq, d))
    lse, ltol = np.full((b, hq), -np.inf), np.zeros((b, hq))
    table = c["table"].long()
    for i in range(b):
        first = 0 if c["starts"] is None else max(0, int(c["starts"][i]))
        t = torch.arange(first, max(first, int(c["lengths"][i])), device="cuda")
        if leave:
            t = torch.tensor([x for x in t.tolist() if (i, x) not in leave], device="cuda", dtype=torch.long)
        if t.numel() == 0:
            continue
        page, slot = table[i][t // c["page"]], t % c["page"]
        for h in range(hq):
            kv = c["k"].values(page, slot, h // c["g"])
            vv = c["v"].values(page, slot, h // c["g"])
            q = c["q"][i, h].double().cpu().numpy()
            s = kv @ q * scale
            e = (np.abs(kv) @ np.abs(q) * abs(scale) * (d / 8 + 16) * 2.0 ** -23 + np.abs(s) * 2.0 ** -21).max()
            top = s.max()
            p = np.exp(s - top)
            lse[i, h] = top + math.log(p.sum())
            p /= p.sum()
            out[i, h] = p @ vv
            n = t.numel()
            tol[i, h] = U[c["dtype"]] * np.abs(out[i, h]) + (4 * e + 2.0 ** -15 + (n + 64) * 2.0 ** -23) * (p @ np.abs(vv)) + 2.0 ** -25
            ltol[i, h] = e + (n + 64) * 2.0 ** -23 + np.abs(lse[i, h]) * 2.0 ** -22
    return out, tol, lse, ltol


def check(got, want):
    out, lse = (t.double().cpu().numpy() for t in got)
    ro, to, rl, tl = want
    assert np.isfinite(out).all()
    bad = ~(np.abs(out - ro) <= to)
    assert not bad.any(), (np.argwhere(bad)[:4], out[bad][:4], ro[bad][:4], to[bad][:4])
    empty = np.isneginf(rl)
    assert (np.isneginf(lse) == empty).all()
    assert (out[empty] == 0).all()
    assert (np.abs(lse[~empty] - rl[~empty]) <= tl[~empty]).all(), (lse, rl)


@pytest.mark.parametrize("dtype,levels", KINDS)
@pytest.mark.parametrize("lengths,page,order", [
    ([0, 1, 2, 15, 16, 17], 16, "nhd"), ([31, 32, 33, 64, 100, 0], 5, "hnd"), ([300, 7, 129], 1, "nhd"),
    ([1000, 0, 640], 24, "hnd"), ([257], 64, "nhd"), ([0], 16, "nhd"), ([1], 128, "hnd"), ([5000, 4999], 32, "nhd"),
])
def test_lengths_and_pages(lengths, page, order, dtype, levels):
    c = make(lengths, 2, 2, 64, page, dtype, levels, order, seed=len(lengths) + page)
    check(call(c), reference(c))


@pytest.mark.parametrize("dtype,levels", KINDS)
@pytest.mark.parametrize("hkv,g,d", [(1, 1, 32), (2, 3, 96), (3, 8, 128), (1, 12, 128), (2, 5, 256), (1, 16, 64), (4, 1, 192),
                                     (1, 2, 160), (1, 9, 224)])
def test_heads(hkv, g, d, dtype, levels):
    c = make([77, 400], hkv, g, d, 16, dtype, levels, "nhd", seed=d + g)
    check(call(c), reference(c))


@pytest.mark.parametrize("dtype,d", [("f32", 4), ("f32", 36), ("f32", 100), ("f16", 8), ("bf16", 40), ("bf16", 72), ("f16", 80),
                                     ("bf16", 248), ("f32", 252)])
def test_odd_row_lengths(dtype, d):
    c = make([50, 333], 2, 2, d, 7, dtype, 0, "hnd", seed=d)
    check(call(c), reference(c))


@pytest.mark.parametrize("dtype,levels", KINDS)
def test_starts_and_what_lies_outside(dtype, levels):
    """Only [start, length) is seen: NaN everywhere else, in the same pages and in others, changes nothing."""
    lengths, starts = [100, 90, 37, 64, 33, 5], [0, 37, 36, 64, 40, -4]
    c = make(lengths, 2, 4, 64, 16, dtype, levels, "nhd", seed=4, starts=starts, max_len=160)
    want = reference(c)
    before = call(c)
    for side in (c["k"], c["v"]):
        values = side.rows if levels == 0 else side.levels
        seen = torch.zeros(values.shape[:2], dtype=torch.bool, device="cuda")
        for i, (s, n) in enumerate(zip(starts, lengths)):
            t = torch.arange(max(0, s), max(n, max(0, s)), device="cuda")
            seen[c["table"][i].long()[t // 16], t % 16] = True
        values[~seen] = float("nan")
    after = call(c)
    check(after, want)
    assert torch.equal(before[0], after[0]) and torch.equal(before[1], after[1])
    assert (call(c)[0][[3, 4]] == 0).all()


@pytest.mark.parametrize("dtype,levels", KINDS)
@pytest.mark.parametrize("b,n,page", [(1, 20011, 16), (2, 9001, 24), (40, 130, 16)])
def test_split_over_the_length(b, n, page, dtype, levels):
    """Long sequences alone, and many short ones."""
    c = make([max(0, n - 37 * i) for i in range(b)], 1, 4, 64, page, dtype, levels, "hnd", seed=n)
    check(call(c), reference(c))


@pytest.mark.parametrize("dtype,levels", KINDS)
def test_sharp_flat_and_negative_scales(dtype, levels):
    c = make([200, 31], 2, 3, 64, 16, dtype, levels, seed=11)
    check(call(c, scale=0.0), reference(c, scale=0.0))
    check(call(c, scale=-0.3), reference(c, scale=-0.3))
    # One key far ahead of the others: weights that underflow, and nothing else.
    c["q"] *= 20
    check(call(c, scale=2.0), reference(c, scale=2.0))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_keys_of_minus_infinity(dtype):
    """Keys whose scores are -inf have no weight; where all are, the sequence counts as empty."""
    c = make([40, 40], 1, 2, 64, 16, dtype, 0, seed=12)
    c["q"].abs_()
    c["q"].add_(0.1)
    t = torch.arange(40, device="cuda")
    page = c["table"].long()
    c["k"].rows[page[0][t // 16], t % 16] = -float("inf")
    few = torch.tensor([0, 15, 16, 39], device="cuda")
    c["k"].rows[page[1][few // 16], few % 16] = -float("inf")
    leave = {(0, x) for x in range(40)} | {(1, x) for x in few.tolist()}
    check(call(c), reference(c, leave=leave))


@pytest.mark.parametrize("dtype,levels", KINDS)
def test_bad_pages_and_lengths_are_reported(dtype, levels):
    import paper_2608_18147_gb300 as E
    c = make([64, 50, 200], 2, 2, 64, 16, dtype, levels, seed=13)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    call(c, status=status)
    assert status.item() == 0
    pages = c["k"].rows.shape[0]
    c["table"][0, 1], c["table"][1, 0] = pages, -1
    leave = {(0, x) for x in range(16, 32)} | {(1, x) for x in range(16)}
    good = c["table"].clone()
    good[0, 1] = good[1, 0] = 0
    got = call(c, status=status)
    assert status.item() == E.BAD_PAGE
    check(got, reference(dict(c, table=good), leave=leave))
    status.zero_()
    c["lengths"][2] = 1000  # longer than the table
    got = call(dict(c, table=good), status=status)
    assert status.item() == E.BAD_LENGTH
    c["lengths"][2] = good.shape[1] * 16
    check(got, reference(dict(c, table=good)))
    c["lengths"][1] = -5
    got = call(dict(c, table=good))
    check(got, reference(dict(c, table=good)))


@pytest.mark.parametrize("dtype,levels", KINDS)
def test_strided_queries_and_out(dtype, levels):
    c = make([60, 17], 2, 2, 64, 16, dtype, levels, seed=14)
    qkv = torch.randn(2, 8 * 64 + 6, device="cuda").to(dt(dtype))
    q = qkv[:, 6:].view(2, 8, 64)[:, 1:8:2]
    q.copy_(c["q"])
    room = torch.full((2, 4, 65), 7.0, dtype=dt(dtype), device="cuda")
    want = reference(c)
    got = call(dict(c, q=q), out=room[:, :, 1:])
    check(got, want)
    assert (room[:, :, 0] == 7).all()


@pytest.mark.parametrize("dtype,levels", KINDS)
def test_equal_bits_whatever_else_is_in_the_batch(dtype, levels):
    """Equal calls, a replayed graph, another stream and other sequences' lengths: the same bits."""
    c = make([3000, 40, 1500], 2, 4, 128, 16, dtype, levels, seed=15)
    first = call(c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = call(c)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(first, second))
    import paper_2608_18147_gb300 as E
    ws = E.workspace_attend(3, 8, 2, 128, c["table"].shape[1] * 16)
    out = torch.empty_like(first[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = call(c, ws=ws, out=out)
    for _ in range(2):
        out.zero_()
        ws.fill_(255)  # the workspace needs no preparation
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(first, third))
    c["lengths"][0] = 0
    other = call(c)
    assert all(torch.equal(x[1:], y[1:]) for x, y in zip(first, other))


@pytest.mark.parametrize("dtype,levels", KINDS)
@pytest.mark.parametrize("page", [16, 32, 9])
def test_keys_and_values_laid_out_differently(page, dtype, levels):
    """Keys with the heads inside the slots, values the other way round, in a wider cache."""
    c = make([70, 333], 3, 2, 64, page, dtype, levels, "nhd", seed=19)
    v = c["v"]

    def turned(t):
        wide = torch.full((t.shape[0] + 1, t.shape[2] + 2, t.shape[1], t.shape[3]), 1, dtype=t.dtype, device="cuda")
        part = wide[1:, 1:-1].transpose(1, 2)
        part.copy_(t)
        return part

    v.rows = turned(v.rows)
    if levels:
        v.levels = turned(v.levels)
    check(call(c), reference(c))


@pytest.mark.parametrize("dtype,levels", KINDS)
def test_many_sequences(dtype, levels):
    """Hundreds of short sequences: a join a warp a head, and sequences of one split beside longer ones."""
    lengths = [(37 * i) % 300 for i in range(400)]
    c = make(lengths, 2, 2, 32, 16, dtype, levels, "hnd", seed=20)
    few = [0, 1, 7, 100, 250, 399]
    got = call(c)
    part = dict(c, q=c["q"][few], table=c["table"][few], lengths=c["lengths"][few])
    check((got[0][few], got[1][few]), reference(part))


@pytest.mark.parametrize("dtype,levels", KINDS)
@pytest.mark.parametrize("lengths,max_len,starts", [([500, 0, 1, 130, 64], 512, None), ([256, 255], 256, [255, 0]), ([65, 3, 400], 1000, [0, 2, 399]),
                                                    ([900], 960, [17])])
def test_few_splits(lengths, max_len, starts, dtype, levels):
    """Two to eight splits, of which a short sequence fills one or none; twice for equal bits."""
    c = make(lengths, 2, 3, 96, 16, dtype, levels, "nhd", seed=22, starts=starts, max_len=max_len)
    got = call(c, max_len=max_len)
    check(got, reference(c))
    again = call(c, max_len=max_len)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("dtype,levels", KINDS)
def test_starts_beyond_every_key(dtype, levels):
    """A start past the end leaves no key, however far past it is."""
    c = make([50, 50, 600, 600], 2, 4, 32, 16, dtype, levels, "nhd", seed=21, starts=[2 ** 31 - 1, 49, 2 ** 31 - 40, 3])
    got = call(c)
    check(got, reference(c))
    assert (got[0][[0, 2]] == 0).all() and (got[1][[0, 2]] == -math.inf).all()


@pytest.mark.parametrize("dtype,levels", [("bf16", 0), ("f16", 8)])
def test_offsets_beyond_32_bits(dtype, levels):
    """Pages more than 2^32 entries from the cache's start."""
    hkv, d, page = 8, 128, 64
    row = d // 2 if levels else d
    pages = (1 << 32) // (page * hkv * row) + 40
    kind = torch.uint8 if levels else dt(dtype)
    c = make([150, 70], hkv, 2, d, page, dtype, levels, seed=16)
    for name in ("k", "v"):
        side, few = c[name], c[name].rows.shape[0]
        rows = torch.empty((pages, page, hkv, row), dtype=kind, device="cuda")
        rows[-few:] = side.rows
        side.rows = rows
        if levels:
            table = torch.empty((pages, page, hkv, levels), dtype=dt(dtype), device="cuda")
            table[-few:] = side.levels
            side.levels = table
    c["table"] += pages - few
    check(call(c), reference(c))


def test_refusals():
    import paper_2608_18147_gb300 as E
    c = make([40, 3], 2, 2, 64, 16, "bf16", 0, seed=17)
    good = dict(q=c["q"], k=c["k"].rows, v=c["v"].rows, table=c["table"], lengths=c["lengths"])
    E.ecasq_attend(**good)
    empty = E.ecasq_attend(**dict(good, q=c["q"][:0], table=c["table"][:0], lengths=c["lengths"][:0]))
    assert empty[0].shape == (0, 4, 64) and empty[1].shape == (0, 4)
    k = c["k"].rows
    bad = [dict(q=c["q"].float()), dict(q=c["q"][:, :3]), dict(q=c["q"][:, :, :32]), dict(q=c["q"].cpu()), dict(k=k.half()),
           dict(k=k[:, :8]), dict(k=k[:-1]), dict(k=k[:, :, :1]), dict(table=c["table"].long()), dict(table=c["table"][:1]),
           dict(lengths=c["lengths"].long()), dict(lengths=c["lengths"][:1]), dict(starts=c["lengths"].long()),
           dict(max_len=10 ** 6), dict(max_len=-1), dict(k_levels=k), dict(out=c["q"].float()), dict(status=c["lengths"].long()),
           dict(k=k[..., 4:36], v=k[..., 4:36], q=c["q"][..., :32])]
    for change in bad:
        with pytest.raises(E.EcasqError):
            E.ecasq_attend(**dict(good, **change))
    coded = make([40, 3], 2, 2, 64, 16, "bf16", 8, seed=17)
    levels = coded["k"].levels
    good = dict(q=coded["q"], k=coded["k"].rows, v=coded["v"].rows, table=coded["table"], lengths=coded["lengths"],
                k_levels=levels, v_levels=coded["v"].levels)
    E.ecasq_attend(**good)
    bad = [dict(k_levels=None), dict(k_levels=levels.half()), dict(k_levels=levels.float()), dict(k_levels=levels[..., :4]),
           dict(k_levels=levels[:-1]), dict(q=coded["q"].half()),
           dict(k=coded["k"].rows[..., :24], v=coded["v"].rows[..., :24], q=coded["q"][..., :48])]
    for change in bad:
        with pytest.raises(E.EcasqError):
            E.ecasq_attend(**dict(good, **change))
    wide = make([700, 3], 2, 2, 64, 16, "bf16", 0, seed=18)
    need = E.workspace_attend(2, 4, 2, 64, 700).numel()
    if need:
        with pytest.raises(E.EcasqError):
            call(wide, ws=torch.empty(need - 1, dtype=torch.uint8, device="cuda"), max_len=700)
