"""Encode of cache rows (ecasq_cache_write): codes and levels equal the rounding rule's, bit for bit."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

MASK = (1 << 64) - 1


def dt(name):
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def draws(seed, count):
    """Top 24 bits of SplitMix64(seed + (c + 1) gamma), c < count."""
    z = (np.uint64(seed & MASK) + np.arange(1, count + 1, dtype=np.uint64) * np.uint64(0x9E3779B97F4A7C15))
    z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
    z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    z = z ^ (z >> np.uint64(31))
    return (z >> np.uint64(40)).astype(np.float32) * np.float32(2.0 ** -24)


def reference(x, Q, m, levels, dtype, seed):
    """(codes [rows, d], levels [rows, levels] of the cache's type) by the rule, entry by entry."""
    rows, d = x.shape
    u = draws(seed, rows * d).reshape(rows, d)
    codes = np.zeros((rows, d), np.uint8)
    book = torch.zeros(rows, levels, dtype=dt(dtype))
    for r in range(rows):
        n = int(m[r])
        q = Q[r, :n].to(dt(dtype))
        book[r, :n] = q
        book[r, n:] = q[-1]
        q = q.float().numpy()
        for e in range(d):
            v = x[r, e]
            below = np.flatnonzero(q <= v)
            t = int(below[-1]) if below.size else 0
            if t < n - 1 and q[t] != v and u[r, e] * (q[t + 1] - q[t]) < v - q[t]:
                t += 1
            codes[r, e] = t
    return codes, book


def make(n, heads, d, levels, dtype, x_dtype, seed=0, s=None, short=True):
    g = torch.Generator().manual_seed(seed)
    s = levels if s is None else s
    x = (torch.randn(n, heads, d, generator=g) * (0.1 + torch.rand(n, heads, 1, generator=g))).to(dt(x_dtype))
    rows = n * heads
    m = torch.randint(1 if short else s, s + 1, (rows,), generator=g, dtype=torch.int32)
    xr = torch.sort(x.float().view(rows, d), dim=1).values
    Q = torch.zeros(rows, s)
    for r in range(rows):  # values of the row itself, its ends among them where there are two or more
        at = torch.linspace(0, d - 1, int(m[r])).long() if m[r] > 1 else torch.tensor([d // 2])
        Q[r, :int(m[r])] = xr[r, at]
    return x, Q, m


def cache(pages, page, heads, d, levels, dtype, order="nhd"):
    shape = (pages, page, heads) if order == "nhd" else (pages, heads, page)
    codes = torch.full((*shape, d // 2), 0xA5, dtype=torch.uint8, device="cuda")
    table = torch.full((*shape, levels), 77.0, dtype=dt(dtype), device="cuda")
    return (codes, table) if order == "nhd" else (codes.transpose(1, 2), table.transpose(1, 2))


def expect(codes, table, want, book, slots, page, heads):
    """The cache before the call with the written rows in their slots."""
    codes, table = codes.cpu().clone(), table.cpu().clone()
    for i, slot in enumerate(slots.tolist()):
        if 0 <= slot < codes.shape[0] * page:
            for h in range(heads):
                c = want[i * heads + h]
                codes[slot // page, slot % page, h] = torch.from_numpy(c[0::2] | (c[1::2] << 4))
                table[slot // page, slot % page, h] = book[i * heads + h]
    return codes, table


@pytest.mark.parametrize("levels,dtype,x_dtype", [(8, "f16", "f32"), (8, "bf16", "bf16"), (16, "f16", "f16"), (16, "bf16", "f32")])
@pytest.mark.parametrize("n,heads,d,page,order", [(1, 1, 32, 16, "nhd"), (5, 3, 64, 7, "hnd"), (9, 2, 96, 1, "nhd"), (40, 8, 128, 64, "hnd"),
                                                  (3, 5, 256, 24, "nhd"), (2, 1, 224, 16, "nhd")])
def test_codes_are_the_rules(n, heads, d, page, order, levels, dtype, x_dtype):
    import paper_2608_18147_gb300 as E
    x, Q, m = make(n, heads, d, levels, dtype, x_dtype, seed=n + d)
    pages = -(-n // page) + 2
    slots = torch.randperm(pages * page)[:n]
    codes, table = cache(pages, page, heads, d, levels, dtype, order)
    seed = (1 << 63) + 12345 * d + n
    want, book = reference(x.float().view(n * heads, d).numpy(), Q, m, levels, dtype, seed)
    full = expect(codes, table, want, book, slots, page, heads)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = E.ecasq_cache_write(x.cuda(), Q.cuda(), m.cuda(), slots.cuda(), codes, table, seed, status=status)
    assert got[0] is codes and got[1] is table and status.item() == 0
    assert torch.equal(codes.cpu(), full[0])
    assert torch.equal(table.cpu(), full[1])


def test_same_indices_as_the_flat_encode():
    """A codebook that its rounding leaves alone gives ecasq_quantize's indices for the same seed."""
    import paper_2608_18147_gb300 as E
    x = torch.randn(1, 1, 256).to(torch.bfloat16)
    Q, _ = torch.sort(torch.unique(x.float().view(-1))[::40])
    Q = torch.unique(torch.cat([Q, x.float().view(-1).min()[None], x.float().view(-1).max()[None]]))[:16]
    Q[-1] = x.float().max()
    m = Q.numel()
    idx, _, _ = E.ecasq_quantize(x.float().view(-1).cuda(), Q.cuda(), 99)
    codes, table = cache(1, 1, 1, 256, 16, "bf16")
    E.ecasq_cache_write(x.cuda(), Q.view(1, m).cuda(), None, torch.zeros(1, dtype=torch.int64, device="cuda"), codes, table, 99)
    c = codes.view(-1)
    assert torch.equal(torch.stack((c & 15, c >> 4), -1).view(-1), idx)


def test_codebooks_of_the_batched_solve():
    """ecasq_solve_batched's rows go in as they come out: fewer levels than the cache has, m of its own for each row."""
    import paper_2608_18147_gb300 as E
    n, heads, d = 6, 2, 128
    x = torch.randn(n, heads, d)
    Q, m, _ = E.ecasq_solve_batched(x.view(n * heads, d).cuda(), 8, budget_bits=2.0)
    for levels in (8, 16):
        codes, table = cache(2, 4, heads, d, levels, "f16")
        slots = torch.tensor([0, 1, 2, 5, 6, 7])
        want, book = reference(x.view(n * heads, d).numpy(), Q.cpu(), m.cpu(), levels, "f16", 3)
        full = expect(codes, table, want, book, slots, 4, heads)
        E.ecasq_cache_write(x.cuda(), Q, m, slots.cuda(), codes, table, 3)
        assert torch.equal(codes.cpu(), full[0]) and torch.equal(table.cpu(), full[1])


def test_rounding_is_unbiased():
    """The mean over many seeds: 4096 draws of a decision with probability f have a standard error of at most 2^-7."""
    import paper_2608_18147_gb300 as E
    f = torch.linspace(0.01, 0.99, 32)
    x = f.view(1, 1, 32).expand(4096, 1, 32).contiguous()
    Q = torch.tensor([[0.0, 1.0]]).expand(4096, 2).contiguous()
    codes, table = cache(64, 64, 1, 32, 8, "f16")
    E.ecasq_cache_write(x.cuda(), Q.cuda(), None, torch.arange(4096, device="cuda"), codes, table, 5)
    c = codes.view(4096, 16).cpu()
    mean = torch.stack((c & 15, c >> 4), -1).view(4096, 32).float().mean(0)
    assert ((mean - f).abs() <= 5 * 2.0 ** -7).all()


def test_slots_counts_and_values_that_are_wrong():
    import paper_2608_18147_gb300 as E
    n, heads, d, page = 6, 1, 32, 4
    x, Q, m = make(n, heads, d, 8, "f16", "f32", seed=1, short=False)
    slots = torch.tensor([-1, 0, 8, 5, 1 << 40, -(1 << 50)])
    codes, table = cache(2, page, heads, d, 8, "f16")
    want, book = reference(x.view(n, d).numpy(), Q, m, 8, "f16", 1)
    full = expect(codes, table, want, book, slots, page, heads)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    E.ecasq_cache_write(x.cuda(), Q.cuda(), m.cuda(), slots.cuda(), codes, table, 1, status=status)
    assert status.item() == E.BAD_PAGE
    assert torch.equal(codes.cpu(), full[0]) and torch.equal(table.cpu(), full[1])
    # NaN takes code 0, the infinities the ends; counts outside [1, s] are clamped
    x[0, 0, :3] = torch.tensor([float("nan"), float("inf"), -float("inf")])
    m[1], m[2] = 0, 99
    clamped = m.clone()
    clamped[1], clamped[2] = 1, 8
    slots = torch.arange(n)
    want, book = reference(x.view(n, d).numpy(), Q, clamped, 8, "f16", 1)
    assert want[0, 0] == 0 and want[0, 1] == 7 and want[0, 2] == 0
    full = expect(codes, table, want, book, slots, page, heads)
    status.zero_()
    E.ecasq_cache_write(x.cuda(), Q.cuda(), m.cuda(), slots.cuda(), codes, table, 1, status=status)
    assert status.item() == E.BAD_COUNT | E.BAD_VALUE
    assert torch.equal(codes.cpu(), full[0]) and torch.equal(table.cpu(), full[1])


def test_entries_beyond_the_codebook_and_levels_that_coincide():
    """Entries outside the codebook take its ends; levels that round to one value act as the last of them."""
    import paper_2608_18147_gb300 as E
    x = torch.linspace(-3, 3, 64).view(1, 1, 64)
    Q = torch.tensor([[-1.0, -1.0 + 1e-6, 0.5, 0.5 + 1e-7, 1.0]])
    codes, table = cache(1, 1, 1, 64, 8, "bf16")
    want, book = reference(x.view(1, 64).numpy(), Q, [5], 8, "bf16", 8)
    E.ecasq_cache_write(x.cuda(), Q.cuda(), None, torch.zeros(1, dtype=torch.int64, device="cuda"), codes, table, 8)
    c = codes.view(-1).cpu().numpy()
    np.testing.assert_array_equal(np.stack((c & 15, c >> 4), -1).reshape(1, 64), want)
    assert torch.equal(table.view(1, 8).cpu(), book)


def test_strided_rows():
    """x as a part of a fused projection's output."""
    import paper_2608_18147_gb300 as E
    n, heads, d = 7, 2, 64
    x, Q, m = make(n, heads, d, 16, "bf16", "bf16", seed=3)
    wide = torch.zeros(n, 5, d + 1, dtype=x.dtype, device="cuda")
    part = wide[:, 1:5:2, 1:]
    part.copy_(x)
    codes, table = cache(1, 8, heads, d, 16, "bf16")
    slots = torch.arange(n)
    want, book = reference(x.float().view(n * heads, d).numpy(), Q, m, 16, "bf16", 2)
    full = expect(codes, table, want, book, slots, 8, heads)
    E.ecasq_cache_write(part, Q.view(n, heads, 16).cuda(), m.cuda(), slots.cuda(), codes, table, 2)
    assert torch.equal(codes.cpu(), full[0]) and torch.equal(table.cpu(), full[1])


@pytest.mark.parametrize("d", [64, 128])
def test_slots_beyond_32_bits(d):
    """Slot numbers of 2^31 and more (slots that share memory, as only two rows are written)."""
    import paper_2608_18147_gb300 as E
    x, Q, m = make(2, 1, d, 8, "bf16", "f32", seed=6)
    room = torch.zeros(4, d // 2, dtype=torch.uint8, device="cuda")
    books = torch.zeros(4, 8, dtype=torch.bfloat16, device="cuda")
    codes = room.as_strided((4, 1 << 30, 1, d // 2), (d // 2, 0, d // 2, 1))
    table = books.as_strided((4, 1 << 30, 1, 8), (8, 0, 8, 1))
    slots = torch.tensor([(1 << 31) + 77, (3 << 30) + 5, ], device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    want, book = reference(x.view(2, d).numpy(), Q, m, 8, "bf16", 4)
    E.ecasq_cache_write(x.cuda(), Q.cuda(), m.cuda(), slots, codes, table, 4, status=status)
    assert status.item() == 0 and not room[:2].any() and not books[:2].any()
    c = room[2:].cpu().numpy()
    np.testing.assert_array_equal(np.stack((c & 15, c >> 4), axis=-1).reshape(2, d), want)
    assert torch.equal(books[2:].cpu(), book)
    E.ecasq_cache_write(x.cuda(), Q.cuda(), m.cuda(), slots + (1 << 31), codes, table, 5, status=status)
    assert status.item() == E.BAD_PAGE
    assert np.array_equal(room[2:].cpu().numpy(), c)


def test_refusals():
    import paper_2608_18147_gb300 as E
    x, Q, m = make(4, 2, 64, 8, "f16", "f32")
    x, Q, m = x.cuda(), Q.cuda(), m.cuda()
    slots = torch.arange(4, device="cuda")
    codes, table = cache(2, 4, 2, 64, 8, "f16")
    good = [x, Q, m, slots, codes, table]
    E.ecasq_cache_write(*good, seed=0)
    E.ecasq_cache_write(x[:0], Q[:0], m[:0], slots[:0], codes, table, seed=0)
    bad = [(0, x.bfloat16()), (0, x[:3]), (0, x[:, :1]), (0, x.cpu()), (1, Q.half()), (1, Q[:7]), (1, Q.t()),
           (1, torch.zeros(8, 9, device="cuda")), (2, m.long()), (2, m[:7]), (3, slots.int()), (4, codes.int()), (4, codes[..., :24]),
           (5, table.float()), (5, table[..., :4]), (5, table[:1]), (5, None)]
    for at, value in bad:
        args = list(good)
        args[at] = value
        with pytest.raises(E.EcasqError):
            E.ecasq_cache_write(*args, seed=0)
