"""Calls of the operators on 4-bit codes in a row, each reading what the one before wrote, with nothing between them: a call's kernels are
placed while those of the call before still run, and have to wait for their end themselves.  The same calls with a
synchronisation after each give the same bits."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def matrix(n, k, dtype, gen):
    """A coded matrix whose products keep about the size of x."""
    import paper_2608_18147_gb300 as E
    idx = torch.randint(0, 16, (n, k), generator=gen, device="cuda", dtype=torch.uint8)
    levels = torch.linspace(-1, 1, 16, device="cuda").to(dtype)
    scales = (0.5 + torch.rand(n, -(-k // 128), generator=gen, device="cuda")) * 1.6 / k ** 0.5
    return E.ecasq_pack(idx), levels, scales


def both(steps):
    """What `steps` leaves with a synchronisation after each of its calls, and ten times without any."""
    def run(wait):
        out = []
        torch.cuda.synchronize()
        for result in steps():
            if wait:
                torch.cuda.synchronize()
            out.append(result)
        torch.cuda.synchronize()
        return [t.clone() for t in out[-1]]

    want = run(True)
    assert all(torch.isfinite(t.float()).all() and t.float().abs().sum() > 0 for t in want)
    for _ in range(10):
        assert all(torch.equal(x, y) for x, y in zip(run(False), want))


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("sizes,b", [((1024, 1024), 3), ((16384, 1024), 1), ((300, 24576), 2), ((8192, 520), 8), ((9000, 640), 11)])
def test_products_in_a_chain(sizes, b, dtype):
    """x through W1 [n, k], W2 [k, n] and so on, in place of one another."""
    import paper_2608_18147_gb300 as E
    n, k = sizes
    gen = torch.Generator(device="cuda").manual_seed(n)
    there, back = matrix(n, k, dtype, gen), matrix(k, n, dtype, gen)
    first = torch.randn(b, k, generator=gen, device="cuda").to(dtype)
    x, y = torch.empty(b, k, dtype=dtype, device="cuda"), torch.empty(b, n, dtype=dtype, device="cuda")

    def steps():
        x.copy_(first)
        for _ in range(8):
            yield (E.ecasq_matvec(x, *there, 128, out=y),)
            yield (E.ecasq_matvec(y, *back, 128, out=x), y)

    both(steps)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_what_a_call_reads_is_overwritten_by_the_next(dtype):
    import paper_2608_18147_gb300 as E
    gen = torch.Generator(device="cuda").manual_seed(5)
    large, small = matrix(9000, 2048, dtype, gen), matrix(2048, 256, dtype, gen)
    first = torch.randn(4, 2048, generator=gen, device="cuda").to(dtype)
    other = torch.randn(4, 256, generator=gen, device="cuda").to(dtype)
    x, y = torch.empty_like(first), torch.empty(4, 9000, dtype=dtype, device="cuda")

    def steps():
        x.copy_(first)
        yield (E.ecasq_matvec(x, *large, 128, out=y),)  # reads x,
        yield (E.ecasq_matvec(other, *small, 128, out=x), y)  # which this writes

    both(steps)


@pytest.mark.parametrize("levels", [8, 16])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("b,heads,kv,d,n", [(1, 8, 8, 64, 40), (1, 8, 2, 128, 700), (2, 4, 4, 256, 3000), (40, 16, 8, 128, 900), (300, 2, 1, 32, 250)])
def test_a_layer_decodes(b, heads, kv, d, n, dtype, levels):
    """Product, cache writes, attention over the rows just written (one split, a cluster's join, both forms of the join's kernel),
    product, next token."""
    import paper_2608_18147_gb300 as E
    gen = torch.Generator(device="cuda").manual_seed(n)
    width, page, count = 256, 16, 6
    qkv, last = matrix((heads + 2 * kv) * d, width, dtype, gen), matrix(width, heads * d, dtype, gen)
    per = -(-n // page)
    table = torch.randperm(b * per, generator=gen, device="cuda").view(b, per).to(torch.int32)
    kept = []
    for _ in range(2):
        codes = torch.randint(0, 256, (b * per, page, kv, d // 2), generator=gen, device="cuda", dtype=torch.uint8)
        codes &= 0x77 if levels == 8 else 0xFF
        kept.append((codes, torch.sort(torch.randn(b * per, page, kv, levels, generator=gen, device="cuda")).values.to(dtype)))
    (k0, kl0), (v0, vl0) = kept
    caches = [t.clone() for t in (k0, kl0, v0, vl0)]
    k, kl, v, vl = caches
    book = torch.linspace(-2, 2, levels, device="cuda").repeat(b * kv, 1).contiguous()
    at = [n - count + t for t in range(count)]
    slots = [table[:, t // page].long() * page + t % page for t in at]
    lengths = [torch.full((b,), t + 1, dtype=torch.int32, device="cuda") for t in at]
    first = torch.randn(b, width, generator=gen, device="cuda").to(dtype)
    x, made = torch.empty_like(first), torch.empty(b, (heads + 2 * kv) * d, dtype=dtype, device="cuda")
    mixed = torch.empty(b, heads, d, dtype=dtype, device="cuda")
    ws = E.workspace_attend(b, heads, kv, d, n)
    parts = made.view(b, heads + 2 * kv, d)
    q, nk, nv = parts[:, :heads], parts[:, heads:heads + kv], parts[:, heads + kv:]

    def steps():
        x.copy_(first)
        for t, start in zip(caches, (k0, kl0, v0, vl0)):
            t.copy_(start)
        for t in range(count):
            yield (E.ecasq_matvec(x, *qkv, 128, out=made),)
            yield E.ecasq_cache_write(nk, book, None, slots[t], k, kl, 2 * t)
            yield E.ecasq_cache_write(nv, book, None, slots[t], v, vl, 2 * t + 1)
            out, lse = E.ecasq_attend(q, k, v, table, lengths[t], k_levels=kl, v_levels=vl, max_len=n, out=mixed, ws=ws)
            yield out, lse
            yield (E.ecasq_matvec(mixed.view(b, heads * d), *last, 128, out=x), made, k, v, kl, vl, mixed, lse)

    both(steps)
