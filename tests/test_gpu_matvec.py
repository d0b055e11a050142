"""Products with 4-bit weights (ecasq_pack, ecasq_matvec) against a plain implementation in 64 bits.

Tolerance, per output: the one rounding to the output's type (unit roundoff u times |y|) and fp32 sums.
A sum of k products that is built from exact or once-rounded products in any order, every
step within 2^-23 of its result, is within (k + 8) 2^-23 sum |w x| of the exact one; steps that add 16 products
at once take a sixteenth of that many.  The bound below uses k / 8 + 16 steps.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def dtypes():
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def make(n, k, b, group, dtype, scale_dtype, seed=0, m=16):
    g = torch.Generator().manual_seed(seed)
    dt, sd = dtypes()[dtype], dtypes()[scale_dtype]
    idx = torch.randint(0, 16, (n, k), generator=g, dtype=torch.uint8)
    levels = torch.sort(torch.randn(m, generator=g)).values.to(dt)
    scales = (torch.rand(n, -(-k // group), generator=g) + 0.25).to(sd)
    x = torch.randn(b, k, generator=g).to(dt)
    return x, idx, levels, scales


def reference(x, idx, levels, scales, group):
    """(y, sum |w x|) in binary64: codes beyond the codebook stand for 0."""
    book = np.zeros(16)
    book[:levels.numel()] = levels.double().numpy()
    k = idx.shape[1]
    s = np.repeat(scales.double().numpy(), group, axis=1)[:, :k]
    w = book[idx.numpy()] * s
    xd = x.double().numpy()
    return xd @ w.T, np.abs(xd) @ np.abs(w).T


def check(y, ref, size, k, dtype):
    y = y.double().cpu().numpy()
    tol = U[dtype] * np.abs(ref) + (k / 8 + 16) * 2.0 ** -23 * size + 2.0 ** -25  # the last: f16's smallest steps
    bad = ~(np.abs(y - ref) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5], y[bad][:5], ref[bad][:5], tol[bad][:5])


CASES = [
    (1, 1, 1, 32), (1, 7, 2, 32), (3, 31, 1, 32), (8, 32, 1, 32), (9, 33, 8, 32), (16, 127, 3, 64), (17, 128, 2, 128),
    (31, 129, 4, 96), (40, 257, 5, 32), (65, 640, 8, 160), (130, 1000, 1, 96), (300, 2050, 3, 64), (1216, 384, 8, 128),
    (2500, 520, 2, 256), (24, 9000, 8, 64), (7, 20001, 1, 1 << 20),
    (37, 25000, 8, 96), (700, 11400, 8, 128),
]


@pytest.mark.parametrize("dtype,scale_dtype", [("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("n,k,b,group", CASES)
def test_matches_64_bits(n, k, b, group, dtype, scale_dtype):
    import paper_2608_18147_gb300 as E
    x, idx, levels, scales = make(n, k, b, group, dtype, scale_dtype, seed=n + k)
    y = E.ecasq_matvec(x.cuda(), E.ecasq_pack(idx.cuda()), levels.cuda(), scales.cuda(), group)
    assert y.dtype == x.dtype and y.shape == (b, n)
    ref, size = reference(x, idx, levels, scales, group)
    check(y, ref, size, k, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("b", [9, 16, 21])
def test_more_rows_than_eight(b, dtype):
    import paper_2608_18147_gb300 as E
    x, idx, levels, scales = make(200, 500, b, 64, dtype, "f32", seed=b)
    y = E.ecasq_matvec(x.cuda(), E.ecasq_pack(idx.cuda()), levels.cuda(), scales.cuda(), 64)
    ref, size = reference(x, idx, levels, scales, 64)
    check(y, ref, size, 500, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m", [1, 2, 5, 15])
def test_short_codebooks(m, dtype):
    """Codes beyond the codebook stand for 0."""
    import paper_2608_18147_gb300 as E
    x, idx, levels, scales = make(50, 300, 2, 32, dtype, "f32", seed=m, m=m)
    y = E.ecasq_matvec(x.cuda(), E.ecasq_pack(idx.cuda()), levels.cuda(), scales.cuda(), 32)
    ref, size = reference(x, idx, levels, scales, 32)
    check(y, ref, size, 300, dtype)


def test_pack_layout():
    """Word w of a block holds columns 8w .. 8w+7, lowest first, at position 4 (w mod 4) + w div 4; padding is zero."""
    import paper_2608_18147_gb300 as E
    for n, k in ((1, 1), (2, 128), (5, 300), (3, 129)):
        idx = torch.randint(0, 256, (n, k), dtype=torch.uint8)
        got = E.ecasq_pack(idx.cuda()).cpu().numpy()
        assert got.shape == (n, 64 * -(-k // 128))
        want = np.zeros_like(got)
        for c in range(k):
            block, w, j = c // 128, c % 128 // 8, c % 8
            at = 64 * block + 4 * (4 * (w % 4) + w // 4) + j // 2
            want[:, at] |= ((idx[:, c].numpy() & 15) << (4 * (j % 2))).astype(np.uint8)
        np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_columns_beyond_k_do_not_count(dtype):
    """Whatever the padding of the packed rows and of the scales' rows holds."""
    import paper_2608_18147_gb300 as E
    n, k, b, group = 37, 131, 3, 32
    x, idx, levels, scales = make(n, k, b, group, dtype, "f32", seed=5)
    codes = torch.full((n, 64 * 2 + 64), 255, dtype=torch.uint8)
    packed = E.ecasq_pack(idx.cuda()).cpu()
    wide = torch.full((n, 256), 15, dtype=torch.uint8)
    wide[:, :k] = idx
    codes[:, :128] = E.ecasq_pack(wide.cuda()).cpu()
    assert not torch.equal(codes[:, :128], packed)
    many = torch.full((n, 9), float("nan"))
    many[:, :scales.shape[1]] = scales
    wider = torch.full((b, k + 5), float("nan"), dtype=x.dtype)
    wider[:, :k] = x
    y = E.ecasq_matvec(wider.cuda()[:, :k], codes.cuda(), levels.cuda(), many.cuda(), group)
    ref, size = reference(x, idx, levels, scales, group)
    check(y, ref, size, k, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_strides_and_out(dtype):
    """Rows of x and y apart from one another and at odd places; nothing else of out is written."""
    import paper_2608_18147_gb300 as E
    n, k, b, group = 61, 517, 4, 64
    x, idx, levels, scales = make(n, k, b, group, dtype, "f32", seed=9)
    flat = torch.zeros(b * 601 + 3, dtype=x.dtype, device="cuda")
    xs = flat[3:].view(b, 601)[:, 1:1 + k]
    xs.copy_(x)
    room = torch.full((b, n + 7), 42.0, dtype=x.dtype, device="cuda")
    out = room[:, 3:3 + n]
    y = E.ecasq_matvec(xs, E.ecasq_pack(idx.cuda()), levels.cuda(), scales.cuda(), group, out=out)
    assert y is out
    ref, size = reference(x, idx, levels, scales, group)
    check(out, ref, size, k, dtype)
    assert (room[:, :3] == 42).all() and (room[:, 3 + n:] == 42).all()
    one = E.ecasq_matvec(xs[2], E.ecasq_pack(idx.cuda()), levels.cuda(), scales.cuda(), group)
    assert one.shape == (n,)
    check(one, ref[2], size[2], k, dtype)


@pytest.mark.parametrize("dtype,scale_dtype", [("bf16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("before,row", [(1, 0), (3, 1), (5, 3), (8, 8)])
def test_scales_at_any_address(before, row, group, dtype, scale_dtype):
    """Scales that begin anywhere, their rows apart by anything; what lies around them is NaN."""
    import paper_2608_18147_gb300 as E
    n, k, b = 300, 700, 2
    x, idx, levels, scales = make(n, k, b, group, dtype, scale_dtype, seed=before)
    wide = scales.shape[1] + row
    flat = torch.full((before + n * wide + 9,), float("nan"), dtype=scales.dtype, device="cuda")
    part = flat[before:before + n * wide].view(n, wide)[:, :scales.shape[1]]
    part.copy_(scales)
    y = E.ecasq_matvec(x.cuda(), E.ecasq_pack(idx.cuda()), levels.cuda(), part, group)
    ref, size = reference(x, idx, levels, scales, group)
    check(y, ref, size, k, dtype)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,k,b,group", [(90000, 130, 1, 32), (90001, 256, 3, 128), (5000, 4200, 1, 64), (1300, 16500, 2, 128),
                                         (152 * 40, 6144, 1, 32), (20, 16384, 8, 32), (8, 8192, 1, 8192)])
def test_many_rows_and_columns(n, k, b, group, dtype):
    """More rows than one block takes, several passes over the columns, every split of the warps between them."""
    import paper_2608_18147_gb300 as E
    x, idx, levels, scales = make(n, k, b, group, dtype, "f32", seed=n)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    y = E.ecasq_matvec(x.cuda(), E.ecasq_pack(idx.cuda()), levels.cuda(), scales.cuda(), group, status=status)
    assert status.item() == 0
    some = torch.cat([torch.arange(0, n, max(1, n // 500)), torch.arange(max(0, n - 40), n)])
    ref, size = reference(x, idx[some], levels, scales[some], group)
    check(y[:, some.cuda()], ref, size, k, dtype)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,k,b,group", [(393, 15530, 2, 128), (64, 16384, 1, 64), (1000, 8192, 8, 128), (700, 20001, 3, 32), (300, 28672, 5, 96),
                                         (1, 16640, 1, 128), (77, 16385, 7, 256), (2046, 16384, 1, 128), (4100, 28672, 4, 128), (40000, 12800, 1, 128)])
def test_columns_shared_by_a_cluster(n, k, b, group, dtype):
    """Few rows and many columns, whose sums several blocks share, at sizes that do not divide evenly; twice for equal bits."""
    import paper_2608_18147_gb300 as E
    x, idx, levels, scales = make(n, k, b, group, dtype, "f32", seed=n + k)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = (x.cuda(), E.ecasq_pack(idx.cuda()), levels.cuda(), scales.cuda(), group)
    y = E.ecasq_matvec(*args, status=status)
    assert status.item() == 0 and torch.equal(y, E.ecasq_matvec(*args))
    some = torch.cat([torch.arange(0, n, max(1, n // 300)), torch.arange(max(0, n - 40), n)])
    ref, size = reference(x, idx[some], levels, scales[some], group)
    check(y[:, some.cuda()], ref, size, k, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_nan_and_inf_stay_in_their_row(dtype):
    import paper_2608_18147_gb300 as E
    n, k, b = 40, 260, 5
    x, idx, levels, scales = make(n, k, b, 32, dtype, "f32", seed=2)
    x[1, 259] = float("nan")
    x[3, 0] = float("inf")
    y = E.ecasq_matvec(x.cuda(), E.ecasq_pack(idx.cuda()), levels.cuda(), scales.cuda(), 32)
    assert torch.isnan(y[1]).all()
    assert not torch.isfinite(y[3]).any()
    keep = [0, 2, 4]
    ref, size = reference(x[keep], idx, levels, scales, 32)
    check(y[keep], ref, size, k, dtype)


def test_equal_calls_give_equal_bits_in_a_graph_and_on_another_stream():
    import paper_2608_18147_gb300 as E
    x, idx, levels, scales = make(700, 1111, 8, 32, "bf16", "f32", seed=3)
    args = (x.cuda(), E.ecasq_pack(idx.cuda()), levels.cuda(), scales.cuda(), 32)
    first = E.ecasq_matvec(*args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = E.ecasq_matvec(*args)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, second)
    graph = torch.cuda.CUDAGraph()
    out = torch.empty_like(first)
    with torch.cuda.graph(graph):
        E.ecasq_matvec(*args, out=out)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(first, out)


def test_empty_batch_and_refusals():
    import paper_2608_18147_gb300 as E
    x, idx, levels, scales = make(20, 100, 2, 32, "bf16", "f32")
    codes = E.ecasq_pack(idx.cuda())
    x, levels, scales = x.cuda(), levels.cuda(), scales.cuda()
    assert E.ecasq_matvec(x[:0], codes, levels, scales, 32).shape == (0, 20)
    bad = [
        (x.cpu(), codes, levels, scales, 32), (x.double(), codes, levels, scales, 32), (x, codes.int(), levels, scales, 32),
        (x, codes[:, :32], levels, scales, 32), (x, codes, levels.float(), scales, 32), (x, codes, levels, scales, 33),
        (x, codes, levels, scales, 0), (x, codes, levels, scales[:, :3], 32), (x, codes, levels, scales[:19], 32),
        (x, codes, torch.zeros(17, dtype=x.dtype, device="cuda"), scales, 32), (x, codes, levels, scales.double(), 32),
        (x, codes, levels[:0], scales, 32), (x.t().contiguous().t(), codes, levels, scales, 32),
    ]
    for args in bad:
        with pytest.raises(E.EcasqError):
            E.ecasq_matvec(*args)
    room = torch.zeros(20 * 64 + 8, dtype=torch.uint8, device="cuda")
    with pytest.raises(E.EcasqError):  # rows that do not start at multiples of 16 bytes
        E.ecasq_matvec(x, room[8:].view(20, 64), levels, scales, 32)
    for out in (torch.empty(2, 21, dtype=x.dtype, device="cuda"), torch.empty(2, 20, device="cuda")):
        with pytest.raises(E.EcasqError):
            E.ecasq_matvec(x, codes, levels, scales, 32, out=out)
    for idx in (idx, idx.cuda().int(), idx.cuda()[0], idx.cuda().t()):
        with pytest.raises(E.EcasqError):
            E.ecasq_pack(idx)


def test_waits_for_what_came_before():
    """Inputs written by a long kernel before the call, in its stream or in another one that its stream waits for, and outputs
    read behind it; with calls right before and after, whose launches overlap."""
    import paper_2608_18147_gb300 as E
    n, k, b = 1024, 1024, 4
    x, idx, levels, scales = make(n, k, b, 128, "bf16", "f32", seed=31)
    codes, levels, scales, x = E.ecasq_pack(idx.cuda()), levels.cuda(), scales.cuda(), x.cuda()
    right = E.ecasq_matvec(x, codes, levels, scales, 128)
    big = torch.randn(4096, 4096, device="cuda")
    here, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        late = torch.zeros_like(x)
        torch.cuda.synchronize()
        with torch.cuda.stream(here):
            torch.mm(big, big)
            late.copy_(x)
            first = E.ecasq_matvec(late, codes, levels, scales, 128)
            second = E.ecasq_matvec(late * 1, codes, levels, scales, 128)
            kept = second.clone()
            second.zero_()
        torch.cuda.synchronize()
        assert torch.equal(first, right) and torch.equal(kept, right)
        late = torch.zeros_like(x)
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            torch.mm(big, big)
            late.copy_(x)
            done = other.record_event()
        with torch.cuda.stream(here):
            E.ecasq_matvec(x, codes, levels, scales, 128)
            here.wait_event(done)
            third = E.ecasq_matvec(late, codes, levels, scales, 128)
        torch.cuda.synchronize()
        assert torch.equal(third, right)
