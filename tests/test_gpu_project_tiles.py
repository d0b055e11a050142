"""ecasq_project and ecasq_gated on the tensor cores, each of their kernels by value, against 64 bits.

What the choice of the kernel gives for each case is asked of the library and held against what the case is for, on the CPU too, so that a change of that choice
cannot leave a kernel without a test: every width of a tile, gated or not, with one, two and four sums a block of columns, for fp32 and 16-bit rows; columns shared by two to six blocks; blocks with several tiles; several panels of rows of x.

Bounds, with size = sum |w x| and norm = sqrt(sum (w x)^2) of an output.
Sums: 16 products a step, at most 16 steps a span, each cut off by a unit in the last place at most of a sum that is below the span's size, and as much again for the products of a step that are cut off to the largest one's: 32 2^-23 of
the size; the spans' fp32 additions 2^-24 of the size each.  Of fp32 rows the products are 2^-21 of themselves off.  Activations, bias, residual and the last rounding as in test_gpu_project.py.
fp32 in the root mean square, where a term that is lost shows (its products are 2^-17 to 2^-16 of the size): the products' 2^-21, 8 steps of 2^-23, and sqrt(spans) roundings of 2^-24, all of the norm; three times that for a single row or
column of at least nine outputs (the errors go with the results, which are about normal: the root mean square of nine is below 2.1 norms with 1 - 1e-7)."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_gpu_project import STEP, U, cut, dtypes  # noqa: E402

# width, shared by, more: "rounds" (a block takes several tiles), "panels"; n, k, b, group, type, gated
F32 = [
    (32, 1, "", 777, 70, 9, 128, 0), (32, 1, "rounds", 20000, 70, 9, 128, 0), (32, 2, "", 520, 130, 33, 32, 0), (32, 3, "", 777, 260, 9, 64, 0), (32, 6, "", 777, 700, 9, 128, 1),
    (32, 4, "", 777, 390, 9, 64, 1), (32, 5, "", 520, 520, 33, 32, 1),
    (64, 1, "rounds", 20000, 70, 33, 128, 0), (64, 2, "", 130, 130, 1500, 64, 0), (64, 4, "", 130, 390, 600, 32, 0), (64, 6, "", 777, 700, 33, 128, 1), (64, 3, "", 1500, 260, 33, 64, 1),
    (64, 5, "", 1030, 520, 33, 32, 1),
    (128, 1, "", 13000, 70, 65, 128, 0), (128, 4, "", 130, 390, 1500, 64, 0), (128, 5, "", 130, 520, 1030, 32, 0), (128, 6, "panels", 130, 5000, 1030, 128, 0), (128, 1, "rounds", 13000, 70, 65, 128, 1),
    (128, 2, "", 2500, 130, 100, 64, 1), (128, 3, "", 1500, 260, 65, 32, 1),
    (256, 1, "rounds", 9000, 70, 800, 128, 0), (256, 1, "", 13000, 70, 129, 64, 0), (256, 1, "rounds", 20000, 70, 129, 32, 0), (256, 1, "panels", 2500, 5000, 1030, 128, 0),
    (256, 1, "rounds", 13000, 130, 129, 128, 1), (256, 1, "", 4000, 70, 257, 64, 1), (256, 1, "rounds", 13000, 70, 129, 32, 1),
]
F16 = [
    (32, 1, "rounds", 20000, 70, 17, 128, 0), (32, 2, "", 520, 390, 33, 128, 0), (32, 6, "", 520, 2600, 33, 128, 0), (32, 3, "", 520, 260, 33, 64, 0), (32, 4, "", 520, 390, 33, 32, 0), (32, 5, "", 520, 520, 33, 32, 0), (32, 3, "", 520, 520, 33, 96, 0),
    (32, 3, "", 520, 520, 33, 128, 1), (32, 5, "", 520, 520, 33, 64, 1), (32, 2, "", 520, 130, 33, 32, 1), (32, 1, "rounds", 13000, 70, 17, 64, 1),
    (64, 1, "rounds", 20000, 130, 33, 128, 0), (64, 3, "", 2500, 1000, 100, 128, 0), (64, 2, "", 130, 1000, 1500, 64, 0), (64, 5, "", 130, 520, 800, 32, 0), (64, 6, "", 130, 2600, 600, 32, 0),
    (64, 4, "", 1030, 2600, 65, 128, 1), (64, 3, "", 2500, 700, 33, 64, 1), (64, 2, "", 2500, 390, 33, 32, 1), (64, 1, "rounds", 20000, 70, 33, 128, 1),
    (128, 1, "rounds", 4000, 70, 1030, 128, 0), (128, 3, "", 520, 1500, 1030, 128, 0), (128, 6, "", 2500, 5000, 65, 128, 0), (128, 2, "", 4000, 1000, 129, 64, 0), (128, 4, "", 130, 1500, 1500, 32, 0),
    (128, 3, "", 2500, 1500, 100, 128, 1), (128, 5, "", 130, 2600, 1030, 64, 1), (128, 2, "", 4000, 700, 65, 32, 1), (128, 1, "rounds", 6000, 70, 257, 128, 1),
    (256, 1, "rounds", 9000, 70, 800, 128, 0), (256, 1, "", 6000, 200, 600, 128, 0), (256, 1, "", 13000, 130, 129, 64, 0), (256, 1, "rounds", 9000, 70, 800, 64, 0), (256, 1, "", 9000, 70, 257, 32, 0),
    (256, 1, "rounds", 9000, 200, 800, 96, 0), (256, 1, "rounds", 6000, 70, 600, 128, 1), (256, 1, "", 9000, 70, 200, 64, 1), (256, 1, "rounds", 6000, 70, 520, 32, 1),
    (256, 1, "panels", 3000, 16500, 1030, 256, 0), (256, 1, "rounds", 2001, 2048, 2100, 512, 1),
]
CASES = [case + ("f32",) for case in F32] + [case + (("f16", "bf16")[i % 2],) for i, case in enumerate(F16)]


def plan(n, k, b, group, dtype, gated):
    from paper_2608_18147_gb300 import native
    to = (ctypes.c_int64 * 6)()
    kind = {"f32": native.F32, "f16": native.F16, "bf16": native.BF16}[dtype]
    assert native.lib().ecasq_project_plan(b, n, k, kind, group, gated, to) == native.OK
    return dict(zip(("width", "split", "held", "x_tiles", "w_tiles", "panel"), to))


def in_pieces(n, k):
    """The next sizes whose rows are whole pieces of 16 bytes."""
    return -(-n // 8) * 8, -(-k // 8) * 8


@pytest.mark.parametrize("width,split,more,n,k,b,group,gated,dtype", CASES)
def test_cases_reach_the_kernels_that_they_are_for(width, split, more, n, k, b, group, gated, dtype):
    for p in (plan(n, k, b, group, dtype, gated), plan(*in_pieces(n, k), b, group, dtype, gated)):
        assert (p["width"], p["split"]) == (width, split)
        assert more != "rounds" or p["x_tiles"] * p["w_tiles"] > p["held"]
        assert more != "panels" or p["panel"] < p["x_tiles"]


def test_every_kernel_has_a_case():
    spans = lambda group: 1 if group % 128 == 0 else 2 if group % 64 == 0 else 4  # noqa: E731
    have = {(c[0], spans(c[6]), c[7], c[8] == "f32") for c in CASES}
    assert have == {(w, s, g, f) for w in (32, 64, 128, 256) for s in (1, 2, 4) for g in (0, 1) for f in (False, True)}
    for f in (False, True):
        mine = [c for c in CASES if (c[8] == "f32") == f]
        assert {c[1] for c in mine} == {1, 2, 3, 4, 5, 6} and {c[0] for c in mine if c[2] == "rounds"} == {32, 64, 128, 256} and any(c[2] == "panels" for c in mine)


def rms_bound(k):
    return 2.0 ** -21 + 8 * 2.0 ** -23 + (6 * -(-k // 128)) ** 0.5 * 2.0 ** -24 + 2.0 ** -24


def terms(v):
    """The three bf16 terms of fp32 values: their upper 16 bits, of what is left each time."""
    out = []
    for _ in range(3):
        t = (v.view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)
        out.append(t.astype(np.float64))
        v = (v - t).astype(np.float32)
    assert (v == 0).all()
    return out


@pytest.mark.parametrize("k", [70, 390, 5000])
def test_the_fp32_bound_sees_each_product_of_terms(k):
    """The six products of terms stay below the bound, and without any one of them the error is above it."""
    rng = np.random.default_rng(k)
    x = rng.standard_normal((40, k)).astype(np.float32)
    book = rng.standard_normal(16).astype(np.float32)
    w = book[rng.integers(0, 16, (60, k))]
    xt, wt, exact = terms(x), terms(w), x.astype(np.float64) @ w.astype(np.float64).T
    norm = np.sqrt((x.astype(np.float64) ** 2) @ (w.astype(np.float64) ** 2).T)
    pairs = [(0, 0), (0, 1), (0, 2), (1, 0), (1, 1), (2, 0)]
    products = {p: xt[p[0]] @ wt[p[1]].T for p in pairs}
    off = lambda y: np.sqrt((((y - exact) / norm) ** 2).mean())  # noqa: E731
    assert off(sum(products.values())) < 2.0 ** -21 < rms_bound(k)
    for p in pairs:
        assert off(sum(products.values()) - products[p]) > 2 * rms_bound(k), p


def inputs(n, k, b, group, dtype, gated, m, gen):
    import paper_2608_18147_gb300 as E
    dt, rows = dtypes()[dtype], 2 * n if gated else n
    idx = torch.randint(0, 16, (rows, k), generator=gen, device="cuda", dtype=torch.uint8)
    levels = torch.sort(torch.randn(m, generator=gen, device="cuda")).values.to(dt)
    scales = ((torch.rand(rows, -(-k // group), generator=gen, device="cuda") + 0.25) / k ** 0.5).to(dt if n % 2 and dtype != "f32" else torch.float32)
    x = (2 * torch.randn(b, k, generator=gen, device="cuda")).to(dt)
    book = torch.zeros(16, dtype=torch.float64, device="cuda")
    book[:m] = levels.double()
    w = book[idx.long()]
    w *= scales.double().repeat_interleave(group, dim=1)[:, :k]
    return x, E.ecasq_pack(idx), levels, scales, w


def act64(v, name):
    if name == "relu":
        return v.clamp(min=0)
    if name == "silu":
        return v * torch.sigmoid(v)
    if name == "gelu":
        return v * torch.special.erfc(-v / 2 ** 0.5) / 2
    if name == "gelu_tanh":
        return v * torch.sigmoid(2 * (2 / np.pi) ** 0.5 * (v + 0.044715 * v ** 3))
    return v


def check(y, ref, tol, dtype):
    y = y.double()
    tol = U[dtype] * (ref.abs() + tol) + tol + STEP
    bad = ~((y - ref).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:5].tolist(), y[bad][:5].tolist(), ref[bad][:5].tolist(), tol[bad][:5].tolist())


def sums(x, w, k, dtype):
    """The products and how far off they may be."""
    xd = x.double()
    spans = -(-k // (128 if dtype == "f32" else 32)) * (6 if dtype == "f32" else 1)
    of_size = 32 * 2.0 ** -23 + spans * 2.0 ** -24 + (2.0 ** -21 if dtype == "f32" else 0)
    return xd @ w.T, of_size * (xd.abs() @ w.abs().T)


def check_fp32(y, p, x, w, k):
    norm = (x.double().square() @ w.square().T).sqrt()
    off = ((y.double() - p) / norm).square()
    bound = rms_bound(k)
    assert off.mean().sqrt() <= bound, (off.mean().sqrt().item(), bound)
    for d in (0, 1):
        if off.shape[d] >= 9:
            assert off.mean(dim=d).amax().sqrt() <= 3 * bound, (d, off.mean(dim=d).amax().sqrt().item(), bound)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["pieces", "anywhere"])
@pytest.mark.parametrize("width,split,more,n,k,b,group,gated,dtype", CASES)
def test_values(width, split, more, n, k, b, group, gated, dtype, layout):
    """The product alone; then with an activation and, not gated, bias and residual.  Rows of whole pieces, side by side; or in wider tensors at odd places, of which nothing
    else is touched."""
    import paper_2608_18147_gb300 as E
    gen = torch.Generator(device="cuda").manual_seed(n + k + b)
    lead, pad = (0, 0) if layout == "pieces" else (1 + n % 3, 2)
    if layout == "pieces":
        n, k = in_pieces(n, k)
    m = 16 if layout == "pieces" else 13
    x, codes, levels, scales, w = inputs(n, k, b, group, dtype, gated, m, gen)
    p, dp = sums(x, w, k, dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    given = cut(x, lead, pad)

    def run(**more):
        out = cut(torch.zeros(b, n, dtype=x.dtype), lead, pad)
        fn = E.ecasq_gated if gated else E.ecasq_project
        y = fn(given, codes, levels, scales, group, out=out, status=status, **more)
        assert y is out and status.item() == 0
        if lead:
            assert out._base[:, :lead].isnan().all() and out._base[:, lead + n:].isnan().all()
        return y

    act = ("relu", "silu", "gelu", "gelu_tanh")[(n + k + b) % 4]
    slope = 1.13
    if gated:
        for name in (None, act):
            y = run(activation=name)
            g, dg = act64(p[:, :n], name), slope * dp[:, :n] + (2.0 ** -18 * p[:, :n].abs() if name else 0)
            u, du = p[:, n:], dp[:, n:]
            ref = g * u
            check(y, ref, dg * u.abs() + g.abs() * du + dg * du + 2.0 ** -23 * ref.abs(), dtype)
            if dtype == "f32" and not name:  # each factor's error goes with the other factor: the larger of two ratios, whose squares add up to no more than twice the bound's
                norm = (x.double().square() @ w.square().T).sqrt()
                off = ((y.double() - ref) / (norm[:, :n] * u.abs() + norm[:, n:] * g.abs())).square()
                assert off.mean().sqrt() <= 2 ** 0.5 * rms_bound(k), (off.mean().sqrt().item(), rms_bound(k))
        return
    y = run()
    check(y, p, dp, dtype)
    if dtype == "f32":
        check_fp32(y, p, x, w, k)
    bias = torch.randn(n, generator=gen, device="cuda").to(x.dtype)
    residual = cut((3 * torch.randn(b, n, generator=gen, device="cuda")).to(x.dtype), lead, pad)
    v = p + bias.double()
    ref = act64(v, act) + residual.double()
    tol = slope * (dp + 2.0 ** -23 * v.abs()) + 2.0 ** -18 * v.abs() + 2.0 ** -23 * ref.abs()
    check(run(bias=bias, activation=act, residual=residual), ref, tol, dtype)
    check(run(residual=residual), p + residual.double(), dp + 2.0 ** -23 * (p.abs() + residual.double().abs()), dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("gated", [0, 1])
def test_a_prompt_by_its_rows_and_columns(gated):
    """8192 x 8192 by 4096 rows, seven tiles a pair and several panels: 60 of the rows of x against all outputs, and 60 outputs against all rows."""
    import paper_2608_18147_gb300 as E
    n, k, b, group = 8192 // (1 + gated), 8192, 4096, 128
    p = plan(n, k, b, group, "bf16", gated)
    assert p["width"] == 256 and p["panel"] < p["x_tiles"] and p["x_tiles"] * p["w_tiles"] > 6 * p["held"]
    gen = torch.Generator(device="cuda").manual_seed(gated)
    x, codes, levels, scales, w = inputs(n, k, b, group, "bf16", gated, 16, gen)
    residual = torch.randn(b, n, generator=gen, device="cuda").bfloat16()
    y = E.ecasq_gated(x, codes, levels, scales, group, activation=None) if gated else E.ecasq_project(x, codes, levels, scales, group, residual=residual)
    some_x, some_n = (torch.randperm(s, generator=gen, device="cuda")[:60] for s in (b, n))
    for rows, cols in ((some_x, torch.arange(n, device="cuda")), (torch.arange(b, device="cuda"), some_n)):
        part = torch.cat([cols, cols + n]) if gated else cols
        q, dq = sums(x[rows], w[part], k, "bf16")
        got = y[rows][:, cols]
        if gated:
            (g, u), (dg, du) = q.chunk(2, dim=1), dq.chunk(2, dim=1)
            check(got, g * u, dg * u.abs() + g.abs() * du + dg * du + 2.0 ** -23 * (g * u).abs(), "bf16")
        else:
            r = residual[rows][:, cols].double()
            check(got, q + r, dq + 2.0 ** -23 * (q.abs() + r.abs()), "bf16")
