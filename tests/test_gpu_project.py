"""Products with 4-bit weights and what follows them (ecasq_project, ecasq_gated) against plain implementations in 64 bits.

Tolerance, per output.  The product p of k terms: fp32 sums of products that are exact or rounded once are, in any order that
adds sixteen terms a step, within (k / 8 + 16) 2^-23 sum |w x| =: dp of the exact one.  An activation stretches an error by
at most 1.13 (gelu's steepest slope) and is itself off by at most 2^-18 |v|: an exponential off by 2^-21 of itself, of an argument below 17 rounded
to 2^-20 or better (beyond 17 every activation is within 2^-22 |v| of its limit).  Bias and residual are fp32 additions (2^-23 of the result), and the result is rounded once, by half a step at most.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
STEP = 2.0 ** -25  # half of f16's smallest step


def dtypes():
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def act64(v, name):
    if name == "relu":
        return np.where(v > 0, v, 0)
    if name == "silu":
        return v / (1 + np.exp(-v))
    if name == "gelu":
        return torch.nn.functional.gelu(torch.from_numpy(v)).numpy()
    if name == "gelu_tanh":
        return 0.5 * v * (1 + np.tanh(np.sqrt(2 / np.pi) * (v + 0.044715 * v ** 3)))
    return v


def matrix(g, n, k, group, dtype, scale_dtype, m=16):
    dt, sd = dtypes()[dtype], dtypes()[scale_dtype]
    idx = torch.randint(0, 16, (n, k), generator=g, dtype=torch.uint8)
    levels = torch.sort(torch.randn(m, generator=g)).values.to(dt)
    scales = ((torch.rand(n, -(-k // group), generator=g) + 0.25) / k ** 0.5).to(sd)
    return idx, levels, scales


def products(x, idx, levels, scales, group):
    """(p, dp) in binary64: codes beyond the codebook stand for 0."""
    book = np.zeros(16)
    book[:levels.numel()] = levels.double().numpy()
    k = idx.shape[1]
    w = book[idx.numpy()] * np.repeat(scales.double().numpy(), group, axis=1)[:, :k]
    xd = x.double().numpy()
    return xd @ w.T, (k / 8 + 16) * 2.0 ** -23 * (np.abs(xd) @ np.abs(w).T)


def check(y, ref, tol, dtype):
    y = y.double().cpu().numpy()
    tol = U[dtype] * (np.abs(ref) + tol) + tol + STEP
    bad = ~(np.abs(y - ref) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5], y[bad][:5], ref[bad][:5], tol[bad][:5])


def cut(t, lead, pad, dev="cuda"):
    """t [rows, cols] on the device as a part of a wider tensor: `lead` entries before each row, `pad` behind it."""
    wide = torch.full((t.shape[0], lead + t.shape[1] + pad), float("nan") if t.is_floating_point() else 85, dtype=t.dtype, device=dev)
    part = wide[:, lead:lead + t.shape[1]]
    part.copy_(t)
    return part


def project_case(n, k, b, group, dtype, scale_dtype, act, bias, residual, lead=0, pad=0, m=16, seed=0, ws=True):
    import paper_2608_18147_gb300 as E
    g = torch.Generator().manual_seed(seed + 7 * n + k + b)
    dt = dtypes()[dtype]
    idx, levels, scales = matrix(g, n, k, group, dtype, scale_dtype, m)
    x = (torch.randn(b, k, generator=g) * 2).to(dt)
    vec = torch.randn(n, generator=g).to(dt) if bias else None
    res = (3 * torch.randn(b, n, generator=g)).to(dt) if residual else None
    codes = E.ecasq_pack(idx.cuda())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = cut(torch.zeros(b, n, dtype=dt), lead, pad)
    space = E.workspace_project(b, n, k, dt) if ws else None
    y = E.ecasq_project(cut(x, lead, pad), codes, levels.cuda(), scales.cuda(), group, bias=None if vec is None else vec.cuda(), activation=act,
                        residual=None if res is None else cut(res, lead, pad), out=out, ws=space, status=status)
    assert y is out and status.item() == 0
    around = out._base.double().cpu() if out._base is not None else None
    if around is not None and (lead or pad):  # what lies beside the rows is left as it was
        assert around[:, :lead].isnan().all() and around[:, lead + n:].isnan().all()
    p, dp = products(x, idx, levels, scales, group)
    v = p + (vec.double().numpy() if bias else 0)
    tol = 1.13 * (dp + 2.0 ** -23 * np.abs(v)) + (2.0 ** -18 * np.abs(v) if act else 0)
    ref = act64(v, act) + (res.double().numpy() if residual else 0)
    check(y, ref, tol + 2.0 ** -23 * np.abs(ref), dtype)


def gated_case(n, k, b, group, dtype, scale_dtype, act, lead=0, pad=0, m=16, seed=0):
    import paper_2608_18147_gb300 as E
    g = torch.Generator().manual_seed(seed + 7 * n + k + b)
    dt = dtypes()[dtype]
    idx, levels, scales = matrix(g, 2 * n, k, group, dtype, scale_dtype, m)
    x = (torch.randn(b, k, generator=g) * 2).to(dt)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = cut(torch.zeros(b, n, dtype=dt), lead, pad)
    y = E.ecasq_gated(cut(x, lead, pad), E.ecasq_pack(idx.cuda()), levels.cuda(), scales.cuda(), group, activation=act, out=out, status=status)
    assert y is out and status.item() == 0
    p, dp = products(x, idx, levels, scales, group)
    a, da = act64(p[:, :n], act), 1.13 * dp[:, :n] + 2.0 ** -18 * np.abs(p[:, :n])
    u, du = p[:, n:], dp[:, n:]
    ref = a * u
    check(y, ref, da * np.abs(u) + np.abs(a) * du + da * du + 2.0 ** -23 * np.abs(ref), dtype)


CASES = [
    # n, k, b, group, dtype, scales
    (1, 1, 1, 32, "bf16", "f32"),
    (5, 33, 1, 32, "f16", "f16"),
    (64, 128, 2, 128, "bf16", "bf16"),
    (100, 300, 8, 64, "f16", "f32"),
    (257, 1000, 9, 96, "bf16", "f32"),
    (300, 520, 16, 128, "f16", "f16"),
    (130, 2048, 17, 256, "bf16", "bf16"),
    (513, 129, 31, 32, "f16", "f32"),
    (384, 640, 33, 128, "bf16", "f32"),
    (1000, 384, 64, 32, "bf16", "bf16"),
    (259, 1100, 65, 64, "f16", "f32"),
    (512, 513, 100, 128, "bf16", "f32"),
    (140, 700, 128, 96, "f16", "f16"),
    (1025, 256, 129, 128, "bf16", "f32"),
    (300, 1536, 200, 1536, "f16", "f32"),
    (260, 896, 256, 64, "bf16", "f32"),
    (777, 400, 257, 32, "f16", "f32"),
    (512, 1024, 513, 128, "bf16", "bf16"),
    (33, 70, 700, 64, "f16", "f16"),
    (7, 50, 1, 32, "f32", "f32"),
    (300, 513, 3, 96, "f32", "f32"),
    (130, 1024, 8, 128, "f32", "f32"),
    (257, 640, 9, 64, "f32", "f32"),
    (512, 300, 40, 128, "f32", "f32"),
    (140, 2000, 130, 32, "f32", "f32"),
    (600, 513, 300, 256, "f32", "f32"),
]


@pytest.mark.parametrize("n,k,b,group,dtype,scales", CASES)
def test_project(n, k, b, group, dtype, scales):
    project_case(n, k, b, group, dtype, scales, None, False, False)


@pytest.mark.parametrize("n,k,b,group,dtype,scales", CASES)
def test_project_with_everything(n, k, b, group, dtype, scales):
    """Bias, an activation and the residual; rows off 16-byte boundaries, in wider tensors."""
    act = ("relu", "silu", "gelu", "gelu_tanh")[(n + k + b) % 4]
    project_case(n, k, b, group, dtype, scales, act, True, True, lead=1 + (n + b) % 3, pad=2, m=13, seed=1)


@pytest.mark.parametrize("n,k,b,group,dtype,scales", CASES)
def test_gated(n, k, b, group, dtype, scales):
    act = ("silu", "gelu", "gelu_tanh", "relu", None)[(n + k + b) % 5]
    gated_case(n, k, b, group, dtype, scales, act)


@pytest.mark.parametrize("n,k,b,group,dtype,scales", CASES[::3])
def test_gated_in_wider_tensors(n, k, b, group, dtype, scales):
    gated_case(n, k, b, group, dtype, scales, "silu", lead=3, pad=1, m=11, seed=2)


@pytest.mark.parametrize("act", [None, "relu", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("b", [3, 50])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_activations(dtype, b, act):
    project_case(200, 260, b, 64, dtype, "f32", act, True, False, seed=3)
    project_case(200, 260, b, 64, dtype, "f32", act, False, True, seed=4)
    gated_case(72, 260, b, 64, dtype, "f32", act, seed=5)


def some(n=320, k=384, b=24, dtype="bf16", seed=9, rows=None):
    import paper_2608_18147_gb300 as E
    g = torch.Generator().manual_seed(seed)
    idx, levels, scales = matrix(g, rows or n, k, 128, dtype, "f32")
    x = torch.randn(b, k, generator=g).to(dtypes()[dtype])
    return x.cuda(), E.ecasq_pack(idx.cuda()), levels.cuda(), scales.cuda(), 128


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("b", [1, 6, 24, 200])
def test_the_residual_in_place(dtype, b):
    import paper_2608_18147_gb300 as E
    args = some(b=b, dtype=dtype)
    res = torch.randn(b, 320, device="cuda").to(args[0].dtype)
    want = E.ecasq_project(*args, residual=res, activation="silu")
    got = E.ecasq_project(*args, residual=res, activation="silu", out=res)
    assert got is res and torch.equal(got, want)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_one_row_without_a_batch(dtype):
    import paper_2608_18147_gb300 as E
    x, *rest = some(b=1, dtype=dtype)
    bias, res = torch.randn(320, device="cuda").to(x.dtype), torch.randn(320, device="cuda").to(x.dtype)
    y = E.ecasq_project(x[0], *rest, bias=bias, residual=res)
    assert y.shape == (320,) and torch.equal(y, E.ecasq_project(x, *rest, bias=bias, residual=res[None])[0])
    h = E.ecasq_gated(x[0], *rest)
    assert h.shape == (160,) and torch.equal(h, E.ecasq_gated(x, *rest)[0])


def test_no_rows():
    import paper_2608_18147_gb300 as E
    x, *rest = some()
    assert E.ecasq_project(x[:0], *rest).shape == (0, 320) and E.ecasq_gated(x[:0], *rest).shape == (0, 160)


@pytest.mark.parametrize("b", [1, 5, 24, 300])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_rows_do_not_depend_on_the_others(dtype, b):
    """Rows that are not finite change no other, and nothing else but them."""
    import paper_2608_18147_gb300 as E
    x, *rest = some(b=b + 2, dtype=dtype)
    bad = x.clone()
    bad[0, 3] = float("inf")
    bad[-1, 7] = float("nan")
    for fn in (E.ecasq_project, E.ecasq_gated):
        y, z = fn(x, *rest), fn(bad, *rest)
        assert torch.equal(y[1:-1], z[1:-1]) and not z[0].isfinite().any() and z[-1].isnan().all()


@pytest.mark.parametrize("b", [2, 40, 200])
def test_equal_calls_give_equal_bits(b):
    import paper_2608_18147_gb300 as E
    for dtype in ("f32", "bf16"):
        args = some(n=1000, k=2000, b=b, dtype=dtype)
        assert torch.equal(E.ecasq_project(*args), E.ecasq_project(*args))
        assert torch.equal(E.ecasq_gated(*args), E.ecasq_gated(*args))


@pytest.mark.parametrize("b", [4, 40, 300])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_a_graph_and_on_another_stream(dtype, b):
    import paper_2608_18147_gb300 as E
    x, *rest = some(b=b, dtype=dtype)
    ws = E.workspace_project(b, 320, 384, x.dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = E.ecasq_project(x, *rest, activation="gelu", ws=ws), E.ecasq_gated(x, *rest, ws=ws)
    torch.cuda.current_stream().wait_stream(side)
    y, h = torch.zeros_like(want[0]), torch.zeros_like(want[1])
    x2 = x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        E.ecasq_project(x2, *rest, activation="gelu", out=y, ws=ws)
        E.ecasq_gated(x2, *rest, out=h, ws=ws)
    for scale in (1.0, 2.0):
        x2.copy_(x * scale)
        graph.replay()
        assert torch.equal(y, E.ecasq_project(x2, *rest, activation="gelu")) and torch.equal(h, E.ecasq_gated(x2, *rest))
        if scale == 1.0:
            assert torch.equal(y, want[0]) and torch.equal(h, want[1])


def test_refusals():
    import paper_2608_18147_gb300 as E
    x, codes, levels, scales, group = args = some()
    good = torch.zeros(24, 320, dtype=x.dtype, device="cuda")
    bias = torch.zeros(320, dtype=x.dtype, device="cuda")
    for change in (dict(activation="tanh"), dict(activation=3), dict(bias=bias[:-1]), dict(bias=bias.float()), dict(bias=bias.cpu()),
                   dict(residual=good[:, :-1]), dict(residual=good.float()), dict(residual=good.T), dict(out=good[:-1]), dict(out=good.half()),
                   dict(out=torch.zeros(320, 24, dtype=x.dtype, device="cuda").T), dict(ws=bias), dict(status=bias), dict(residual=good[0])):
        with pytest.raises(E.EcasqError) as err:
            E.ecasq_project(*args, **change)
        assert err.value.code == -1
    for wrong in ((x.double(),) + args[1:], (x[:, :-1].T,) + args[1:], (x, codes[:, :-64], levels, scales, group), (x, codes, levels.float(), scales, group),
                  (x, codes, levels, scales[:, :-1], group), (x, codes, levels, scales, 48), (x, codes, levels, scales[:-1], group), (x, codes, levels, scales, "a")):
        for fn in (E.ecasq_project, E.ecasq_gated):
            with pytest.raises(E.EcasqError):
                fn(*wrong)
    with pytest.raises(E.EcasqError, match="even"):
        E.ecasq_gated(x, codes[:-1], levels, scales[:-1], group)
    with pytest.raises(E.EcasqError):
        E.ecasq_gated(*args, out=good)


def test_gradients_are_refused():
    import paper_2608_18147_gb300 as E
    x, codes, levels, scales, group = some(dtype="f16")
    bias, res = torch.zeros(320, device="cuda").half(), torch.zeros(24, 320, device="cuda").half()
    good = dict(x=x, codes=codes, levels=levels, scales=scales, group=group)
    for fn, names in ((E.ecasq_project, ("x", "levels", "scales", "bias", "residual")), (E.ecasq_gated, ("x", "levels", "scales"))):
        full = dict(good, bias=bias, residual=res) if fn is E.ecasq_project else good
        for name in names:
            wants = dict(full, **{name: full[name].clone().requires_grad_()})
            with pytest.raises(E.EcasqError, match="gradient"):
                fn(**wants)
            with torch.no_grad():
                fn(**wants)
