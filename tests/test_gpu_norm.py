"""Norms with the residual's addition and 8-bit outputs (ecasq_norm) against a plain implementation in 64 bits.

Tolerance.  s is one fp32 addition and a rounding to the type, so equal bits are asked for.  The mean of k squares in fp32, added in any
tree of at most k / 16 + 16 steps, is within (k / 16 + 18) 2^-24 of itself; half of that enters y, with five more fp32 roundings
and the last to the type.  An 8-bit value is off by half a step of e4m3: 2^-4 of itself, or 2^-10 below 2^-6, and by what
the value before it is off.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def dtypes():
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def cut(t, lead, pad):
    wide = torch.full((t.shape[0], lead + t.shape[1] + pad), 0 if t.dtype == torch.float8_e4m3fn else float("nan"), dtype=torch.float32, device="cuda").to(t.dtype)
    part = wide[:, lead:lead + t.shape[1]]
    part.copy_(t)
    return part


def within(got, ref, rel, floor):
    got, room = got.double().cpu(), rel * ref.abs() + floor
    bad = ~((got - ref).abs() <= room)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4], got[bad][:4], ref[bad][:4])


def norm_case(b, k, dtype, weight_dtype, residual, group, lead=0, pad=0, eps=1e-6, seed=0, size=1.0):
    import paper_2608_18147_gb300 as E
    g = torch.Generator().manual_seed(seed + b + 3 * k)
    dt = dtypes()[dtype]
    x = (size * torch.randn(b, k, generator=g) * (torch.rand(b, 1, generator=g) + 0.1)).to(dt)
    res = (size * 2 * torch.randn(b, k, generator=g)).to(dt) if residual else None
    w = (1 + 0.3 * torch.randn(k, generator=g)).to(dtypes()[weight_dtype])
    given = {}
    if lead or pad:
        given["out"] = cut(torch.zeros(b, k, dtype=torch.float8_e4m3fn if group else dt), lead, pad)
        if residual:
            given["out_sum"] = cut(torch.zeros(b, k, dtype=dt), lead, pad)
        if group:
            given["out_scales"] = cut(torch.zeros(b, -(-k // group)), lead, pad)
    out = E.ecasq_norm(cut(x, lead, pad), w.cuda(), eps, residual=None if res is None else cut(res, lead, pad), group=group or None, **given)
    out = out if isinstance(out, tuple) else (out,)
    assert len(out) == 1 + bool(group) + residual
    for t in (given.get("out"), given.get("out_sum")):
        assert t is None or t is out[0] or t is out[-1]
    s = x if res is None else (x.float() + res.float()).to(dt)
    if residual:
        assert torch.equal(out[-1].cpu(), s)
    v = s.double()
    y = v / (v.square().mean(dim=1, keepdim=True) + eps).sqrt() * w.double()
    fp32 = (k / 32 + 15) * 2.0 ** -24
    if not group:
        within(out[0], y, U[dtype] * (1 + fp32) + fp32, 2.0 ** -25 if dtype == "f16" else 0)
        return
    groups = -(-k // group)
    wide = torch.nn.functional.pad(y, (0, groups * group - k)).view(b, groups, group)
    scale = wide.abs().amax(dim=2) / 448
    within(out[1], torch.where(scale > 0, scale, torch.ones_like(scale)), fp32 + 2.0 ** -23, 0)
    q = (wide / torch.where(scale > 0, scale, torch.ones_like(scale))[..., None]).flatten(1)[:, :k]
    off = 2 * fp32 + 2.0 ** -22
    within(out[0].float(), q, 2.0 ** -4 * (1 + off) + off, 2.0 ** -10 * (1 + off))


CASES = [(1, 1), (3, 7), (1, 64), (5, 100), (2, 255), (4, 256), (7, 1000), (1, 4096), (3, 4097), (9, 5003), (64, 6000), (300, 128), (2, 8192),
         (33, 2048), (5, 16384), (2, 20001), (3, 40000), (1, 70000), (1000, 96), (2, 131072)]


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype,weight", [("f32", "f32"), ("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("b,k", CASES)
def test_norm(b, k, dtype, weight, residual):
    norm_case(b, k, dtype, weight, residual, 0)
    norm_case(b, k, dtype, weight, residual, 0, lead=1 + k % 5, pad=3, seed=1)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("b,k", CASES)
def test_norm_to_8_bits(b, k, dtype, residual):
    for i, group in enumerate((16, 48, 64, 128, 512, k, k + 5)):
        lead = (0, 0, 3, 0, 1, 0, 2)[i]
        norm_case(b, k, dtype, "f32" if i % 2 else dtype, residual, group, lead=lead, pad=lead, seed=i)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_rows_of_zeros(dtype):
    """Zeros give zeros, whatever eps, and a scale of 1; with eps = 0 they have no size to divide by."""
    import paper_2608_18147_gb300 as E
    x = torch.zeros(3, 300, dtype=dtypes()[dtype], device="cuda")
    x[1] = 1
    w = torch.full((300,), 2.0, device="cuda")
    y = E.ecasq_norm(x, w, 1e-5)
    assert (y[0] == 0).all() and (y[2] == 0).all() and (y[1].float() - 2).abs().max() < 0.02
    q, scales = E.ecasq_norm(x, w, 1e-5, group=64)
    assert (q[0].float() == 0).all() and (scales[0] == 1).all() and (q[1].float() == 448).all()
    assert E.ecasq_norm(x, w, 0.0)[0].isnan().all()


def test_a_row_that_is_not_finite_changes_no_other():
    import paper_2608_18147_gb300 as E
    x = torch.randn(5, 500, device="cuda")
    bad = x.clone()
    bad[1, 3], bad[3, 9] = float("nan"), float("inf")
    w = torch.rand(500, device="cuda")
    y, z = E.ecasq_norm(x, w), E.ecasq_norm(bad, w)
    assert torch.equal(y[::2], z[::2]) and z[1].isnan().all() and z[3, 9].isnan()
    (y, s), (z, t) = E.ecasq_norm(x, w, group=32), E.ecasq_norm(bad, w, group=32)
    assert torch.equal(y[::2].float(), z[::2].float()) and torch.equal(s[::2], t[::2]) and not t[1].isfinite().any()


@pytest.mark.parametrize("dtype,k", [("f32", 700), ("bf16", 4096), ("f16", 5001), ("bf16", 70001)])
def test_in_place(dtype, k):
    import paper_2608_18147_gb300 as E
    x, r = (torch.randn(6, k, device="cuda").to(dtypes()[dtype]) for _ in range(2))
    w = torch.rand(k, device="cuda")
    y, s = E.ecasq_norm(x, w, residual=r)
    x2, r2 = x.clone(), r.clone()
    y2, s2 = E.ecasq_norm(x2, w, residual=r2, out=x2, out_sum=r2)
    assert y2 is x2 and s2 is r2 and torch.equal(y, y2) and torch.equal(s, s2)
    x2, r2 = x.clone(), r.clone()
    y2, s2 = E.ecasq_norm(x2, w, residual=r2, out=r2, out_sum=x2)
    assert y2 is r2 and s2 is x2 and torch.equal(y, y2) and torch.equal(s, s2)
    x2 = x.clone()
    assert torch.equal(E.ecasq_norm(x2, w, out=x2), E.ecasq_norm(x, w))


def test_one_row_and_no_rows():
    import paper_2608_18147_gb300 as E
    x, r, w = (torch.randn(333, device="cuda") for _ in range(3))
    y, s = E.ecasq_norm(x, w, residual=r)
    both = E.ecasq_norm(x[None], w, residual=r[None])
    assert y.shape == (333,) and torch.equal(y, both[0][0]) and torch.equal(s, both[1][0])
    q, scales = E.ecasq_norm(x, w, group=64)
    assert q.shape == (333,) and scales.shape == (6,)
    q, scales, s = E.ecasq_norm(x[None][:0], w, residual=r[None][:0], group=64)
    assert q.shape == (0, 333) and scales.shape == (0, 6) and s.shape == (0, 333)


def test_in_a_graph():
    import paper_2608_18147_gb300 as E
    x, r = torch.randn(8, 512, device="cuda").half(), torch.randn(8, 512, device="cuda").half()
    w = torch.rand(512, device="cuda")
    E.ecasq_norm(x, w, residual=r, group=128)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q, scales, s = E.ecasq_norm(x, w, residual=r, group=128)
    x.mul_(3)
    graph.replay()
    want = E.ecasq_norm(x, w, residual=r, group=128)
    assert torch.equal(q.float(), want[0].float()) and torch.equal(scales, want[1]) and torch.equal(s, want[2])


def test_refusals():
    import paper_2608_18147_gb300 as E
    x, w = torch.randn(4, 96, device="cuda"), torch.rand(96, device="cuda")
    for args, kw in (((x.double(), w), {}), ((x.T, w), {}), ((x, w[:-1]), {}), ((x, w.half()), {}), ((x, w, -1.0), {}), ((x, w), dict(residual=x[:-1])),
                     ((x, w), dict(residual=x.half())), ((x, w), dict(group=0)), ((x, w), dict(group=24)), ((x, w), dict(group=-16)),
                     ((x, w), dict(out=x.half())), ((x, w), dict(out=x, group=32)), ((x, w), dict(out_sum=x)), ((x, w), dict(out_scales=x)),
                     ((x, w), dict(out_scales=x, group=32)), ((x.cpu(), w), {}), ((x, w, float("nan")), {}), ((x[:, :0], w[:0]), {}), ((x, w, "a"), {})):
        with pytest.raises(E.EcasqError) as err:
            E.ecasq_norm(*args, **kw)
        assert err.value.code == -1, (args, kw)
    for name in ("x", "weight", "residual"):
        good = dict(x=x, weight=w, residual=x.clone())
        with pytest.raises(E.EcasqError, match="gradient"):
            E.ecasq_norm(**dict(good, **{name: good[name].clone().requires_grad_()}))
