"""Rows with infinities and NaN: each output is what the sum of the products is in IEEE arithmetic, by every kernel.

An infinity times a level is an infinity of the product's sign, or NaN where the level is zero; infinities of both signs add up to NaN."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("zero", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,k,b,group", [(40, 300, 5, 32), (1000, 700, 300, 128), (9000, 520, 1500, 64), (1030, 390, 600, 32)])
def test_infinities(n, k, b, group, dtype, zero, gated):
    import paper_2608_18147_gb300 as E
    gen = torch.Generator(device="cuda").manual_seed(n + b)
    idx = torch.randint(0, 16, (n, k), generator=gen, device="cuda", dtype=torch.uint8)
    # Levels that take one bf16 term, two and three; one that is zero.
    levels = (torch.tensor([-2.0, -1.5, -1 - 2.0 ** -9, -0.7, -0.5, -1 / 3, -0.1, -0.01, 0.01, 0.1, 0.3, 0.5, 0.625, 1 + 2.0 ** -20, 1.5, 2.0], device="cuda")).to(dtype)
    if zero:
        levels[8] = 0
    scales = (torch.rand(n, -(-k // group), generator=gen, device="cuda") + 0.5) / k ** 0.5
    x = torch.randn(b, k, generator=gen, device="cuda").to(dtype)
    inf = float("inf")
    x[0, 3] = inf
    x[1, k - 1] = -inf
    x[2, 5], x[2, 40] = inf, inf
    x[3, 0], x[3, 200] = inf, -inf
    x[b - 1, 7] = float("nan")
    w = levels.double()[idx.long()] * scales.double().repeat_interleave(group, dim=1)[:, :k]
    p = torch.stack([(x[i].double() * w).sum(1) for i in (0, 1, 2, 3, b - 1)])
    rows = (0, 1, 2, 3, b - 1)
    if gated:
        y = E.ecasq_gated(x, E.ecasq_pack(idx), levels, scales, group, activation="relu")
        gate, up = p.chunk(2, dim=1)
        want = torch.where(gate <= 0, torch.zeros_like(gate), gate) * up
    else:
        y = E.ecasq_project(x, E.ecasq_pack(idx), levels, scales, group)
        want = p
    got = y[list(rows)].double()
    assert not want[:4].isfinite().all() and torch.equal(got.isnan(), want.isnan())
    infinite = want.isinf()
    assert torch.equal(got[infinite], want[infinite]) and torch.equal(got.isinf(), infinite)
    assert y[4:b - 1].isfinite().all()
