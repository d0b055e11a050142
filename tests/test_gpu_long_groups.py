"""Products in long scale groups on the tensor cores: sums are not cut off more than those of short ones.

Values of one sign, so that whatever is lost at each step adds up, and a residual of minus the result rounded to fp16, so that what is left shows the sums' own error.  The
tensor core's sum of 16 products a step may lose a unit in the last place of the sum at each of a span's steps, and no more than 16 steps (256 columns) are summed there: the mean error is within 16 steps 2^-23 of
the sum.  The fp32 additions of the spans, scaled, round to nearest and add no mean error; each is within 2^-24 of the sum, k / 256 of them.  The output, which is at most half a step of fp16 (2^-11 of the sum) and the sums'
error, is rounded by 2^-11 of itself.  Nothing in the mean's bound grows with k."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SIZES = [(600, 4096, 40), (520, 16384, 40), (520, 16384, 100), (1100, 16384, 600), (300, 28672, 24)]


def matrix(n, k, group, gen):
    import paper_2608_18147_gb300 as E
    idx = torch.randint(0, 16, (n, k), generator=gen, device="cuda", dtype=torch.uint8)
    levels = (torch.rand(16, generator=gen, device="cuda") + 0.2).half()
    scales = (torch.rand(n, -(-k // group), generator=gen, device="cuda") + 0.5) / k
    w = levels.double()[idx.long()] * scales.double().repeat_interleave(group, dim=1)[:, :k]
    return (E.ecasq_pack(idx), levels, scales, group), w


@pytest.mark.parametrize("n,k,b", SIZES)
@pytest.mark.parametrize("of", ["384", "640", "1024", "1920", "row", "beyond"])
def test_sums_of_one_sign(n, k, b, of):
    import paper_2608_18147_gb300 as E
    group = {"row": k, "beyond": 1 << 20}.get(of) or int(of)
    gen = torch.Generator(device="cuda").manual_seed(k + b)
    args, w = matrix(n, k, group, gen)
    x = (torch.rand(b, k, generator=gen, device="cuda") + 0.1).half()
    p = x.double() @ w.T
    residual = -p.half()
    rest = p + residual.double()
    error = (E.ecasq_project(x, *args, residual=residual).double() - rest) / p
    assert error.mean().abs() <= 16 * 2.0 ** -23, error.mean().item()
    most = 32 * 2.0 ** -23 + k / 256 * 2.0 ** -24
    assert (error.abs() <= most + 2.0 ** -11 * (2.0 ** -11 + most) + 2.0 ** -25 / p).all(), error.abs().max().item()


@pytest.mark.parametrize("n,k,b,group", [(300, 5000, 40, 640), (260, 3000, 700, 384), (150, 9000, 100, 9088), (2000, 2900, 130, 1152)])
def test_groups_that_end_inside_a_span(n, k, b, group):
    """Gated and not, groups of an odd number of blocks, columns shared by a cluster: against 64 bits.  fp32 sums of k terms of both signs, 16 a step: within (k / 8 + 16) 2^-23 of
    the sum of their sizes; a product of two such: each error times the other factor; the result is rounded by 2^-11 of itself."""
    import paper_2608_18147_gb300 as E
    gen = torch.Generator(device="cuda").manual_seed(k)
    args, w = matrix(2 * n, k, group, gen)
    x = torch.randn(b, k, generator=gen, device="cuda").half()
    p, size = x.double() @ w.T, (k / 8 + 16) * 2.0 ** -23 * (x.double().abs() @ w.T)
    y = E.ecasq_project(x, *args).double()
    assert ((y - p).abs() <= size + 2.0 ** -11 * (p.abs() + size) + 2.0 ** -25).all()
    h = E.ecasq_gated(x, *args, activation=None).double()
    (g, u), (dg, du) = p.chunk(2, dim=1), size.chunk(2, dim=1)
    off = dg * u.abs() + du * g.abs() + dg * du + 2.0 ** -23 * (g * u).abs()
    assert ((h - g * u).abs() <= off + 2.0 ** -11 * ((g * u).abs() + off) + 2.0 ** -25).all()
