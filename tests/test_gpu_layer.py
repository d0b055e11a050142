"""The operators around coded matrices in a row, each reading what the one before wrote, with nothing between them: with a synchronisation after each the
same calls give the same bits.  And calls whose first data are in the caches already, so that what they bring in comes at once."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_overlap import both, matrix  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("width,n,b", [(1024, 1024, 1), (520, 1300, 3), (1024, 2048, 12), (517, 1023, 33), (1024, 700, 100), (640, 1024, 300), (264, 5000, 40)])
def test_a_feed_forward_block(width, n, b, dtype):
    """Norm, gated half, projection back into the residual stream, norm of that, projection, in place of one another."""
    import paper_2608_18147_gb300 as E
    gen = torch.Generator(device="cuda").manual_seed(n + b)
    gate_up, down, square = matrix(2 * n, width, dtype, gen), matrix(width, n, dtype, gen), matrix(width, width, dtype, gen)
    w = 1 + 0.1 * torch.randn(width, generator=gen, device="cuda")
    bias = 0.1 * torch.randn(width, generator=gen, device="cuda").to(dtype)
    first = torch.randn(b, width, generator=gen, device="cuda").to(dtype)
    x, y, z = (torch.empty_like(first) for _ in range(3))
    h = torch.empty(b, n, dtype=dtype, device="cuda")
    ws = E.workspace_project(b, 2 * n, max(n, width), dtype)

    def steps():
        x.copy_(first)
        for _ in range(4):
            yield (E.ecasq_norm(x, w, out=y),)
            yield (E.ecasq_gated(y, *gate_up, 128, out=h, ws=ws),)
            yield (E.ecasq_project(h, *down, 128, residual=x, out=x, ws=ws),)
            yield E.ecasq_norm(x, w, residual=y, out=z, out_sum=y)
            yield (E.ecasq_project(z, *square, 128, bias=bias, activation="gelu", residual=y, out=x, ws=ws), y, z, h)

    both(steps)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128, 1536])
@pytest.mark.parametrize("n,k,b", [(300, 1536, 200), (300, 1536, 100), (500, 1536, 60), (500, 1537, 20), (129, 4000, 700)])
def test_first_and_later_calls_agree(n, k, b, group, gated):
    """Fresh tensors, rows off 16-byte boundaries (a kernel in front of the product copies x), a residual: what a call gives does not depend on what is in
    the caches or on how soon its codes come."""
    import paper_2608_18147_gb300 as E
    for seed in range(6):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        codes, levels, _ = matrix(2 * n if gated else n, k, torch.float16, gen)
        scales = (torch.rand(codes.shape[0], -(-k // group), generator=gen, device="cuda") + 0.5) / k ** 0.5
        x = torch.randn(b, k + 5, generator=gen, device="cuda").half()[:, 3:k + 3]
        residual = torch.randn(b, n + 5, generator=gen, device="cuda").half()[:, 3:n + 3]
        call = lambda: E.ecasq_gated(x, codes, levels, scales, group) if gated else E.ecasq_project(x, codes, levels, scales, group, residual=residual)  # noqa: E731
        first = call()
        second, third = call(), call()
        torch.empty(200 << 20, dtype=torch.uint8, device="cuda").zero_()
        torch.cuda.synchronize()
        alone = call()
        assert torch.equal(first, alone) and torch.equal(second, alone) and torch.equal(third, alone)


def test_two_streams_at_once():
    """Products with workspaces of their own on two streams, their blocks beside one another on the card."""
    import paper_2608_18147_gb300 as E
    gen = torch.Generator(device="cuda").manual_seed(3)
    sides, jobs = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for i, (n, k, b) in enumerate(((512, 1000, 90), (700, 777, 300))):
        m = matrix(n, k, torch.bfloat16, gen)
        x = torch.randn(b, k, generator=gen, device="cuda").bfloat16()
        jobs.append((x, m, torch.empty(b, n, dtype=x.dtype, device="cuda"), E.workspace_project(b, n, k, x.dtype), E.ecasq_project(x, *m, 128)))
    torch.cuda.synchronize()
    for _ in range(20):
        for side, (x, m, out, ws, _) in zip(sides, jobs):
            with torch.cuda.stream(side):
                E.ecasq_project(x, *m, 128, out=out, ws=ws)
    torch.cuda.synchronize()
    for x, m, out, ws, want in jobs:
        assert torch.equal(out, want)
