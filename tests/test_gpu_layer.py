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


def test_captured_before_any_other_call():
    """A process whose first calls are captured into a graph: what the library asks the card once is asked then."""
    import os
    import subprocess
    import sys
    src = """
import torch
import paper_2608_18147_gb300 as E
gen = torch.Generator(device="cuda").manual_seed(1)
idx = torch.randint(0, 16, (512, 640), generator=gen, device="cuda", dtype=torch.uint8)
codes, levels, scales = E.ecasq_pack(idx), torch.linspace(-1, 1, 16, device="cuda").half(), torch.rand(512, 5, generator=gen, device="cuda")
few, many, most = (torch.randn(b, 640, generator=gen, device="cuda").half() for b in (3, 100, 700))
w = torch.rand(640, device="cuda")
side = torch.cuda.Stream()
side.wait_stream(torch.cuda.current_stream())
graph = torch.cuda.CUDAGraph()
with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
    got = [f(x, codes, levels, scales, 128) for x in (few, many, most) for f in (E.ecasq_project, E.ecasq_gated)] + [E.ecasq_norm(many, w)]
graph.replay()
torch.cuda.synchronize()
want = [f(x, codes, levels, scales, 128) for x in (few, many, most) for f in (E.ecasq_project, E.ecasq_gated)] + [E.ecasq_norm(many, w)]
assert all(torch.equal(a, b) and a.float().abs().sum() > 0 for a, b in zip(got, want))
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", src], cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]


@pytest.mark.parametrize("b", [1, 9, 40, 130, 600])
def test_levels_scales_and_rows_of_a_larger_tensor(b):
    """Levels that begin off 4-byte boundaries, 16-bit scales in a wider tensor at odd places, codes with longer rows."""
    import paper_2608_18147_gb300 as E
    gen = torch.Generator(device="cuda").manual_seed(b)
    n, k, group = 270, 900, 32
    idx = torch.randint(0, 16, (n, k), generator=gen, device="cuda", dtype=torch.uint8)
    packed = E.ecasq_pack(idx)
    codes = torch.full((n, packed.shape[1] + 48), 255, dtype=torch.uint8, device="cuda")
    codes[:, :packed.shape[1]] = packed
    levels = torch.cat([torch.zeros(1, device="cuda"), torch.linspace(-1, 1, 16, device="cuda")]).bfloat16()[1:]
    for lead in (1, 2, 3):
        scales = torch.full((n, 29 + lead + 2), float("nan"), dtype=torch.bfloat16, device="cuda")[:, lead:lead + 29]
        scales.copy_(torch.rand(n, 29, generator=gen, device="cuda") / 30)
        x = torch.randn(b, k, generator=gen, device="cuda").bfloat16()
        want = E.ecasq_project(x, packed, levels.clone(), scales.contiguous(), group)
        assert torch.equal(E.ecasq_project(x, codes[:, :packed.shape[1]], levels, scales, group), want) and want.isfinite().all()
        half = E.ecasq_gated(x, packed, levels.clone(), scales.contiguous(), group)
        assert torch.equal(E.ecasq_gated(x, codes[:, :packed.shape[1]], levels, scales, group), half)


@pytest.mark.parametrize("b", [2, 400])
@pytest.mark.parametrize("dtype,weight,k", [(torch.bfloat16, torch.float32, k) for k in (12176, 12192, 12200, 12224, 12248, 12256, 12264)] +
                         [(torch.float32, torch.float32, k) for k in (12192, 12208, 12240, 12268, 12272, 12276)] +
                         [(torch.float16, torch.float16, k) for k in (24448, 24512, 24544, 24552)])
def test_norm_where_weights_nearly_fill_the_ordinary_shared_memory(b, dtype, weight, k):
    """Weights of 48 KB less a few words: what the kernel has beside them is counted too.  Roundings: fp32 sums of k squares in any order k 2^-24
    at most (their root half of that), four more of a product, the output's half step."""
    import paper_2608_18147_gb300 as E
    gen = torch.Generator(device="cuda").manual_seed(k)
    x = torch.randn(b, k, generator=gen, device="cuda").to(dtype)
    w = torch.rand(k, generator=gen, device="cuda").to(weight)
    got = E.ecasq_norm(x, w, 1e-6)
    want = x.double() / (x.double().square().mean(1, keepdim=True) + 1e-6).sqrt() * w.double()
    assert ((got.double() - want).abs() <= want.abs() * (torch.finfo(dtype).eps / 2 + (k / 2 + 4) * 2.0**-24) + 1e-7).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_workspaces_that_do_not_do(dtype):
    """Too small, or not on a 16-byte boundary: refused where one is needed; one of the right size gives what a call without one does."""
    import paper_2608_18147_gb300 as E
    gen = torch.Generator(device="cuda").manual_seed(5)
    b, n, k = 600, 2048, 1001  # rows of 1001 values do not begin on 16-byte boundaries
    codes = E.ecasq_pack(torch.randint(0, 16, (n, k), generator=gen, device="cuda", dtype=torch.uint8))
    levels, scales = torch.linspace(-1, 1, 16, device="cuda").to(dtype), torch.rand(n, 8, generator=gen, device="cuda")
    x = torch.randn(b, k, generator=gen, device="cuda").to(dtype)
    room = E.workspace_project(b, n, k, dtype)
    room = room.numel() * room.element_size()
    want = E.ecasq_project(x, codes, levels, scales, 128)
    whole = torch.empty(room + 16, dtype=torch.uint8, device="cuda")
    for ws in (whole[:room - 256], whole[:0], whole[1:room + 1], whole[8:room + 8], whole[:room].cpu()):
        with pytest.raises((ValueError, RuntimeError, TypeError)):
            E.ecasq_project(x, codes, levels, scales, 128, ws=ws)
        with pytest.raises((ValueError, RuntimeError, TypeError)):
            E.ecasq_gated(x, codes, levels, scales, 128, ws=ws)
    whole.fill_(255)
    assert torch.equal(E.ecasq_project(x, codes, levels, scales, 128, ws=whole[:room]), want)
    assert torch.equal(E.ecasq_project(x, codes, levels, scales, 128, ws=whole[16:]), want)


def right_or_refused(call, want):
    """The same bits as `want`, or an error of the framework's own."""
    import paper_2608_18147_gb300 as E
    try:
        got = call()
    except E.EcasqError:
        return False
    assert torch.equal(got, want)
    return True


@pytest.mark.parametrize("b", [3, 40, 600])
def test_strided_and_expanded_arguments(b):
    """Every second entry of a vector, columns for rows, one row for all: never read as if they lay side by side."""
    import paper_2608_18147_gb300 as E
    gen = torch.Generator(device="cuda").manual_seed(b)
    n, k = 256, 384
    codes = E.ecasq_pack(torch.randint(0, 16, (n, k), generator=gen, device="cuda", dtype=torch.uint8))
    levels, scales = torch.linspace(-1, 1, 16, device="cuda").half(), torch.rand(n, 3, generator=gen, device="cuda")
    x, bias, residual = (torch.randn(*s, generator=gen, device="cuda").half() for s in ((b, k), (n,), (b, n)))
    second = lambda v: v.repeat_interleave(2)[::2]  # noqa: E731
    project = lambda *a, **o: E.ecasq_project(*a, 128, **o)  # noqa: E731
    want = project(x, codes, levels, scales, bias=bias, residual=residual)
    right_or_refused(lambda: project(x, codes, levels, scales, bias=second(bias), residual=residual), want)
    right_or_refused(lambda: project(x, codes, second(levels), scales, bias=bias, residual=residual), want)
    right_or_refused(lambda: project(x, codes, levels, scales.T.contiguous().T, bias=bias, residual=residual), want)
    right_or_refused(lambda: project(x.T.contiguous().T, codes, levels, scales, bias=bias, residual=residual), want)
    right_or_refused(lambda: project(x, codes, levels, scales, bias=bias, residual=residual.T.contiguous().T), want)
    same = x[:1].expand(b, k)
    right_or_refused(lambda: project(same, codes, levels, scales), project(same.contiguous(), codes, levels, scales))
    right_or_refused(lambda: project(x, codes, levels, scales, residual=residual[:1].expand(b, n)),
                     project(x, codes, levels, scales, residual=residual[:1].expand(b, n).contiguous()))
    right_or_refused(lambda: project(x, codes, levels, scales[:1].expand(n, 3)), project(x, codes, levels, scales[:1].expand(n, 3).contiguous()))
    right_or_refused(lambda: project(x, codes, levels, scales, bias=bias[:1].expand(n)), project(x, codes, levels, scales, bias=bias[:1].expand(n).contiguous()))
    with pytest.raises(E.EcasqError):
        project(x, codes, levels, scales, out=torch.empty(1, n, dtype=x.dtype, device="cuda").expand(b, n))
    w = torch.rand(k, generator=gen, device="cuda").half()
    want = E.ecasq_norm(x, w)
    right_or_refused(lambda: E.ecasq_norm(x, second(w)), want)
    right_or_refused(lambda: E.ecasq_norm(x.T.contiguous().T, w), want)
    right_or_refused(lambda: E.ecasq_norm(same, w), E.ecasq_norm(same.contiguous(), w))
    right_or_refused(lambda: E.ecasq_norm(x, w, residual=same)[0], E.ecasq_norm(x, w, residual=same.contiguous())[0])
    right_or_refused(lambda: E.ecasq_norm(x, w[:1].expand(k)), E.ecasq_norm(x, w[:1].expand(k).contiguous()))
    with pytest.raises(E.EcasqError):
        E.ecasq_norm(x, w, out=torch.empty(1, k, dtype=x.dtype, device="cuda").expand(b, k))
    with pytest.raises(E.EcasqError):
        E.ecasq_norm(x, w, group=128, out_scales=torch.empty(1, 3, device="cuda").expand(b, 3))


def test_threads_that_call_at_once():
    """Four threads with streams of their own, each with calls of every kernel: the results of calls in a row."""
    import threading
    import paper_2608_18147_gb300 as E
    gen = torch.Generator(device="cuda").manual_seed(11)
    n, k = 512, 640
    codes = E.ecasq_pack(torch.randint(0, 16, (n, k), generator=gen, device="cuda", dtype=torch.uint8))
    levels, scales = torch.linspace(-1, 1, 16, device="cuda").bfloat16(), torch.rand(n, 5, generator=gen, device="cuda")
    w = torch.rand(k, device="cuda")
    xs = [torch.randn(b, k, generator=gen, device="cuda").bfloat16() for b in (2, 50, 300, 700)]
    run = lambda x: (E.ecasq_project(x, codes, levels, scales, 128, activation="gelu"), E.ecasq_gated(x, codes, levels, scales, 128), E.ecasq_norm(x, w))  # noqa: E731
    want = [run(x) for x in xs]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for turn in range(20):
                    j = (i + turn) % len(xs)
                    got = run(xs[j])
                    stream.synchronize()
                    if not all(torch.equal(a, c) for a, c in zip(got, want[j])):
                        wrong.append((i, turn))
        except Exception as e:  # noqa: BLE001
            wrong.append(repr(e))
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_norm_refuses_one_tensor_for_both_outputs():
    import paper_2608_18147_gb300 as E
    x, r, w = torch.ones(3, 64, device="cuda"), torch.ones(3, 64, device="cuda"), torch.ones(64, device="cuda")
    for t in (x, r, torch.empty_like(x)):
        with pytest.raises(E.EcasqError):
            E.ecasq_norm(x, w, residual=r, out=t, out_sum=t)
    y, s = E.ecasq_norm(x, w, 0.0, residual=r, out=x, out_sum=r)
    assert (y == 1).all() and (s == 2).all()
