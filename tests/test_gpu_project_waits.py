"""The bounded waits of products with an epilogue: a wait that runs out leaves no plausible number behind.

With ECASQ_TEST_LOST_WAIT each block goes on as if a wait of its first had run out: it brings nothing in, all of its results are NaN, ECASQ_BAD_WAIT
is set.  Nothing else is written, and the next call is as ever."""
import time

import pytest

torch = pytest.importorskip("torch")
from test_gpu_project import dtypes, matrix  # noqa: E402

pytestmark = pytest.mark.gpu

# the matrix-vector kernels; single blocks; columns shared by a cluster; several tiles a block; pairs of blocks
CASES = [(9, 100, 3, 32), (5000, 1000, 8, 128), (300, 500, 9, 96), (200, 9000, 20, 128), (700, 3000, 60, 64), (40000, 300, 30, 32), (130, 5000, 100, 128),
         (40000, 260, 100, 128), (1000, 700, 300, 128), (9000, 520, 1500, 64)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,k,b,group", CASES)
def test_a_lost_wait_gives_nan_and_says_so(n, k, b, group, dtype, gated):
    import paper_2608_18147_gb300 as E
    from paper_2608_18147_gb300 import native
    g = torch.Generator().manual_seed(n + k)
    rows = 2 * n if gated else n
    idx, levels, scales = (t.cuda() for t in matrix(g, rows, k, group, dtype, "f32"))
    x = torch.randn(b, k, generator=g).to(dtypes()[dtype]).cuda()
    codes = E.ecasq_pack(idx)
    right = E.ecasq_gated(x, codes, levels, scales, group) if gated else E.ecasq_project(x, codes, levels, scales, group, activation="silu")
    assert torch.isfinite(right).all()
    room = torch.full((b, n + 5), 7.0, dtype=x.dtype, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kind = {"f32": native.F32, "f16": native.F16, "bf16": native.BF16}[dtype]
    ws = E.workspace_project(b, rows, k, x.dtype)

    def call(flag):
        L = native.lib()
        matrix_args = (x.data_ptr(), k, kind | flag, b, codes.data_ptr(), codes.shape[1], levels.data_ptr(), 16, scales.data_ptr(), scales.shape[1], native.F32, n,
                       k, group)
        rest = (room.data_ptr(), n + 5, ws.data_ptr(), ws.numel(), status.data_ptr(), torch.cuda.current_stream().cuda_stream)
        return L.ecasq_gated(*matrix_args, 2, *rest) if gated else L.ecasq_project(*matrix_args, None, 2, None, 0, *rest)

    torch.cuda.synchronize()
    t0 = time.perf_counter()
    assert call(native.TEST_LOST_WAIT) == native.OK
    torch.cuda.synchronize()
    assert time.perf_counter() - t0 < 5.0
    assert status.item() == E.BAD_WAIT
    assert torch.isnan(room[:, :n]).all() and (room[:, n:] == 7).all()
    status.zero_()
    assert call(0) == native.OK
    assert status.item() == 0 and torch.equal(room[:, :n], right) and (room[:, n:] == 7).all()
