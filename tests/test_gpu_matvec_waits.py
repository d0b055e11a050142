"""The products' bounded waits: a wait that runs out in one warp leaves no plausible number behind.

With ECASQ_TEST_LOST_WAIT each block goes on as if a thread's wait of the first round had run out: it asks for no more copies, waits for
those on their way, writes NaN to every row of its own and sets ECASQ_BAD_WAIT.  Nothing else is written, and the next
call is as ever."""
import time

import pytest

torch = pytest.importorskip("torch")
from test_gpu_matvec import dtypes, make  # noqa: E402

pytestmark = pytest.mark.gpu

# one round; several rounds and stages; several passes; columns shared by a cluster; more rows of x than eight
CASES = [(9, 100, 3, 32), (5000, 1000, 8, 128), (40000, 300, 1, 32), (90001, 256, 3, 128), (1300, 16500, 2, 128), (393, 15530, 2, 128),
         (40, 28672, 8, 64), (300, 500, 19, 96)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,k,b,group", CASES)
def test_a_lost_wait_gives_nan_and_says_so(n, k, b, group, dtype):
    import paper_2608_18147_gb300 as E
    from paper_2608_18147_gb300 import native
    x, idx, levels, scales = (t.cuda() for t in make(n, k, b, group, dtype, "f32", seed=n + k))
    codes = E.ecasq_pack(idx)
    right = E.ecasq_matvec(x, codes, levels, scales, group)
    assert torch.isfinite(right).all()
    room = torch.full((b, n + 5), 7.0, dtype=x.dtype, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kind = {"f32": native.F32, "f16": native.F16, "bf16": native.BF16}[dtype]

    def call(flag):
        return native.lib().ecasq_matvec(x.data_ptr(), k, kind | flag, b, codes.data_ptr(), codes.shape[1], levels.data_ptr(), 16,
                                         scales.data_ptr(), scales.shape[1], native.F32, n, k, group, room.data_ptr(), n + 5,
                                         status.data_ptr(), torch.cuda.current_stream().cuda_stream)

    assert x.dtype == dtypes()[dtype]
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
