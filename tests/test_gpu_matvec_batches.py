"""Products with more than eight rows of x where every warp has columns, rounds and passes are several and the last eight are cut."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_matvec import check, make, reference  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,k,b,group", [(6000, 2050, 9, 32), (3001, 8192, 33, 128), (700, 20001, 17, 96), (90001, 256, 12, 64), (5, 40, 1000, 32)])
def test_batches(n, k, b, group, dtype):
    import paper_2608_18147_gb300 as E
    x, idx, levels, scales = make(n, k, b, group, dtype, "f32", seed=n + b)
    y = E.ecasq_matvec(x.cuda(), E.ecasq_pack(idx.cuda()), levels.cuda(), scales.cuda(), group)
    assert y.shape == (b, n)
    some = torch.cat([torch.arange(0, n, max(1, n // 300)), torch.arange(max(0, n - 40), n)])
    ref, size = reference(x, idx[some], levels, scales[some], group)
    check(y[:, some.cuda()], ref, size, k, dtype)
