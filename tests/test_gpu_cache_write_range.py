"""Encode of cache rows (ecasq_cache_write) whose codebooks leave the range of the cache's type: the largest finite value stands
for what lies beyond it, the rounding goes by that level, and the status word says so."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_cache_write import cache, expect, reference  # noqa: E402

pytestmark = pytest.mark.gpu

LARGEST = {"f16": 65504.0, "bf16": torch.finfo(torch.bfloat16).max}


def write(x, Q, m, levels, dtype, seed):
    import paper_2608_18147_gb300 as E
    n, heads, d = x.shape
    codes, table = cache(1, n, heads, d, levels, dtype)
    before = codes.cpu().clone(), table.cpu().clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    E.ecasq_cache_write(x.cuda(), Q.cuda(), m.cuda(), torch.arange(n, device="cuda"), codes, table, seed, status=status)
    return codes.cpu(), table.cpu(), status.item(), before


@pytest.mark.parametrize("dtype,big", [("f16", 70000.0), ("f16", 3e38), ("bf16", 3.4e38)])
@pytest.mark.parametrize("levels,d", [(8, 64), (16, 128), (8, 256)])
@pytest.mark.parametrize("low,high", [(True, False), (False, True), (True, True)])
def test_levels_beyond_the_type(low, high, levels, d, dtype, big):
    import paper_2608_18147_gb300 as E
    gen = torch.Generator().manual_seed(d + levels)
    n, heads = 3, 2
    x = torch.randn(n, heads, d, generator=gen)
    if dtype == "f16":
        x *= 8000
    Q = torch.sort(x.view(n * heads, d)[:, :levels].contiguous(), dim=1).values
    m = torch.full((n * heads,), levels, dtype=torch.int32)
    m[2] = levels - 3
    for row in (0, 2, 5):  # the other rows are in range
        if low:
            x.view(n * heads, d)[row, 1] = Q[row, 0] = -big
        if high:
            x.view(n * heads, d)[row, 2] = Q[row, int(m[row]) - 1] = big
    codes, table, status, before = write(x, Q, m, levels, dtype, 17)
    assert status == E.BAD_VALUE
    assert torch.isfinite(table).all()
    held = Q.clamp(-LARGEST[dtype], LARGEST[dtype])
    want, book = reference(x.view(n * heads, d).numpy(), held, m, levels, dtype, 17)
    full = expect(*before, want, book, torch.arange(n), n, heads)
    assert torch.equal(table, full[1])
    assert torch.equal(codes, full[0])


def test_what_rounds_into_the_range_is_no_error():
    """65519.9 rounds to binary16's largest value; what a codebook holds beyond its m does not count."""
    x = torch.linspace(-65519.9, 65519.9, 64).view(1, 1, 64)
    Q = torch.tensor([[-65519.9, 0.0, 65519.9, 1e30, float("inf"), float("nan")]])
    m = torch.tensor([3], dtype=torch.int32)
    codes, table, status, before = write(x, Q, m, 8, "f16", 3)
    assert status == 0 and torch.isfinite(table).all()
    want, book = reference(x.view(1, 64).numpy(), Q, m, 8, "f16", 3)
    full = expect(*before, want, book, torch.arange(1), 1, 1)
    assert torch.equal(table, full[1]) and torch.equal(codes, full[0])


def test_levels_that_are_no_numbers_are_reported():
    import paper_2608_18147_gb300 as E
    x = torch.linspace(-1, 1, 64).view(1, 1, 64)
    for wrong in (float("nan"), float("inf"), -float("inf")):
        Q = torch.tensor([[-1.0, 0.0, 1.0]])
        Q[0, 0 if wrong < 0 else 2] = wrong
        _, table, status, _ = write(x, Q, torch.tensor([3], dtype=torch.int32), 8, "f16", 3)
        assert status == E.BAD_VALUE
        assert not torch.isinf(table).any()
