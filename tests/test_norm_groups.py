"""Any scale group from a row's length on is one scale a row, up to the largest number (no GPU: refusals; on one: equal results)."""
import pytest

MOST = 2 ** 63 - 1


@pytest.mark.parametrize("group", [100, 2 ** 31, 2 ** 32, MOST - 100, MOST - 1, MOST])
def test_a_row_of_scales_too_short_is_refused(group):
    from paper_2608_18147_gb300 import native
    at = 1 << 20  # stands for a device address: the call is refused before anything is read
    for scale_row in (0, -1):
        assert native.lib().ecasq_norm(at, 100, native.BF16, 3, 100, None, 0, at, native.F32, 1e-6, group, at, 100, None, 0, at, scale_row, None) == native.EINVAL


@pytest.mark.gpu
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("b,k", [(1, 17), (3, 100), (400, 520), (2, 4097), (3, 70001)])  # rows in registers, aligned or not; rows read twice
def test_the_largest_group_is_one_scale_a_row(b, k, residual):
    torch = pytest.importorskip("torch")
    import paper_2608_18147_gb300 as E
    gen = torch.Generator(device="cuda").manual_seed(k)
    x, r = (torch.randn(b, k, generator=gen, device="cuda").bfloat16() for _ in range(2))
    w = torch.rand(k, generator=gen, device="cuda")
    want = E.ecasq_norm(x, w, residual=r if residual else None, group=k)
    assert want[1].shape == (b, 1)
    for group in (k + 1, 2 ** 31, 2 ** 40 + 5, MOST - 1, MOST):
        scales = torch.full((b, 1), -1.0, device="cuda")
        got = E.ecasq_norm(x, w, residual=r if residual else None, group=group, out_scales=scales)
        assert all(torch.equal(a.float(), c.float()) for a, c in zip(want, got)) and got[1] is scales
        made = E.ecasq_norm(x, w, residual=r if residual else None, group=group)
        assert all(torch.equal(a.float(), c.float()) for a, c in zip(want, made))
