"""Products do not overwrite the rows that they read: a result at x's address is refused (no GPU: before anything is launched; on one: through the binding)."""
import pytest

from test_project_abi import BAD_PRODUCTS, V, product


@pytest.mark.parametrize("b", [1, 3, 20])
def test_the_entry_points_refuse_a_result_at_the_address_of_x(b):
    from paper_2608_18147_gb300 import native
    L, at = native.lib(), 1 << 20  # stands for a device address: nothing is launched with it
    matrix = lambda n: (200, native.BF16, b, at, 128, at, 16, at, 2, native.F32, n, 200, 128)  # noqa: E731
    assert L.ecasq_project(at, *matrix(200), None, 0, None, 0, at, 200, None, 0, None, None) == native.EINVAL
    assert L.ecasq_gated(at, *matrix(100), 2, at, 100, None, 0, None, None) == native.EINVAL


def test_refusals_with_the_result_elsewhere():
    """What test_project_abi.py has refused, with a y that is not x, so that each is refused for itself."""
    from paper_2608_18147_gb300 import native
    L = native.lib()
    y, more = V + (1 << 16), dict(ws=V, ws_bytes=1 << 30, status=None, stream=None)
    project = dict(product(native), bias=V, activation=2, residual=V, residual_row=6, y=y, y_row=6, **more)
    gated = dict(product(native), activation=2, y=y, y_row=6, **more)
    for change in BAD_PRODUCTS:
        assert L.ecasq_project(*dict(project, **change).values()) == native.EINVAL, change
        assert L.ecasq_gated(*dict(gated, **change).values()) == native.EINVAL, change
    assert L.ecasq_project(*dict(project, residual_row=5).values()) == native.EINVAL
    assert L.ecasq_gated(*dict(gated, n=1 << 30).values()) == native.EINVAL


@pytest.mark.gpu
@pytest.mark.parametrize("b", [1, 20, 300])
def test_the_binding_refuses_x_as_the_result(b):
    torch = pytest.importorskip("torch")
    import paper_2608_18147_gb300 as E
    n = 256
    codes = E.ecasq_pack(torch.randint(0, 16, (2 * n, n), device="cuda", dtype=torch.uint8))
    levels, scales = torch.linspace(-1, 1, 16, device="cuda").half(), torch.rand(2 * n, 2, device="cuda")
    x = torch.randn(b, n, device="cuda").half()
    kept = x.clone()
    with pytest.raises(E.EcasqError) as err:
        E.ecasq_project(x, codes[:n], levels, scales[:n], 128, out=x)
    assert err.value.code == -1
    with pytest.raises(E.EcasqError) as err:
        E.ecasq_gated(x, codes, levels, scales, 128, out=x)
    assert err.value.code == -1 and torch.equal(x, kept)
    wide = torch.cat([x, x], dim=1)  # side by side with x they are two places
    assert torch.equal(E.ecasq_project(wide[:, :n], codes[:n], levels, scales[:n], 128, out=wide[:, n:]), E.ecasq_project(x, codes[:n], levels, scales[:n], 128))
