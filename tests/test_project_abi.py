"""Host side of the operators around coded matrices (no GPU): refusals before any launch, sizes of workspaces."""
import pytest

V = 1 << 20  # stands for a device address: nothing is launched with it


def product(native):
    return dict(x=V, x_row=300, type=native.BF16, b=20, codes=V, code_row=192, levels=V, m=16, scales=V, scale_row=10, scale_type=native.F32, n=6,
                k=300, group=32)


BAD_PRODUCTS = [dict(x=None), dict(type=3), dict(type=-1), dict(b=-1), dict(b=524281), dict(codes=None), dict(codes=V + 8), dict(code_row=191),
                dict(code_row=128), dict(code_row=200), dict(levels=None), dict(m=0), dict(m=17), dict(scales=None), dict(scale_row=9), dict(scale_type=1),
                dict(scale_type=7), dict(n=0), dict(n=1 << 31), dict(k=0), dict(k=1 << 31), dict(group=0), dict(group=16), dict(group=40), dict(group=-32),
                dict(y=None), dict(x_row=299), dict(y_row=5), dict(activation=-1), dict(activation=5)]


def test_project_refusals():
    from paper_2608_18147_gb300 import native
    L = native.lib()
    good = dict(product(native), bias=V, activation=2, residual=V, residual_row=6, y=V, y_row=6, ws=V, ws_bytes=1 << 30, status=None, stream=None)
    assert L.ecasq_project(*dict(good, b=0).values()) == native.OK
    for change in BAD_PRODUCTS + [dict(residual_row=5)]:
        assert L.ecasq_project(*dict(good, **change).values()) == native.EINVAL, change


def test_gated_refusals():
    from paper_2608_18147_gb300 import native
    L = native.lib()
    good = dict(product(native), activation=2, y=V, y_row=6, ws=V, ws_bytes=1 << 30, status=None, stream=None)
    assert L.ecasq_gated(*dict(good, b=0).values()) == native.OK
    for change in BAD_PRODUCTS + [dict(n=1 << 30)]:
        assert L.ecasq_gated(*dict(good, **change).values()) == native.EINVAL, change


def test_norm_refusals():
    from paper_2608_18147_gb300 import native
    L = native.lib()
    good = dict(x=V, x_row=100, type=native.BF16, b=3, k=100, residual=V, residual_row=100, weight=V, weight_type=native.F32, eps=1e-6, group=32, y=V, y_row=100,
                sum=V, sum_row=100, scales=V, scale_row=4, stream=None)
    assert L.ecasq_norm(*dict(good, b=0).values()) == native.OK
    for change in (dict(x=None), dict(type=3), dict(b=-1), dict(b=1 << 31), dict(k=0), dict(k=1 << 31), dict(weight=None), dict(weight_type=1), dict(eps=-1e-9),
                   dict(eps=float("nan")), dict(group=-16), dict(group=24), dict(group=1), dict(y=None), dict(residual=None), dict(scales=None), dict(scale_row=3),
                   dict(x_row=99), dict(y_row=99), dict(residual_row=99), dict(sum_row=99)):
        assert L.ecasq_norm(*dict(good, **change).values()) == native.EINVAL, change


def test_workspace():
    """One made for the largest batch serves all smaller ones; one token needs none; bad sizes need none."""
    from paper_2608_18147_gb300 import native
    size = native.lib().ecasq_workspace_size_project
    for kind in (native.F32, native.F16, native.BF16):
        assert size(1, 4096, 4096, kind) == 0 and size(0, 4096, 4096, kind) == 0
        for n, k in ((1, 1), (257, 1000), (8192, 4097), (100000, 333)):
            last = 0
            for b in list(range(1, 70)) + [100, 128, 129, 255, 256, 257, 1000, 4096, 10000, 524280]:
                now = size(b, n, k, kind)
                assert now >= last and now % 256 == 0, (kind, n, k, b)
                last = now
    for bad in ((-1, 5, 5, 1), (5, 0, 5, 1), (5, 5, 0, 1), (5, 5, 5, 3), (5, 5, 5, -1), (524281, 5, 5, 1)):
        assert size(*bad) == 0


def test_binding_refuses_tensors_of_the_host():
    torch = pytest.importorskip("torch")
    from paper_2608_18147_gb300 import native
    z, f = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 64)
    for fn, args in ((native.ecasq_project, (f, z, f[0, :16], f, 32)), (native.ecasq_gated, (f, z, f[0, :16], f, 32)), (native.ecasq_norm, (f, f[0]))):
        with pytest.raises(native.EcasqError) as err:
            fn(*args)
        assert err.value.code == native.EINVAL
    with pytest.raises(native.EcasqError, match="activation"):
        native.ecasq_gated(f, z, f[0, :16], f, 32, activation="tanh")


def test_norm_refuses_one_place_for_both_outputs():
    from paper_2608_18147_gb300 import native
    L = native.lib()
    x, y, residual = V, V + 4096, V + 8192  # addresses that nothing reads: the call is refused
    good = dict(x=x, x_row=100, type=native.BF16, b=3, k=100, residual=residual, residual_row=100, weight=V, weight_type=native.F32, eps=1e-6, group=0, y=y, y_row=100,
                sum=None, sum_row=100, scales=None, scale_row=0, stream=None)
    assert L.ecasq_norm(*dict(good, b=0).values()) == native.OK
    for at in (x, y, residual):
        assert L.ecasq_norm(*dict(good, y=at, sum=at).values()) == native.EINVAL
