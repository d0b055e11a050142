"""gelu's Phi in fp32: its own error and that of its tail, through an identity matrix of codes.

Every product is a value of x itself (1 times x and zeros; x's terms add up exactly), so y is the operator's v Phi(v) rounded once.  Bounds: Phi to 2^-23, and for v >= -12 to
(2^-21 + v^2 2^-23) of itself, as include/ecasq.h states; the product's rounding adds 2^-24 of y, and what is below fp32's normal numbers is off by 2^-126."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def identity():
    import paper_2608_18147_gb300 as E
    idx = torch.eye(128, device="cuda").to(torch.uint8)
    return E.ecasq_pack(idx), torch.tensor([0.0, 1.0], device="cuda"), torch.ones(128, 1, device="cuda"), 128


@pytest.mark.parametrize("rows", [8, 4000])  # the kernels for few rows, and the tensor cores
def test_gelu_and_its_tail(rows):
    import paper_2608_18147_gb300 as E
    v = torch.linspace(-12, 12, rows * 128, device="cuda")
    v = v[torch.randperm(v.numel(), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")].view(rows, 128)
    assert torch.equal(E.ecasq_project(v, *identity()), v)
    y = E.ecasq_project(v, *identity(), activation="gelu").double()
    x = v.double()
    phi = torch.special.erfc(-x / 2 ** 0.5) / 2  # (ndtr's 1 + erf has no tail below 2^-53)
    off, size = (y - x * phi).abs(), x.abs() * phi
    assert (off <= x.abs() * 2.0 ** -23 + size * 2.0 ** -24).all(), (off - x.abs() * 2.0 ** -23).max().item()
    of_itself = 2.0 ** -21 + x * x * 2.0 ** -23
    worst = (off / (size * (of_itself + 2.0 ** -24) + 2.0 ** -126))
    assert (worst <= 1).all(), (worst.max().item(), v.flatten()[worst.argmax()].item())


@pytest.mark.parametrize("rows", [1, 4000])
def test_gelu_far_out(rows):
    """Beyond the tail gelu is 0 or v itself; zeros and NaN stay what they are."""
    import paper_2608_18147_gb300 as E
    far = torch.tensor([14.0, 15.0, 40.0, 1e4, 1e10, 1e19, 3e38], device="cuda")
    x = torch.zeros(rows, 128, device="cuda")
    x[:, :7], x[:, 7:14] = far, -far
    y = E.ecasq_project(x, *identity(), activation="gelu")
    assert torch.equal(y[:, :7], x[:, :7]) and (y[:, 7:].abs() < 1e-40).all()
    x[:, 20] = float("nan")
    assert E.ecasq_project(x, *identity(), activation="gelu").isnan().all()
