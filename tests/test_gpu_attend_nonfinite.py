"""Values that are not finite among those seen reach the entries that they enter and, in 16-bit attention, at most the neighbours in their
pairs (2i, 2i + 1): other entries, key heads and sequences keep their bits."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_attend import KINDS, call, make  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,levels", KINDS)
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("g,d,entry", [(1, 64, 0), (4, 128, 77), (8, 96, 95), (6, 256, 130)])
def test_a_value_that_is_not_finite(g, d, entry, bad, dtype, levels):
    c = make([90, 300], 2, g, d, 16, dtype, levels, seed=g + d)
    key, head = 37, 1
    page, slot = int(c["table"][1, key // 16]), key % 16
    if levels == 0:
        before = call(c)
        c["v"].rows[page, slot, head, entry] = bad
    else:  # a level that this entry alone has
        codes = c["v"].rows[page, slot, head]
        nibbles = torch.stack((codes & 15, codes >> 4), -1).view(-1).clamp_(max=levels - 2)
        nibbles[entry] = levels - 1
        codes.copy_(nibbles[0::2] | (nibbles[1::2] << 4))
        before = call(c)
        c["v"].levels[page, slot, head, levels - 1] = bad
    after = call(c)
    assert torch.equal(before[1], after[1])  # lse does not know the values
    assert not torch.isfinite(after[0][1, head * g:(head + 1) * g, entry]).any()
    touched = torch.zeros_like(after[0], dtype=torch.bool)
    first = entry if dtype == "f32" else entry // 2 * 2
    touched[1, head * g:(head + 1) * g, first:entry + 1 if dtype == "f32" else first + 2] = True
    assert torch.equal(before[0][~touched], after[0][~touched])


@pytest.mark.parametrize("dtype,levels", KINDS)
def test_a_key_that_is_not_a_number(dtype, levels):
    c = make([90, 300], 2, 4, 64, 16, dtype, levels, seed=3)
    before = call(c)
    page, slot = int(c["table"][1, 2]), 5
    (c["k"].rows if levels == 0 else c["k"].levels)[page, slot, 1] = float("nan")
    out, lse = call(c)
    assert torch.isnan(out[1, 4:]).all() and torch.isnan(lse[1, 4:]).all()
    for x, y in zip(before, (out, lse)):
        assert torch.equal(x[0], y[0]) and torch.equal(x[1, :4], y[1, :4])
