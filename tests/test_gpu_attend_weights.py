"""Attention where one key takes nearly all of the weight and holds zeros: what the light keys give is the whole result.

Tolerance: that of test_gpu_attend.py, whose term 2^-15 sum p |v| covers weights of 16 bits, and for fp16 the step of its weights.
They enter the values' product as two binary16 parts of 2^15 times a weight (at most 1), so the second part is off by
its half step 2^-25 at most: 2^-40 of the heaviest weight for each key, 2^-40 sum |v| in all.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_gpu_attend import call, check, dt, make, reference  # noqa: E402

pytestmark = pytest.mark.gpu


def sink(n, at, gap, g, d, dtype, levels, seed):
    """One sequence of n keys: key `at` is about `gap` ahead of the others in score (scale 1) and its value is 0; the others'
    values are in the thousands."""
    c = make([n], 1, g, d, 16, dtype, levels, seed=seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    c["q"].copy_((1 + 0.1 * torch.randn(1, g, d, generator=gen, device="cuda")).to(dt(dtype)))
    page, slot = int(c["table"][0, at // 16]), at % 16
    for name, shrink, own in (("k", 0.02, gap / d), ("v", 1000.0, 0.0)):
        side = c[name]
        held = side.rows if levels == 0 else side.levels
        held.copy_((held.float() * shrink).to(dt(dtype)))
        held[page, slot] = own
    return c


@pytest.mark.parametrize("dtype,levels", [("f16", 0), ("f16", 8), ("f16", 16), ("bf16", 0), ("bf16", 8), ("f32", 0)])
@pytest.mark.parametrize("gap", [3, 8, 11, 14, 15.2, 16.3, 18, 22])
@pytest.mark.parametrize("n,at,g,d", [(16, 3, 2, 64), (16, 15, 8, 128), (300, 0, 4, 96), (40, 20, 5, 256)])
def test_a_sink_with_zero_values(n, at, g, d, gap, dtype, levels):
    c = sink(n, at, gap, g, d, dtype, levels, seed=n + g)
    out, tol, lse, ltol = reference(c, scale=1.0)
    values = c["v"].values(*(lambda t: (c["table"].long()[0][t // 16], t % 16))(torch.arange(n, device="cuda")), 0)
    if dtype == "f16":
        tol = tol + 2.0 ** -40 * np.abs(values).sum(0)
    assert (np.abs(out).max() > 100 * tol.max()) or gap > 18  # the light keys count
    check(call(c, scale=1.0), (out, tol, lse, ltol))
