"""The block example: what its calls give is what their definitions give from the same codes."""
import importlib.util
import os

import pytest

from conftest import ROOT

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def load():
    spec = importlib.util.spec_from_file_location("coded_block", os.path.join(ROOT, "examples", "coded_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def near(got, want, size):
    """A bfloat16 result is off by its rounding, 2^-8 of itself; sums of fp32 by some 2^-16 of what they add up."""
    assert ((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -16 * size + 1e-6).all()


def normed(s, weight):
    s = s.double()
    return s / (s.square().mean(1, keepdim=True) + 1e-6).sqrt() * weight.double()


def test_each_step_is_what_the_codes_say():
    module = load()
    seen, block = module.decode(width=256, heads=4, kv_heads=2, d=64, hidden=320, b=3, steps=10, page_size=8, seed=1)
    w = {name: m.values().double() for name, m in block.coded.items()}
    for s in seen:
        near(s["first"], normed(s["x"], block.norms[0]), 0)
        near(s["made"].reshape(3, -1), s["first"].double() @ w["qkv"].T + block.bias.double(), s["first"].double().abs() @ w["qkv"].abs().T)
        mixed = s["mixed"].double().reshape(3, -1)
        near(s["out"], mixed @ w["back"].T, mixed.abs() @ w["back"].abs().T)
        assert torch.equal(s["s"], (s["out"].float() + s["x"].float()).bfloat16())
        check_feed_forward(block, w, s["s"], s["y"], s["h"], s["end"])


def check_feed_forward(block, w, s, y, h, end):
    near(y, normed(s, block.norms[1]), 0)
    gate, up = (y.double() @ w["gate_up"].T).chunk(2, dim=1)
    gate_size, up_size = (y.double().abs() @ w["gate_up"].abs().T).chunk(2, dim=1)
    near(h, gate * torch.sigmoid(gate) * up, 2 * (gate_size * up.abs() + up_size * gate.abs()))
    near(end, h.double() @ w["down"].T + s.double(), h.double().abs() @ w["down"].abs().T + s.double().abs())


@pytest.mark.parametrize("rows", [1, 7, 40, 100, 400])
def test_a_prompt_through_the_feed_forward_part(rows):
    module = load()
    block = module.Block(256, 4, 2, 64, 320, 5)
    w = {name: m.values().double() for name, m in block.coded.items()}
    x = torch.randn(rows, 256, generator=torch.Generator(device="cuda").manual_seed(rows), device="cuda").bfloat16()
    end, seen = block.feed_forward(x)
    check_feed_forward(block, w, x, seen["y"], seen["h"], end)


def test_it_prints(capsys):
    load().main()
    assert "steps decoded" in capsys.readouterr().out
