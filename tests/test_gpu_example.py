"""The decoding example: what its calls give is what their definitions give from the same codes."""
import importlib.util
import os

import pytest

from conftest import ROOT

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def load():
    spec = importlib.util.spec_from_file_location("coded_decode", os.path.join(ROOT, "examples", "coded_decode.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def rows(cache, slots, page_size):
    """Values [n, heads, d] of a coded cache's slots, in binary64."""
    page, slot = slots // page_size, slots % page_size
    c, levels = cache.codes[page, slot].long(), cache.levels[page, slot].double()
    return torch.gather(levels, 2, torch.stack((c & 15, c >> 4), dim=-1).flatten(2))


def test_each_step_is_what_the_codes_say():
    """Products and attention from the stored codes in binary64; a bfloat16 result is off by its rounding, 2^-8, and fp32
    sums a thousand times less."""
    module = load()
    seen, layer = module.decode(width=256, heads=6, kv_heads=2, d=32, b=3, steps=21, page_size=8, seed=1)
    first, last = layer["qkv"].values().double(), layer["last"].values().double()
    slots = []
    for t, s in enumerate(seen):
        slots.append(s["slots"])
        q = (s["x"].double() @ first.T).view(3, 10, 32)[:, :6]
        assert ((s["q"].double() - q).abs() <= 2.0 ** -8 * q.abs() + 1e-4).all()
        at = torch.stack(slots, 1)  # [b, t + 1]
        k, v = (rows(layer[n], at.view(-1), 8).view(3, t + 1, 2, 32).repeat_interleave(3, dim=2) for n in ("keys", "values"))
        score = torch.einsum("bhd,bthd->bht", s["q"].double(), k) * 32 ** -0.5
        p = torch.softmax(score, dim=-1)
        mixed = torch.einsum("bht,bthd->bhd", p, v)
        room = torch.einsum("bht,bthd->bhd", p, v.abs())
        assert ((s["mixed"].double() - mixed).abs() <= 2.0 ** -8 * mixed.abs() + 2.0 ** -13 * room).all()
        assert (s["lse"].double() - torch.logsumexp(score, dim=-1)).abs().max() < 1e-4
        out = s["mixed"].double().reshape(3, -1) @ last.T
        size = s["mixed"].double().reshape(3, -1).abs() @ last.abs().T
        assert ((s["out"].double() - out).abs() <= 2.0 ** -8 * out.abs() + 2.0 ** -16 * size).all()
