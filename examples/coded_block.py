"""One block of a language model decoding with coded weights and a coded cache.

    python examples/coded_block.py

Norm, one product for queries, keys and values with its bias, the new rows into the coded cache, attention, the product back into the
residual stream; norm, the gated half of the feed-forward part, the product back into the residual stream: ecasq_norm,
ecasq_project, ecasq_cache_write, ecasq_attend and ecasq_gated around the matrices and caches of coded_decode.py.  A prompt's rows go
through the feed-forward part at once with the same calls.  Printed is how far the block's output is from that of the same block
without any coding.
"""
import os
import sys

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2608_18147_gb300 as E  # noqa: E402
from coded_decode import GROUP, CodedCache, CodedMatrix  # noqa: E402


class Block:
    """The block's coded matrices and what is not coded, with random weights."""

    def __init__(self, width, heads, kv_heads, d, hidden, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda n, k: torch.randn(n, k, generator=gen, device="cuda") / k ** 0.5  # noqa: E731
        self.heads, self.kv_heads, self.d = heads, kv_heads, d
        self.plain = dict(qkv=rand((heads + 2 * kv_heads) * d, width), back=rand(width, heads * d), gate_up=rand(2 * hidden, width), down=rand(width, hidden))
        self.coded = {name: CodedMatrix(w, 5.0, seed + i) for i, (name, w) in enumerate(self.plain.items())}
        self.bias = (0.1 * rand(1, self.plain["qkv"].shape[0]))[0].bfloat16()
        self.norms = [(1 + 0.1 * torch.randn(width, generator=gen, device="cuda")).bfloat16() for _ in range(2)]

    def project(self, name, x, **more):
        m = self.coded[name]
        return E.ecasq_project(x, m.codes, m.levels, m.scales, GROUP, **more)

    def feed_forward(self, x, residual=None):
        """The block's second part for rows x (their sum with `residual`): its output, and what went into it."""
        y = E.ecasq_norm(x, self.norms[1], residual=residual)
        y, s = y if residual is not None else (y, x)
        m = self.coded["gate_up"]
        h = E.ecasq_gated(y, m.codes, m.levels, m.scales, GROUP, activation="silu")
        return self.project("down", h, residual=s), dict(s=s, y=y, h=h)

    def decode(self, x, keys, values, slots, table, lengths, seed, status):
        """One token of each sequence: the new residual stream, and what was computed on the way."""
        b, (heads, kv, d) = x.shape[0], (self.heads, self.kv_heads, self.d)
        y = E.ecasq_norm(x, self.norms[0])
        made = self.project("qkv", y, bias=self.bias, status=status).view(b, heads + 2 * kv, d)
        q, k, v = made[:, :heads], made[:, heads:heads + kv], made[:, heads + kv:]
        keys.write(k, slots, 4.0, seed, status)
        values.write(v, slots, 4.0, seed + 1, status)
        mixed, _ = E.ecasq_attend(q, keys.codes, values.codes, table, lengths, k_levels=keys.levels, v_levels=values.levels, status=status)
        out = self.project("back", mixed.view(b, heads * d), status=status)
        end, seen = self.feed_forward(out, residual=x)
        return end, dict(seen, first=y, made=made, mixed=mixed, out=out)


def decode(width=512, heads=8, kv_heads=2, d=64, hidden=1024, b=4, steps=24, page_size=16, seed=0):
    """Decodes `steps` tokens of `b` sequences; what each step saw and gave, and the block."""
    block = Block(width, heads, kv_heads, d, hidden, seed)
    gen = torch.Generator(device="cuda").manual_seed(seed + 100)
    keys, values = (CodedCache(b, kv_heads, d, steps, page_size) for _ in range(2))
    pages = torch.randperm(b * keys.per, generator=gen, device="cuda").view(b, keys.per)
    table, status, seen = pages.to(torch.int32), torch.zeros(1, dtype=torch.int32, device="cuda"), []
    for t in range(steps):
        x = torch.randn(b, width, generator=gen, device="cuda").bfloat16()
        slots = pages[:, t // page_size] * page_size + t % page_size
        lengths = torch.full((b,), t + 1, dtype=torch.int32, device="cuda")
        end, parts = block.decode(x, keys, values, slots, table, lengths, seed + 2 * t, status)
        seen.append(dict(parts, x=x, end=end))
    assert status.item() == 0, status.item()
    return seen, block


def main():
    seen, block = decode()
    x = torch.cat([s["x"] for s in seen])
    prompt, _ = block.feed_forward(x)
    s = x.float()
    y = s * torch.rsqrt(s.square().mean(1, keepdim=True) + 1e-6) * block.norms[1].float()
    gate, up = (y @ block.plain["gate_up"].T).chunk(2, dim=1)
    want = s + (torch.nn.functional.silu(gate) * up) @ block.plain["down"].T
    print("feed-forward part of %d rows: %.3f of the added rows' size from the uncoded part's" %
          (len(x), ((prompt.float() - want).norm() / (want - s).norm()).item()))
    print("%d steps decoded, %d sequences" % (len(seen), len(seen[0]["x"])))


if __name__ == "__main__":
    main()
