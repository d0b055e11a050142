"""One attention layer decoding with coded weights and a coded cache.

    python examples/coded_decode.py

The layer's four weight matrices are divided by a scale for each group of 128 columns; one codebook of at most 16
values is solved for each (ecasq_solve), the weights are rounded to it without bias
(ecasq_quantize) and packed (ecasq_pack).  At each step the new token's queries, keys
and values come from products with the codes (ecasq_matvec); every new key and value row gets a codebook of at
most eight values of its own (ecasq_solve_batched) and goes into a paged cache as codes
(ecasq_cache_write); the token attends over the cache (ecasq_attend), and the last product gives the
layer's output.  Printed are the sizes and how far the output is from the layer's without any coding.  (Unbiased
rounding to four bits or fewer costs a good part of the norm on random data like this; what a trained layer loses is for its
user to measure.)
"""
import os
import sys

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_18147_gb300 as E

GROUP, WEIGHT_LEVELS, ROW_LEVELS = 128, 16, 8


class CodedMatrix:
    """W [n, k] as 4-bit codes: W[r, c] is about scales[r, c // GROUP] * levels[code[r, c]]."""

    def __init__(self, weight, budget_bits, seed, sample=16384):
        n, k = weight.shape
        wide = torch.nn.functional.pad(weight.float(), (0, -k % GROUP)).view(n, -1, GROUP)
        self.scales = wide.abs().amax(dim=2).clamp_(min=1e-30)
        # In bfloat16 the codebook's values, being values of its input, are bfloat16 too.
        unit = (wide / self.scales[..., None]).bfloat16().float().flatten(1)[:, :k].contiguous()
        flat = unit.view(-1)
        picked = flat[torch.randperm(flat.numel(), generator=torch.Generator().manual_seed(seed))[:sample].to(flat.device)]
        picked = torch.cat([picked, flat.min()[None], flat.max()[None]])
        book, _ = E.ecasq_solve(picked, WEIGHT_LEVELS, budget_bits=budget_bits)
        idx, _, self.entropy = E.ecasq_quantize(flat, book, seed)
        self.codes, self.levels, self.shape = E.ecasq_pack(idx.view(n, k)), book.bfloat16(), (n, k)
        self.idx = idx.view(n, k)

    def __call__(self, x):
        return E.ecasq_matvec(x, self.codes, self.levels, self.scales, GROUP)

    def values(self):
        scales = self.scales.repeat_interleave(GROUP, dim=1)[:, :self.shape[1]]
        return self.levels.float()[self.idx.long()] * scales

    def bytes(self):
        return self.codes.numel() + 4 * self.scales.numel() + 2 * self.levels.numel()


class CodedCache:
    """Keys or values of `b` sequences in pages of coded rows."""

    def __init__(self, b, heads, d, most, page_size):
        self.per = -(-most // page_size)
        pages = b * self.per
        self.codes = torch.zeros(pages, page_size, heads, d // 2, dtype=torch.uint8, device="cuda")
        self.levels = torch.zeros(pages, page_size, heads, ROW_LEVELS, dtype=torch.bfloat16, device="cuda")

    def write(self, rows, slots, budget_bits, seed, status):
        n, heads, d = rows.shape
        books, m, _ = E.ecasq_solve_batched(rows.float().reshape(n * heads, d), ROW_LEVELS, budget_bits=budget_bits)
        E.ecasq_cache_write(rows, books, m, slots, self.codes, self.levels, seed, status=status)


def decode(width=512, heads=8, kv_heads=2, d=64, b=4, steps=48, page_size=16, seed=0):
    """Decodes `steps` tokens of `b` sequences; a list of what each step saw and gave, and the layer."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    plain = [rand((heads + 2 * kv_heads) * d, width) / width ** 0.5, rand(width, heads * d) / (heads * d) ** 0.5]
    qkv, last = (CodedMatrix(w, 5.0, seed + i) for i, w in enumerate(plain))
    keys, values = (CodedCache(b, kv_heads, d, steps, page_size) for _ in range(2))
    pages = torch.randperm(b * keys.per, generator=gen, device="cuda").view(b, keys.per)
    table = pages.to(torch.int32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = E.workspace_attend(b, heads, kv_heads, d, steps)
    seen, whole_k, whole_v = [], [], []
    for t in range(steps):
        x = rand(b, width).bfloat16()
        made = qkv(x).view(b, heads + 2 * kv_heads, d)
        q, k, v = made[:, :heads], made[:, heads:heads + kv_heads], made[:, heads + kv_heads:]
        slots = pages[:, t // page_size] * page_size + t % page_size
        keys.write(k, slots, 4.0, seed + 2 * t, status)
        values.write(v, slots, 4.0, seed + 2 * t + 1, status)
        lengths = torch.full((b,), t + 1, dtype=torch.int32, device="cuda")
        mixed, lse = E.ecasq_attend(q, keys.codes, values.codes, table, lengths, k_levels=keys.levels, v_levels=values.levels,
                                    max_len=t + 1, ws=ws, status=status)
        out = last(mixed.view(b, heads * d))
        # the same token through the layer without any coding
        exact = (x.float() @ plain[0].T).view(b, heads + 2 * kv_heads, d)
        whole_k.append(exact[:, heads:heads + kv_heads])
        whole_v.append(exact[:, heads + kv_heads:])
        group = heads // kv_heads
        kk, vv = (torch.stack(w, 2).repeat_interleave(group, dim=1) for w in (whole_k, whole_v))
        p = torch.softmax((exact[:, :heads, None] @ kk.transpose(2, 3)) * d ** -0.5, dim=-1)
        want = (p @ vv).reshape(b, heads * d) @ plain[1].T
        seen.append(dict(x=x, q=q, mixed=mixed, lse=lse, out=out, want=want, slots=slots))
    assert status.item() == 0, status.item()
    return seen, dict(qkv=qkv, last=last, keys=keys, values=values, table=table, pages=pages, page_size=page_size)


def main():
    seen, layer = decode()
    far = [((s["out"].float() - s["want"]).norm() / s["want"].norm()).item() for s in seen]
    for name in ("qkv", "last"):
        w = layer[name]
        print("%-5s %d x %d: %.2f bits a weight stored, entropy of the codes %.2f bits" %
              (name, *w.shape, 8.0 * w.bytes() / (w.shape[0] * w.shape[1]), w.entropy))
    row = layer["keys"].codes.shape[3] + 2 * ROW_LEVELS
    print("cache rows of %d values: %d bytes, in bfloat16 %d" % (2 * layer["keys"].codes.shape[3], row, 4 * layer["keys"].codes.shape[3]))
    print("%d steps; distance of the output from the uncoded layer's: first %.3f, median %.3f, last %.3f" %
          (len(far), far[0], sorted(far)[len(far) // 2], far[-1]))


if __name__ == "__main__":
    main()
