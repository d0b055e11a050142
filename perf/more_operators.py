"""Timed calls of the operators around coded matrices in a served layer, with their inputs, work and plain forms.

A case is a dict of plain values: its "kind" names the operator, the rest its sizes and types.
listed() gives twelve of them, draw() more of the same ranges; prepare() makes what a program has
in hand before the call, run() is one call, exact() the same outputs from the definitions in 64 bits.
Where `own` is false run() computes them from elementary torch operations in 32 bits.

project  y = act(x W^T + bias) + residual, W[r, c] = scale[r, c div group] * levels[code[r, c]], 4-bit codes
gated    h = act(x G^T) * (x U^T) for the rows G, then U, of one coded matrix
norm     s = x + residual, y = s / sqrt(mean(s^2) + eps) * weight; or y as e4m3 values with a scale for each group
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6


def listed():
    return [
        # One token through a small projection back into the residual stream: launch and latency.
        dict(name="project_1024x1024_b1_bf16", kind="project", n=1024, k=1024, b=1, group=128, dtype="bf16", scales="f32",
             bias=False, act="none", residual=True),
        # A few sequences decoded together through a square projection with bias, fine groups.
        dict(name="project_8192x8192_b4_f16", kind="project", n=8192, k=8192, b=4, group=64, dtype="f16", scales="f16",
             bias=True, act="none", residual=False),
        # Single-precision activations; a group size that is no power of two.
        dict(name="project_2999x2050_b3_f32", kind="project", n=2999, k=2050, b=3, group=96, dtype="f32", scales="f32",
             bias=True, act="silu", residual=False),
        # A larger batch decoded together, a ragged matrix, the finest groups, everything in the epilogue; rows off 16-byte boundaries.
        dict(name="project_5003x4097_b40_bf16", kind="project", n=5003, k=4097, b=40, group=32, dtype="bf16", scales="bf16",
             bias=True, act="gelu", residual=True),
        # A prompt through a square projection back into the residual stream.
        dict(name="project_8192x8192_b4096_bf16", kind="project", n=8192, k=8192, b=4096, group=128, dtype="bf16", scales="f32",
             bias=False, act="none", residual=True),
        # One token through a feed-forward block's first half.
        dict(name="gated_8192x4096_b1_bf16", kind="gated", n=8192, k=4096, b=1, group=128, dtype="bf16", scales="f32", act="silu"),
        # A larger batch, odd sizes, finer groups, the other activation.
        dict(name="gated_5001x4104_b100_f16", kind="gated", n=5001, k=4104, b=100, group=64, dtype="f16", scales="f16",
             act="gelu_tanh"),
        # Several prompts packed together.
        dict(name="gated_16384x4096_b2048_bf16", kind="gated", n=16384, k=4096, b=2048, group=128, dtype="bf16", scales="f32",
             act="silu"),
        # One token between two blocks.
        dict(name="norm_1x4096_bf16", kind="norm", b=1, k=4096, dtype="bf16", weight="bf16", residual=True, group=0),
        # Odd rows in single precision, without a residual.
        dict(name="norm_3001x5003_f32", kind="norm", b=3001, k=5003, dtype="f32", weight="f32", residual=False, group=0),
        # A prompt, coded to 8 bits in blocks of 128.
        dict(name="norm_8192x8192_bf16_8bit", kind="norm", b=8192, k=8192, dtype="bf16", weight="bf16", residual=True, group=128),
        # A decoded batch, coded to 8 bits with a scale a row.
        dict(name="norm_64x6000_f16_8bit", kind="norm", b=64, k=6000, dtype="f16", weight="f32", residual=True, group=6000),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("project", "project", "gated", "gated", "norm"))
    dtype = rng.choice(("f16", "bf16", "bf16"))
    if kind == "norm":
        dtype = rng.choice(("f16", "bf16", "bf16", "f32"))
        k = _log_int(rng, 64, 16384)
        b = _log_int(rng, 1, min(8192, (1 << 26) // k))
        return dict(kind=kind, b=b, k=k, dtype=dtype, weight=rng.choice((dtype, "f32")), residual=rng.random() < 0.7,
                    group=rng.choice((0, 0, 64, 128, k)))
    if kind == "project" and rng.random() < 0.2:
        dtype = "f32"
    n, k = _log_int(rng, 128, 16384), _log_int(rng, 128, 16384)
    if rng.random() < 0.5:  # half of the matrices have whole blocks, the others any size
        n, k = 64 * max(2, n // 64) + 8, 64 * max(2, k // 64)
    # Half of the batches are of decoded tokens, the others of prompts; single precision is for small ones.
    most = 64 if dtype == "f32" else (1 << 38) // (n * k * (2 if kind == "gated" else 1))
    b = min(most, _log_int(rng, 1, 64) if rng.random() < 0.5 else _log_int(rng, 64, 4096))
    case = dict(kind=kind, n=n, k=k, b=b, group=rng.choice((32, 64, 96, 128, 128, 256)), dtype=dtype,
                scales=rng.choice((dtype, "f32")))
    if kind == "gated":
        return dict(case, act=rng.choice(("silu", "gelu", "gelu_tanh", "relu")))
    return dict(case, bias=rng.random() < 0.5, act=rng.choice(("none", "none", "relu", "silu", "gelu", "gelu_tanh")),
                residual=rng.random() < 0.5)


def work(case):
    b, k, e = case["b"], case["k"], SIZES[case["dtype"]]
    if case["kind"] == "norm":
        read = b * k * e * (2 if case["residual"] else 1) + k * SIZES[case["weight"]]
        wrote = b * k * (e if case["residual"] else 0) + (b * k + 4 * b * -(-k // case["group"]) if case["group"] else b * k * e)
        return {"bytes": read + wrote, "flops": 6 * b * k}
    n = case["n"]
    rows = 2 * n if case["kind"] == "gated" else n
    weights = rows * ((k + 1) // 2) + rows * (-(-k // case["group"])) * SIZES[case["scales"]] + 16 * e
    more = 0 if case["kind"] == "gated" else (n * e if case["bias"] else 0) + (b * n * e if case["residual"] else 0)
    return {"bytes": weights + (b * k + b * n) * e + more, "flops": 2 * b * rows * k}


# ------------------------------------------------------------------ inputs

def _matrix(gen, rows, case):
    """Codes as packed rows, levels and scales of a coded matrix."""
    k, group = case["k"], case["group"]
    # Normalised weights are spread normally over +-1: the codes of a codebook fitted to them crowd in the middle.
    wide = -(-k // 128) * 128
    idx = (torch.randn(rows, wide, generator=gen, device="cuda") * 2.6 + 8.0).clamp_(0, 15).to(torch.uint8)
    idx[:, k:] = 0
    # Blocks of 128 columns, sixteen words of eight codes each, the words of a block stored as a transposed 4 x 4 square.
    codes = (idx[:, 0::2] | (idx[:, 1::2] << 4)).view(rows, wide // 128, 4, 4, 4).transpose(2, 3).reshape(rows, wide // 2)
    levels = torch.linspace(-1, 1, 16, device="cuda") ** 3 * 0.6 + torch.linspace(-0.4, 0.4, 16, device="cuda")
    # Spread so that an output has about the spread of the inputs.
    scales = (torch.rand(rows, -(-k // group), generator=gen, device="cuda") + 0.5) / (0.36 * math.sqrt(k))
    return codes, levels.to(DTYPES[case["dtype"]]), scales.to(DTYPES[case["scales"]])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    dt, b, k = DTYPES[case["dtype"]], case["b"], case["k"]
    if case["kind"] == "norm":
        # A residual stream: rows of unequal size, a few columns far above the others; what a block adds is smaller.
        stream = rand(b, k) * (0.5 + 4 * torch.rand(b, 1, generator=gen, device="cuda"))
        stream = torch.where(torch.rand(k, generator=gen, device="cuda") < 0.002, stream * 30, stream)
        x, residual = (rand(b, k), stream) if case["residual"] else (stream, None)
        return dict(case=case, x=x.to(dt), residual=None if residual is None else residual.to(dt),
                    weight=(1 + 0.2 * rand(k)).to(DTYPES[case["weight"]]))
    n = case["n"]
    codes, levels, scales = _matrix(gen, 2 * n if case["kind"] == "gated" else n, case)
    state = dict(case=case, x=rand(b, k).to(dt), codes=codes, levels=levels, scales=scales)
    if case["kind"] == "project":
        state["bias"] = (0.3 * rand(n)).to(dt) if case["bias"] else None
        state["residual"] = (2 * rand(b, n)).to(dt) if case["residual"] else None
    return state


# --------------------------------------------------------------- plain forms

def _act(v, name):
    if name == "relu":
        return torch.where(v > 0, v, 0.0)
    if name == "silu":
        return v / (1 + torch.exp(-v))
    if name == "gelu":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))
    return v


def _plain_products(s):
    case = s["case"]
    k = case["k"]
    codes = s["codes"].view(s["codes"].shape[0], -1, 4, 4, 4).transpose(2, 3).flatten(1)
    idx = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(1)[:, :k].long()
    w = s["levels"].float()[idx]
    del idx
    w *= s["scales"].float().repeat_interleave(case["group"], dim=1)[:, :k]
    return s["x"].float() @ w.T


def _plain_project(s):
    y = _plain_products(s)
    if s["bias"] is not None:
        y = y + s["bias"].float()
    y = _act(y, s["case"]["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


def _plain_gated(s):
    both = _plain_products(s)
    n = s["case"]["n"]
    return (_act(both[:, :n], s["case"]["act"]) * both[:, n:]).to(s["x"].dtype)


def _plain_norm(s):
    case, x = s["case"], s["x"]
    total = x if s["residual"] is None else (x.float() + s["residual"].float()).to(x.dtype)
    v = total.float()
    y = v * torch.rsqrt((v * v).mean(dim=1, keepdim=True) + EPS) * s["weight"].float()
    if not case["group"]:
        out = (y.to(x.dtype),)
    else:
        b, k, group = case["b"], case["k"], case["group"]
        wide = torch.nn.functional.pad(y, (0, -k % group)).view(b, -1, group)
        scale = wide.abs().amax(dim=2) / 448.0
        scale = torch.where(scale > 0, scale, 1.0)
        q = (wide / scale[..., None]).clamp(-448.0, 448.0).flatten(1)[:, :k]
        out = (q.to(torch.float8_e4m3fn), scale)
    return out if s["residual"] is None else out + (total,)


def run(state):
    case = state["case"]
    kind = case["kind"]
    if not own:
        return {"project": _plain_project, "gated": _plain_gated, "norm": _plain_norm}[kind](state)
    import paper_2608_18147_gb300 as E

    if kind == "norm":
        out = E.ecasq_norm(state["x"], state["weight"], EPS, residual=state["residual"], group=case["group"] or None)
        return out if isinstance(out, tuple) else (out,)
    if "ws" not in state:
        state["ws"] = E.workspace_project(case["b"], state["codes"].shape[0], case["k"], state["x"].dtype)
    if kind == "gated":
        return E.ecasq_gated(state["x"], state["codes"], state["levels"], state["scales"], case["group"],
                             activation=case["act"], ws=state["ws"])
    return E.ecasq_project(state["x"], state["codes"], state["levels"], state["scales"], case["group"], bias=state["bias"],
                           activation=None if case["act"] == "none" else case["act"], residual=state["residual"],
                           ws=state["ws"])


# ------------------------------------------------------- definitions in 64 bits

def _phi(v, name):
    """The activations from their other forms: the normal distribution's tail and the logistic function."""
    if name == "relu":
        return v.clamp(min=0)
    if name == "silu":
        return v * torch.sigmoid(v)
    if name == "gelu":
        return v * torch.special.ndtr(v)
    if name == "gelu_tanh":
        return v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
    return v


def _exact_products(s, case):
    """A run of the matrix's rows at a time, the scales folded into the activations of each group."""
    rows, k, b, group = s["codes"].shape[0], case["k"], case["b"], case["group"]
    col = torch.arange(k, device="cuda")
    word = col % 128 // 8
    byte = col // 128 * 64 + (word % 4 * 4 + word // 4) * 4 + col % 8 // 2
    shift = torch.where(col % 2 == 1, 16, 1).int()
    x = s["x"].double()
    y = torch.zeros(b, rows, dtype=torch.float64, device="cuda")
    for at in range(0, rows, 2048):
        w = s["levels"].double()[s["codes"][at:at + 2048][:, byte].int() // shift % 16]
        scale = s["scales"][at:at + 2048].double()
        for i in range(-(-k // group)):
            w[:, i * group:(i + 1) * group] *= scale[:, i:i + 1]
        y[:, at:at + 2048] = x @ w.T
    return y


def _exact_norm(s, case):
    x = s["x"].double()
    total = None
    if s["residual"] is not None:
        total = x + s["residual"].double()
        x = total.to(s["x"].dtype).double()  # what is normalised is the sum as it is stored
    size = torch.linalg.vector_norm(x, dim=1) / math.sqrt(case["k"])
    y = x / torch.hypot(size, torch.tensor(math.sqrt(EPS), dtype=torch.float64, device="cuda"))[:, None] * s["weight"].double()
    if not case["group"]:
        out = (y,)
    else:
        group = case["group"]
        scale = torch.stack([y[:, at:at + group].abs().amax(dim=1) / 448 for at in range(0, case["k"], group)], dim=1)
        at = torch.arange(case["k"], device="cuda") // group
        out = (y / scale[:, at], scale)  # the values before they are rounded
    return out if total is None else out + (total,)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        return _exact_norm(s, case)
    y = _exact_products(s, case)
    if case["kind"] == "gated":
        return _phi(y[:, :case["n"]], case["act"]) * y[:, case["n"]:]
    if s["bias"] is not None:
        y = y + s["bias"].double()
    y = _phi(y, case["act"])
    return y if s["residual"] is None else y + s["residual"].double()
