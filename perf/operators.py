"""Workloads of the 8-bit block-scaled products and of Newton-Schulz orthogonalisation, with their plain forms.

Three operators that one layer's training step runs one after the other:

* ``quantise``: a matrix to 8-bit floating point (e4m3) with one scale for every 1 x 128, or 128 x 128, block;
* ``product``: the matrix product of two such matrices, D = C + sum over blocks of (scale a)(scale b)(A_block B_block^T);
* ``orthogonalise``: Newton-Schulz iteration X <- aX + (bA + cA^2)X with A = X X^T, as the Muon optimiser applies it to an update.
"""
import math

import torch

own = False

FP8_MAX = 448.0
LEAST = 2.0 ** -100                       # smallest block maximum: keeps the inverse scale finite
COEFFS = (3.4445, -4.7750, 2.0315)
STEPS = 5
EPS = 1e-7
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}


def listed():
    return [
        # a decoding step's activations, 16 sequences: latency counts
        {"name": "quantise-decode", "op": "quantise", "rows": 16, "cols": 4096, "block": 1, "both": False, "type": "bfloat16"},
        # output gradients of one layer on the way into its two backward products
        {"name": "quantise-gradient", "op": "quantise", "rows": 8192, "cols": 4096, "block": 1, "both": True, "type": "bfloat16"},
        # master weights after an optimiser step, for the forward and the backward product
        {"name": "quantise-weights", "op": "quantise", "rows": 8192, "cols": 8192, "block": 128, "both": True, "type": "float32"},
        # one token against a square layer
        {"name": "product-token", "op": "product", "m": 1, "n": 4096, "k": 4096, "blocks": "row-tile", "type": "bfloat16", "add": False},
        # a decoding batch against a widening layer
        {"name": "product-batch", "op": "product", "m": 48, "n": 16384, "k": 4096, "blocks": "row-tile", "type": "bfloat16", "add": False},
        # a prompt of odd length and a head of odd width: every edge ragged
        {"name": "product-ragged", "op": "product", "m": 1001, "n": 1999, "k": 1100, "blocks": "row-tile", "type": "bfloat16", "add": False},
        # forward product of a training batch
        {"name": "product-forward", "op": "product", "m": 8192, "n": 8192, "k": 8192, "blocks": "row-tile", "type": "bfloat16", "add": False},
        # weight gradient, added to the one of the earlier micro-batches in 32 bits
        {"name": "product-weight-gradient", "op": "product", "m": 4096, "n": 4096, "k": 8192, "blocks": "row-row", "type": "float32", "add": True},
        # a small projection's update
        {"name": "orthogonalise-small", "op": "orthogonalise", "batch": 1, "m": 300, "n": 200, "type": "float32"},
        # the square projections of 16 layers at once
        {"name": "orthogonalise-layers", "op": "orthogonalise", "batch": 16, "m": 1024, "n": 1024, "type": "bfloat16"},
        # one wide layer
        {"name": "orthogonalise-wide", "op": "orthogonalise", "batch": 1, "m": 1000, "n": 4096, "type": "bfloat16"},
        # a tall layer of a large model
        {"name": "orthogonalise-tall", "op": "orthogonalise", "batch": 1, "m": 16384, "n": 4096, "type": "float32"},
    ]


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]; two in three are rounded to a multiple of 64 where that is possible."""
    v = 3072
    while v == 3072:
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        if rng.random() < 0.66 and v >= 64:
            v = (v + 32) // 64 * 64
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(("quantise", "product", "product", "orthogonalise"))
    if op == "quantise":
        block = rng.choice((1, 1, 128))
        return {"op": op, "rows": _log(rng, 1 if block == 1 else 128, 8192), "cols": _log(rng, 128, 8192), "block": block,
                "both": rng.random() < 0.6, "type": rng.choice(("float32", "bfloat16"))}
    if op == "product":
        wgrad = rng.random() < 0.3
        return {"op": op, "m": _log(rng, 128 if wgrad else 1, 8192), "n": _log(rng, 128, 8192), "k": _log(rng, 128, 8192),
                "blocks": "row-row" if wgrad else "row-tile", "type": "float32" if wgrad else "bfloat16", "add": wgrad}
    m, n = _log(rng, 64, 8192), _log(rng, 64, 8192)
    while min(m, n) > 4096:
        n = _log(rng, 64, 8192)
    small = max(m, n) <= 1500
    return {"op": op, "batch": rng.choice((1, 2, 8, 12)) if small else 1, "m": m, "n": n, "type": rng.choice(("float32", "bfloat16"))}


# ------------------------------------------------------------------------------------------------------- definitions
def _blocks(n):
    return (n + 127) // 128


def _row_scales(x, kind):
    """Scales and inverse scales of the 1 x 128 blocks of a matrix in the type `kind`: [rows, blocks] each."""
    rows, cols = x.shape
    pad = torch.zeros(rows, _blocks(cols) * 128, dtype=kind, device=x.device)
    pad[:, :cols] = x
    top = pad.abs().reshape(rows, -1, 128).amax(2).clamp_min(LEAST)
    return top / FP8_MAX, FP8_MAX / top


def _tile_scales(x, kind):
    """The same of the 128 x 128 blocks: [row blocks, column blocks]."""
    rows, cols = x.shape
    rb, cb = _blocks(rows), _blocks(cols)
    pad = torch.zeros(rb * 128, cb * 128, dtype=kind, device=x.device)
    pad[:rows, :cols] = x
    top = pad.abs().reshape(rb, 128, cb, 128).amax(3).amax(1).clamp_min(LEAST)
    return top / FP8_MAX, FP8_MAX / top


def _spread(s, block, rows, cols):
    """One scale for every entry of a rows x cols matrix from [row blocks, column blocks] of `block` x 128 entries."""
    s = s.repeat_interleave(128, 1)[:, :cols]
    return s if block == 1 else s.repeat_interleave(block, 0)[:rows]


def _to_fp8(x, block, kind=torch.float32):
    x = x.to(kind)
    s, inv = _row_scales(x, kind) if block == 1 else _tile_scales(x, kind)
    q = (x * _spread(inv, block, *x.shape)).clamp(-FP8_MAX, FP8_MAX)
    return q, s


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _activations(rows, cols, g):
    """Normal values with a spread of channel sizes and a few channels far above the rest."""
    size = torch.exp(0.6 * torch.randn(cols, generator=g, device="cuda"))
    size[torch.randint(0, cols, (max(1, cols // 256),), generator=g, device="cuda")] *= 20.0
    return torch.randn(rows, cols, generator=g, device="cuda") * size


def _gradients(rows, cols, g):
    """Normal values with a wide spread over the tokens (rows)."""
    return torch.randn(rows, cols, generator=g, device="cuda") * (1e-3 * torch.exp(1.5 * torch.randn(rows, 1, generator=g, device="cuda")))


def _weights(rows, cols, g):
    return torch.randn(rows, cols, generator=g, device="cuda") * 0.02


def _weight_gradient(batch, m, n, g):
    """Sums over tokens of outer products whose sizes fall off, and a floor of noise."""
    r = max(1, min(m, n) // 2)
    fall = torch.arange(1, r + 1, device="cuda", dtype=torch.float32) ** -0.5
    u = torch.randn(batch, m, r, generator=g, device="cuda") * fall
    v = torch.randn(batch, r, n, generator=g, device="cuda")
    return 1e-3 * (torch.matmul(u, v) + 0.3 * torch.randn(batch, m, n, generator=g, device="cuda"))


def _empty8(rows, cols):
    """An 8-bit matrix whose rows start on 16-byte boundaries."""
    return torch.empty(rows, (cols + 15) // 16 * 16, dtype=torch.float8_e4m3fn, device="cuda")[:, :cols]


def _empty_scales(rows, cols, block):
    """Scales of a rows x cols matrix: [row blocks, column blocks], one column block after the other in memory."""
    return torch.empty(_blocks(cols), rows if block == 1 else _blocks(rows), device="cuda").t()


def _quantised(x, block):
    q, s = _empty8(*x.shape), _empty_scales(*x.shape, block)
    values, scales = _to_fp8(x, block)
    q.copy_(values)
    s.copy_(scales)
    return q, s


def prepare(case, seed):
    g = _generator(seed)
    state = {"case": case}
    if case["op"] == "quantise":
        rows, cols, block, kind = case["rows"], case["cols"], case["block"], TYPES[case["type"]]
        make = _weights if block == 128 else _gradients if case["both"] else _activations
        state["x"] = make(rows, cols, g).to(kind)
        state["q"], state["s"] = _empty8(rows, cols), _empty_scales(rows, cols, block)
        if case["both"]:
            state["qt"], state["st"] = _empty8(cols, rows), _empty_scales(cols, rows, block)
    elif case["op"] == "product":
        m, n, k, kind = case["m"], case["n"], case["k"], TYPES[case["type"]]
        if case["blocks"] == "row-tile":
            state["a"], state["sa"] = _quantised(_activations(m, k, g), 1)
            state["b"], state["sb"] = _quantised(_weights(n, k, g), 128)
        else:
            state["a"], state["sa"] = _quantised(_gradients(k, m, g).t().contiguous(), 1)
            state["b"], state["sb"] = _quantised(_activations(k, n, g).t().contiguous(), 1)
        state["c"] = torch.randn(m, n, generator=g, device="cuda", dtype=kind) if case["add"] else None
        state["d"] = torch.empty(m, n, device="cuda", dtype=kind)
    else:
        state["g"] = _weight_gradient(case["batch"], case["m"], case["n"], g).to(TYPES[case["type"]])
        state["o"] = torch.empty(case["batch"], case["m"], case["n"], device="cuda", dtype=torch.bfloat16)
    return state


# ---------------------------------------------------------------------------------------------------------- the calls
_workspace = [None]


def _library(state, op, *sizes):
    """The library with a workspace that is large enough; the program keeps the workspace, and asks for its size once."""
    from paper_2609_05419_b200 import binding
    if "bytes" not in state:
        state["bytes"] = binding.workspace_bytes(getattr(binding, op), *sizes, 1)
    if _workspace[0] is None or _workspace[0].numel() < state["bytes"]:
        _workspace[0] = torch.zeros(state["bytes"], dtype=torch.uint8, device="cuda")
        binding.set_workspace(_workspace[0])
    return binding


def _run_own(state):
    case = state["case"]
    if case["op"] == "quantise":
        from paper_2609_05419_b200 import binding
        if case["both"]:
            binding.fp8_quantise(state["x"], state["q"], state["s"], state["qt"], state["st"], block_rows=case["block"])
            return state["q"], state["s"], state["qt"], state["st"]
        binding.fp8_quantise(state["x"], state["q"], state["s"], block_rows=case["block"])
        return state["q"], state["s"]
    if case["op"] == "product":
        lib = _library(state, "OP_FP8_GEMM", case["m"], case["n"], case["k"])
        lib.fp8_gemm(state["a"], state["sa"], state["b"], state["sb"], state["d"], C=state["c"],
                     b_block=128 if case["blocks"] == "row-tile" else 1)
        return state["d"]
    lib = _library(state, "OP_NEWTON_SCHULZ", case["m"], case["n"], case["batch"])
    lib.newton_schulz(state["g"], state["o"], steps=STEPS, coeffs=COEFFS, eps=EPS)
    return state["o"]


def _run_plain(state):
    case = state["case"]
    if case["op"] == "quantise":
        q, s = _to_fp8(state["x"], case["block"])
        out = (q.to(torch.float8_e4m3fn), s)
        if case["both"] and case["block"] == 1:
            qt, st = _to_fp8(state["x"].t(), 1)
            out += (qt.to(torch.float8_e4m3fn), st)
        elif case["both"]:
            out += (out[0].t(), s.t())
        return out
    if case["op"] == "product":
        m, n, k = case["m"], case["n"], case["k"]
        a = state["a"].float() * _spread(state["sa"], 1, m, k)
        b = state["b"].float() * _spread(state["sb"], 128 if case["blocks"] == "row-tile" else 1, n, k)
        d = torch.matmul(a, b.t())
        if case["add"]:
            d = d + state["c"]
        return d.to(TYPES[case["type"]])
    a, b, c = COEFFS
    x = state["g"].float()
    x = x / ((x * x).sum((1, 2), keepdim=True).sqrt() + EPS)
    tall = case["m"] > case["n"]
    x = x.transpose(1, 2) if tall else x
    for _ in range(STEPS):
        gram = torch.matmul(x, x.transpose(1, 2))
        x = a * x + torch.matmul(b * gram + c * torch.matmul(gram, gram), x)
    return (x.transpose(1, 2) if tall else x).to(torch.bfloat16)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------ what a pass is worth
def work(case):
    if case["op"] == "quantise":
        rows, cols = case["rows"], case["cols"]
        forms = 2 if case["both"] else 1
        scales = rows * _blocks(cols) + (cols * _blocks(rows) if case["both"] else 0) if case["block"] == 1 \
            else forms * _blocks(rows) * _blocks(cols)
        return {"bytes": rows * cols * (4 if case["type"] == "float32" else 2) + forms * rows * cols + 4 * scales, "flops": 4 * rows * cols}
    if case["op"] == "product":
        m, n, k = case["m"], case["n"], case["k"]
        scales = m * _blocks(k) + (_blocks(n) if case["blocks"] == "row-tile" else n) * _blocks(k)
        out = m * n * (4 if case["type"] == "float32" else 2)
        return {"bytes": m * k + n * k + 4 * scales + out * (2 if case["add"] else 1), "flops": 2 * m * n * k}
    short, long = min(case["m"], case["n"]), max(case["m"], case["n"])
    # the two symmetric products need one half of their entries
    flops = case["batch"] * STEPS * (short * short * long + short ** 3 + 2 * short * short * long)
    return {"bytes": case["batch"] * case["m"] * case["n"] * ((4 if case["type"] == "float32" else 2) + 2), "flops": flops}


# --------------------------------------------------------------------------------------------- the definitions in 64 bits
def _fp8_nearest(v):
    """The e4m3 value nearest to each |v| <= 448 (ties to even): the spacing is 2^(exponent - 3), and 2^-9 below 2^-6."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(v / step) * step


def _exact_quantise(x, block):
    x = x.double()
    rows, cols = x.shape
    s = torch.empty(rows if block == 1 else _blocks(rows), _blocks(cols), dtype=torch.float64, device=x.device)
    q = torch.empty_like(x)
    for j in range(_blocks(cols)):
        part = x[:, 128 * j:128 * (j + 1)]
        top = part.abs().amax(1, keepdim=True).clamp_min(LEAST)
        if block == 128:
            top = torch.cat([t.amax().expand(len(t), 1) for t in top.split(128)])
        s[:, j] = top[::block, 0] / FP8_MAX
        q[:, 128 * j:128 * (j + 1)] = _fp8_nearest(part * FP8_MAX / top)
    return q, s


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "quantise":
        out = _exact_quantise(state["x"], case["block"])
        if case["both"]:
            out += _exact_quantise(state["x"].t(), case["block"])
        return out
    if case["op"] == "product":
        a, b = state["a"].double(), state["b"].double()
        per_tile = case["blocks"] == "row-tile"
        d = state["c"].double() if case["add"] else torch.zeros(case["m"], case["n"], dtype=torch.float64, device="cuda")
        for j in range(_blocks(case["k"])):
            sb = state["sb"][:, j].double()
            if per_tile:
                sb = sb[torch.arange(case["n"], device="cuda") // 128]
            cut = slice(128 * j, 128 * (j + 1))
            d += (a[:, cut] * state["sa"][:, j:j + 1].double()) @ (b[:, cut] * sb[:, None]).t()
        return d
    a, b, c = COEFFS
    out = torch.empty(case["batch"], case["m"], case["n"], dtype=torch.float64, device="cuda")
    for i in range(case["batch"]):
        x = state["g"][i].double()
        x = x / (torch.linalg.vector_norm(x) + EPS)
        for _ in range(STEPS):      # the polynomial from the side that costs less: (X X^T)^j X = X (X^T X)^j
            if case["m"] <= case["n"]:
                y = x @ x.t()
                x = a * x + b * (y @ x) + c * (y @ (y @ x))
            else:
                y = x.t() @ x
                x = a * x + b * (x @ y) + c * ((x @ y) @ y)
        out[i] = x
    return out
