"""Workloads of what stands around the 8-bit products of a layer, with their plain forms.

Four operators, next to ``quantise``, ``product`` and ``orthogonalise`` of a layer's step:

* ``norm``: residual addition and root-mean-square norm, written as the 8-bit operands (e4m3, a scale per 1 x 128 block, along the rows and,
  for the weight gradient, along the columns) of the products that follow;
* ``norm-backward``: the gradients of its input and of its weights;
* ``clip``: the common 2-norm of all gradients of a model, and the gradients scaled down where it is above a limit;
* ``adapters``: low-rank updates of many requests added to a shared projection's output, D = C + s_a (X A_a^T) B_a^T with the adapter a of each token.
"""
import math

import torch

own = False

FP8_MAX = 448.0
LEAST = 2.0 ** -100                       # smallest block maximum: keeps the inverse scale finite
NORM_EPS = 1e-6
CLIP_EPS = 1e-6
TYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
SIZE = {"float32": 4, "float16": 2, "bfloat16": 2}


def listed():
    return [
        # a decoding step of 16 sequences on its way into the next projection: latency counts
        {"name": "norm-decode", "op": "norm", "rows": 16, "cols": 4096, "type": "bfloat16", "residual": True, "both": False, "plain": False},
        # a training batch: the operands of the forward product and of the weight gradient, and what the backward pass needs
        {"name": "norm-training", "op": "norm", "rows": 8192, "cols": 4096, "type": "bfloat16", "residual": True, "both": True, "plain": False},
        # the last norm of a stack of odd width, kept in 32 bits and in 8: every edge ragged, nothing to add
        {"name": "norm-ragged", "op": "norm", "rows": 1001, "cols": 1999, "type": "float32", "residual": False, "both": True, "plain": True},
        # backward pass of the training batch, joined with the gradient that came along the residual path
        {"name": "backward-training", "op": "norm-backward", "rows": 8192, "cols": 4096, "type": "bfloat16", "residual": True},
        # backward pass of the ragged one
        {"name": "backward-ragged", "op": "norm-backward", "rows": 1001, "cols": 1999, "type": "float32", "residual": False},
        # a small network's gradients, 32 bits: latency counts
        {"name": "clip-small", "op": "clip", "layers": 2, "width": 200, "inner": 300, "type": "float32", "limit": 1.0},
        # ten layers of a small model in 16 bits, small enough for the on-chip cache
        {"name": "clip-layers", "op": "clip", "layers": 10, "width": 1024, "inner": 1500, "type": "bfloat16", "limit": 1.0},
        # four layers of a large model, gradients summed in 32 bits over micro-batches
        {"name": "clip-large", "op": "clip", "layers": 4, "width": 4096, "inner": 16384, "type": "float32", "limit": 1.0},
        # one token against one of the resident adapters
        {"name": "adapters-token", "op": "adapters", "tokens": 1, "k": 4096, "n": 4096, "adapters": 8, "rank": 16, "type": "bfloat16", "runs": False, "bare": False},
        # a decoding batch against a widening layer, two sequences to an adapter, some sequences without one
        {"name": "adapters-batch", "op": "adapters", "tokens": 48, "k": 4096, "n": 16384, "adapters": 24, "rank": 16, "type": "bfloat16", "runs": False, "bare": True},
        # prompts of odd lengths side by side, ranks of several sizes, every edge ragged
        {"name": "adapters-ragged", "op": "adapters", "tokens": 1001, "k": 1100, "n": 1999, "adapters": 5, "rank": 24, "type": "float16", "runs": True, "bare": True},
        # long prompts of eight customers at once, large ranks
        {"name": "adapters-prompts", "op": "adapters", "tokens": 8192, "k": 8192, "n": 8192, "adapters": 8, "rank": 64, "type": "bfloat16", "runs": True, "bare": False},
    ]


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]; two in three are rounded to a multiple of 64 where that is possible."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.66 and v >= 64:
        v = (v + 32) // 64 * 64
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(("norm", "norm", "norm-backward", "clip", "adapters", "adapters"))
    if op in ("norm", "norm-backward"):
        kind = rng.choice(("bfloat16", "bfloat16", "float16", "float32"))
        cols = _log(rng, 64, 16384)
        rows = _log(rng, 1, min(16384, max(1, 8192 * 4096 * 2 // (cols * SIZE[kind]))))
        case = {"op": op, "rows": rows, "cols": cols, "type": kind, "residual": rng.random() < 0.7}
        if op == "norm":
            case.update(both=rng.random() < 0.5, plain=rng.random() < 0.3)
        return case
    if op == "clip":
        width, inner = _log(rng, 16, 4096), _log(rng, 16, 16384)
        most = max(1, min(10, 4 * 4096 * 16384 // max(1, width * inner)))
        return {"op": op, "layers": _log(rng, 1, most), "width": width, "inner": inner, "type": rng.choice(("float32", "bfloat16", "float16")),
                "limit": rng.choice((1.0, 1.0, 0.01, 1e4))}
    tokens, adapters = _log(rng, 1, 8192), _log(rng, 1, 64)
    return {"op": op, "tokens": tokens, "k": _log(rng, 64, 8192), "n": _log(rng, 64, 8192), "adapters": adapters, "rank": rng.choice((1, 4, 8, 8, 16, 16, 24, 32, 33, 64)),
            "type": rng.choice(("bfloat16", "bfloat16", "float16")), "runs": tokens >= 256 and rng.random() < 0.8, "bare": rng.random() < 0.5}


# ------------------------------------------------------------------------------------------------------------- inputs
def _blocks(n):
    return (n + 127) // 128


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _stream(rows, cols, g):
    """A residual stream: normal values, a spread of channel sizes, a few channels far above the rest."""
    size = torch.exp(0.5 * _randn(g, cols))
    size[torch.randint(0, cols, (max(1, cols // 512),), generator=g, device="cuda")] *= 30.0
    return _randn(g, rows, cols) * size


def _gradients(rows, cols, g):
    """Normal values with a wide spread over the tokens (rows)."""
    return _randn(g, rows, cols) * (1e-3 * torch.exp(1.5 * _randn(g, rows, 1)))


def _empty8(rows, cols):
    """An 8-bit matrix whose rows start on 16-byte boundaries."""
    return torch.empty(rows, (cols + 15) // 16 * 16, dtype=torch.float8_e4m3fn, device="cuda")[:, :cols]


def _layer_shapes(case):
    """The gradients of one layer: two square projections, a widening and a narrowing one, two norms; the first layer has an input embedding too."""
    w, i = case["width"], case["inner"]
    shapes = [(w, w), (w, w), (i, w), (w, i), (w,), (w,)]
    return [(2 * w, w)] + shapes * case["layers"]


def _ranks(case):
    """Ranks differ from adapter to adapter: the full one, a half, a third."""
    return [max(1, case["rank"] // (1 + a % 3)) for a in range(case["adapters"])]


def prepare(case, seed):
    g = _generator(seed)
    state = {"case": case}
    kind = TYPES[case["type"]]
    if case["op"] == "norm":
        rows, cols = case["rows"], case["cols"]
        state["x"] = _stream(rows, cols, g).to(kind)
        state["w"] = 1 + 0.2 * _randn(g, cols)
        if case["residual"]:
            state["r"] = (0.3 * _randn(g, rows, cols)).to(kind)
            state["h"] = torch.empty(rows, cols, dtype=kind, device="cuda")
        state["y"] = torch.empty(rows, cols, dtype=kind, device="cuda") if case["plain"] else None
        state["q"], state["s"] = _empty8(rows, cols), torch.empty(_blocks(cols), rows, device="cuda").t()
        if case["both"]:
            state["qt"], state["st"] = _empty8(cols, rows), torch.empty(_blocks(rows), cols, device="cuda").t()
            state["rstd"] = torch.empty(rows, device="cuda")
    elif case["op"] == "norm-backward":
        rows, cols = case["rows"], case["cols"]
        state["h"] = _stream(rows, cols, g).to(kind)
        state["w"] = 1 + 0.2 * _randn(g, cols)
        state["rstd"] = (state["h"].float().square().mean(1) + NORM_EPS).rsqrt()
        state["dy"] = _gradients(rows, cols, g).to(kind)
        state["dr"] = _gradients(rows, cols, g).to(kind) if case["residual"] else None
        state["dx"] = torch.empty(rows, cols, dtype=kind, device="cuda")
        state["dw"] = torch.empty(cols, device="cuda")
    elif case["op"] == "clip":
        # the input embedding's gradient has rows of tokens that did not occur; sizes fall off from tensor to tensor
        grads = [_randn(g, *shape).mul_(0.02 / (1 + j % 7)) for j, shape in enumerate(_layer_shapes(case))]
        grads[0] *= (torch.rand(len(grads[0]), 1, generator=g, device="cuda") < 0.25)
        state["g"] = [t.to(kind) for t in grads]
        state["o"] = [torch.empty_like(t) for t in state["g"]]
        state["norm"] = torch.empty((), device="cuda")
    else:
        tokens, k, n, many, rank = case["tokens"], case["k"], case["n"], case["adapters"], case["rank"]
        ranks = torch.tensor(_ranks(case), dtype=torch.int32, device="cuda")
        used = torch.arange(rank, device="cuda")[None, :] < ranks[:, None]
        state["x"] = _stream(tokens, k, g).to(kind)
        state["a"] = (_randn(g, many, rank, k) * k ** -0.5 * used[:, :, None]).to(kind)
        state["b"] = (_randn(g, many, n, rank) * 0.1 * used[:, None, :]).to(kind)
        state["scale"] = 16.0 / ranks.float().sqrt()
        state["ranks"] = ranks
        if case["runs"]:
            cuts = torch.sort(torch.randint(0, tokens + 1, (many - 1,), generator=g, device="cuda"))[0]
            index = torch.searchsorted(cuts, torch.arange(tokens, device="cuda"), right=True)
        else:
            index = torch.randperm(max(tokens, many), generator=g, device="cuda")[:tokens] % many
        if case["bare"]:
            index[torch.randperm(tokens, generator=g, device="cuda")[:tokens // 8]] = -1
        state["index"] = index.to(torch.int32)
        state["c"] = (5 * _randn(g, tokens, n)).to(kind)
        state["d"] = torch.empty(tokens, n, dtype=kind, device="cuda")
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
    if case["op"] == "norm":
        lib = _library(state, "OP_RMS_NORM", case["rows"], case["cols"], 1)
        lib.rms_norm(state["x"], state["w"], R=state.get("r"), H=state.get("h"), Y=state["y"], Q=state["q"], S=state["s"],
                     Qt=state.get("qt"), St=state.get("st"), rstd=state.get("rstd"), eps=NORM_EPS)
        return {name: state[name] for name in ("h", "y", "q", "s", "qt", "st", "rstd") if state.get(name) is not None}
    if case["op"] == "norm-backward":
        lib = _library(state, "OP_RMS_NORM_BACKWARD", case["rows"], case["cols"], 1)
        lib.rms_norm_backward(state["dy"], state["h"], state["w"], state["rstd"], state["dx"], dR=state["dr"], dW=state["dw"])
        return state["dx"], state["dw"]
    if case["op"] == "clip":
        lib = _library(state, "OP_CLIP_GRADIENTS", len(state["g"]), 1, 1)
        lib.clip_gradients(state["g"], case["limit"], out=state["o"], norm=state["norm"], eps=CLIP_EPS)
        return state["o"], state["norm"]
    lib = _library(state, "OP_ADAPTER_ADD", case["tokens"], case["rank"], case["adapters"])
    lib.adapter_add(state["x"], state["a"], state["b"], state["index"], state["d"], C=state["c"], scales=state["scale"], ranks=state["ranks"])
    return state["d"]


def _to_fp8(x):
    """8-bit values and scales of the 1 x 128 blocks of a 32-bit matrix."""
    rows, cols = x.shape
    pad = torch.nn.functional.pad(x, (0, -cols % 128)).view(rows, -1, 128)
    top = pad.abs().amax(2).clamp_min(LEAST)
    q = (pad * (FP8_MAX / top)[:, :, None]).clamp(-FP8_MAX, FP8_MAX).view(rows, -1)[:, :cols]
    return q.to(torch.float8_e4m3fn), top / FP8_MAX


def _run_plain(state):
    case = state["case"]
    kind = TYPES[case["type"]]
    if case["op"] == "norm":
        out = {}
        h = state["x"]
        if case["residual"]:
            h = out["h"] = (h.float() + state["r"].float()).to(kind)
        h = h.float()
        rstd = (h.square().mean(1) + NORM_EPS).rsqrt()
        y = h * rstd[:, None] * state["w"]
        if case["plain"]:
            out["y"] = y.to(kind)
        out["q"], out["s"] = _to_fp8(y)
        if case["both"]:
            out["qt"], out["st"] = _to_fp8(y.t())
            out["rstd"] = rstd
        return out
    if case["op"] == "norm-backward":
        dy, rstd = state["dy"].float(), state["rstd"][:, None]
        n = state["h"].float() * rstd
        dn = dy * state["w"]
        dx = rstd * (dn - n * (dn * n).mean(1, keepdim=True))
        if case["residual"]:
            dx = dx + state["dr"].float()
        return dx.to(kind), (dy * n).sum(0)
    if case["op"] == "clip":
        total = torch.stack([t.double().square().sum() for t in state["g"]]).sum().sqrt()
        factor = (case["limit"] / (total + CLIP_EPS)).clamp_max(1.0).float()
        return [(t.float() * factor).to(kind) for t in state["g"]], total.float()
    # every token against every adapter, with the products of the others' masked out
    tokens, many, rank = case["tokens"], case["adapters"], case["rank"]
    factor = torch.where(state["index"][:, None] == torch.arange(many, device="cuda"), state["scale"], 0.0)
    low = torch.matmul(state["x"].float(), state["a"].float().view(many * rank, -1).t()).view(tokens, many, rank) * factor[:, :, None]
    delta = torch.matmul(low.view(tokens, many * rank), state["b"].float().transpose(1, 2).reshape(many * rank, -1))
    return (state["c"].float() + delta).to(kind)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------ what a pass is worth
def work(case):
    size = SIZE[case["type"]]
    if case["op"] in ("norm", "norm-backward"):
        rows, cols = case["rows"], case["cols"]
        if case["op"] == "norm-backward":
            return {"bytes": rows * cols * size * (4 if case["residual"] else 3) + 4 * rows + 8 * cols, "flops": 12 * rows * cols}
        moved = size * (3 if case["residual"] else 1) + size * case["plain"] + 1 + case["both"]
        scales = rows * _blocks(cols) + (cols * _blocks(rows) + rows if case["both"] else 0)
        return {"bytes": rows * cols * moved + 4 * scales + 4 * cols, "flops": 8 * rows * cols}
    if case["op"] == "clip":
        many = sum(math.prod(s) for s in _layer_shapes(case))
        return {"bytes": 2 * size * many + 4, "flops": 3 * many}
    tokens, k, n = case["tokens"], case["k"], case["n"]
    ranks = sorted(_ranks(case), reverse=True)[:tokens]      # no more adapters at work than tokens
    weighed = sum(ranks) / len(ranks) * (tokens - tokens // 8 if case["bare"] else tokens)
    return {"bytes": size * (tokens * k + 2 * tokens * n + sum(ranks) * (k + n)) + 4 * tokens, "flops": int(2 * weighed * (k + n))}


# --------------------------------------------------------------------------------------------- the definitions in 64 bits
def _fp8_nearest(v):
    """The e4m3 value nearest to each |v| <= 448 (ties to even): the spacing is 2^(exponent - 3), and 2^-9 below 2^-6."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(v / step) * step


def _exact_blocks(y):
    rows, cols = y.shape
    q = torch.empty_like(y)
    s = torch.empty(rows, _blocks(cols), dtype=torch.float64, device=y.device)
    for j in range(_blocks(cols)):
        part = y[:, 128 * j:128 * (j + 1)]
        s[:, j] = part.abs().amax(1).clamp_min(LEAST) / FP8_MAX
        q[:, 128 * j:128 * (j + 1)] = _fp8_nearest(part / s[:, j:j + 1])
    return q, s


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "norm":
        out = {}
        h = state["x"].double()
        if case["residual"]:
            # the residual stream is what is stored: rounded to its type before the norm reads it
            h = (h + state["r"].double()).float().to(TYPES[case["type"]]).double()
            out["h"] = h
        ms = torch.linalg.vector_norm(h, dim=1) ** 2 / case["cols"]
        y = h / torch.sqrt(ms + NORM_EPS)[:, None] * state["w"].double()
        if case["plain"]:
            out["y"] = y
        out["q"], out["s"] = _exact_blocks(y)
        if case["both"]:
            out["qt"], out["st"] = _exact_blocks(y.t().contiguous())
            out["rstd"] = 1 / torch.sqrt(ms + NORM_EPS)
        return out
    if case["op"] == "norm-backward":
        h, w, dy, rstd = (state[name].double() for name in ("h", "w", "dy", "rstd"))
        # with n = h rstd: dx_j = rstd (w_j dy_j - n_j sum_i(w_i dy_i n_i) / cols)
        inner = torch.einsum("ij,ij,j->i", dy, h, w) * rstd / case["cols"]
        dx = (dy * w - h * (rstd * inner)[:, None]) * rstd[:, None]
        if case["residual"]:
            dx += state["dr"].double()
        return dx, torch.einsum("ij,ij,i->j", dy, h, rstd)
    if case["op"] == "clip":
        total = math.sqrt(math.fsum(float(torch.linalg.vector_norm(t.double())) ** 2 for t in state["g"]))
        factor = min(1.0, case["limit"] / (total + CLIP_EPS))
        return [t.double() * factor for t in state["g"]], torch.tensor(total, dtype=torch.float64, device="cuda")
    d = state["c"].double()
    for a, rank in enumerate(_ranks(case)):
        rows = (state["index"] == a).nonzero()[:, 0]
        low = state["x"][rows].double() @ state["a"][a, :rank].double().t()
        d[rows] += float(state["scale"][a]) * (low @ state["b"][a, :, :rank].double().t())
    return d
