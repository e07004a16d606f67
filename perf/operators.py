"""Operators around one packed projection of a language model, as measured cases.

Kinds (one pass = what `run` does):
  gated          H = act(g) * u with [g; u] = W x: the two projections of a gated feed-forward block packed as one matrix
                 (PackedLinear.gated), with the pre-activations kept where a backward pass follows
  gated_grad     its backward pass: gradients of the pre-activations and of the activations x (PackedLinear.gated_grad)
  adapted        Y = W x + scale_k B_k (A_k x): low-rank adapters of many requests beside the shared projection, the adapter k
                 of every vector chosen by an index on the device (PackedLinear.adapted)
  adapted_grad   gradients of A, B and x, the packed matrix being frozen (PackedLinear.adapted_grad)
  grad           dX = dY W through the packed matrix alone (PackedLinear.grad)

W stands for the first `used` bitlayers of its codes, and x for its fixed-point value Int(x * 2^16) / 2^16 in the product with W (the
adapters take x as it is); gradients pass through Int() unchanged.
"""
import math

import torch

own = False

FRAC = 65536.0
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def listed():
    return [
        # The gate and up projections of a small block, one token: latency. An odd number of column chunks, 4 of 4 bitlayers.
        {"name": "gated one token", "kind": "gated", "cols": 1024, "units": 2730, "bits": 4, "used": 4, "batch": 1, "gate": "silu",
         "keep": False},
        # A step of a serving batch on a wider block, 5 of 8 stored bitlayers read.
        {"name": "gated 24 tokens", "kind": "gated", "cols": 4096, "units": 10922, "bits": 8, "used": 5, "batch": 24, "gate": "silu",
         "keep": False},
        # The same block over a training batch, pre-activations kept for the backward pass.
        {"name": "gated train", "kind": "gated", "cols": 4096, "units": 10922, "bits": 8, "used": 8, "batch": 1024, "gate": "gelu",
         "keep": True},
        # Backward pass of a small block and few tokens: launches, a split of the long sum.
        {"name": "gated_grad small", "kind": "gated_grad", "cols": 1000, "units": 2730, "bits": 4, "used": 4, "batch": 40,
         "gate": "gelu"},
        # Backward pass of the training batch.
        {"name": "gated_grad train", "kind": "gated_grad", "cols": 4096, "units": 10922, "bits": 8, "used": 8, "batch": 1024,
         "gate": "silu"},
        # One token of one request on a small layer.
        {"name": "adapted one token", "kind": "adapted", "rows": 1024, "cols": 1024, "bits": 8, "used": 8, "batch": 1, "count": 4,
         "rank": 8, "type": "bfloat16", "order": "mixed"},
        # A decoding step: 48 requests, 32 adapters, in any order.
        {"name": "adapted decode", "kind": "adapted", "rows": 4096, "cols": 4096, "bits": 8, "used": 8, "batch": 48, "count": 32,
         "rank": 16, "type": "bfloat16", "order": "mixed"},
        # Prompts of several requests in one call, vectors of a request next to each other.
        {"name": "adapted prompts", "kind": "adapted", "rows": 8192, "cols": 4096, "bits": 8, "used": 8, "batch": 2048, "count": 6,
         "rank": 32, "type": "float16", "order": "requests"},
        # Tuning three fp32 adapters on an odd layer.
        {"name": "adapted_grad small", "kind": "adapted_grad", "rows": 1500, "cols": 701, "bits": 5, "used": 5, "batch": 100, "count": 3,
         "rank": 9, "type": "float32", "order": "mixed"},
        # Tuning four adapters at once on a full layer and batch.
        {"name": "adapted_grad train", "kind": "adapted_grad", "rows": 4096, "cols": 4096, "bits": 8, "used": 8, "batch": 2048, "count": 4,
         "rank": 16, "type": "bfloat16", "order": "requests"},
        # The gradient through a frozen layer for a few vectors: the packed matrix once from memory.
        {"name": "grad 4 vectors", "kind": "grad", "rows": 8192, "cols": 8192, "bits": 8, "used": 8, "batch": 4},
        # ... and for a batch: the matrix instructions.
        {"name": "grad batch", "kind": "grad", "rows": 8192, "cols": 8192, "bits": 8, "used": 6, "batch": 768},
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["gated", "gated_grad", "adapted", "adapted_grad", "grad"])
    bits = rng.choice([2, 3, 4, 5, 6, 8, 8, 8, 11])
    case = {"kind": kind, "cols": _spread(rng, 500, 8192), "bits": bits, "used": rng.randint(max(1, bits - 3), bits)}
    if kind.startswith("gated"):
        case["units"] = _spread(rng, 600, 12000)
        case["gate"] = rng.choice(["silu", "gelu", "relu", "sigmoid"])
        rows = 2 * case["units"]
    else:
        case["rows"] = rows = _spread(rng, 500, 12000)
    if kind == "gated":
        case["keep"] = rng.random() < 0.5
    if kind.startswith("adapted"):
        case["count"] = _spread(rng, 1, 48)
        case["rank"] = _spread(rng, 4, 64)
        case["type"] = rng.choice(sorted(TYPES))
        case["order"] = rng.choice(["mixed", "requests"])
    # at most the work of the largest listed case
    case["batch"] = _spread(rng, 1, min(2048, max(2, int(6e10 / (rows * case["cols"])))))
    return case


def _inputs(case, seed):
    """Everything that the seed decides, on the GPU."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, device="cuda", generator=g)   # noqa: E731
    kind, n, cols = case["kind"], case["batch"], case["cols"]
    rows = 2 * case["units"] if kind.startswith("gated") else case["rows"]
    s = {"case": case, "W": normal(rows, cols) * 0.02}
    if kind in ("gated", "adapted", "adapted_grad"):
        s["X"] = normal(n, cols)
    if kind.endswith("grad"):
        # gradients: small, of another size in every vector
        size = 10.0 ** (-5 + 3 * torch.rand((n, 1), device="cuda", generator=g))
        s["dY"] = normal(n, rows // 2 if kind == "gated_grad" else rows) * size
    if kind == "gated_grad":
        s["pre"] = normal(n, rows) * 1.5
    if kind.startswith("adapted"):
        count, rank, dtype = case["count"], case["rank"], TYPES[case["type"]]
        s["A"] = (normal(count, rank, cols) / math.sqrt(cols)).to(dtype)
        s["B"] = (normal(count, rows, rank) * 0.05).to(dtype)
        s["scale"] = 0.5 + torch.rand((count,), device="cuda", generator=g)
        # one vector in ten has no adapter
        index = torch.randint(0, count, (n,), device="cuda", generator=g)
        index = torch.where(torch.rand((n,), device="cuda", generator=g) < 0.1, -1, index).to(torch.int32)
        s["index"] = torch.sort(index).values if case["order"] == "requests" else index
    return s


def _codes(W, bits, used):
    """Codes of the symmetric quantizer without their lowest bits - used bits, and the step between them, in 32 bits."""
    step = W.abs().max() / (2 ** (bits - 1) - 1 if bits > 1 else 1)
    q = torch.round(W / step).clamp(-(2 ** (bits - 1)), 2 ** (bits - 1) - 1)
    drop = 2.0 ** (bits - used)
    return torch.floor(q / drop) * drop, step


def prepare(case, seed):
    s = _inputs(case, seed)
    W = s.pop("W")
    if own:
        from paper_2003_00822_amd import pb
        # a gated layer of an even number of units has the layout that the block's single launch takes
        layout = pb.PB_LAYOUT_TILE16_GATES_V1 if case.get("units", 1) % 2 == 0 else None
        # (packed from the quantized matrix: a weight half way between two codes must not depend on how the step was rounded)
        codes, step = _codes(W, case["bits"], case["bits"])
        s["layer"] = pb.PackedLinear(codes * step, case["bits"], max_batch=case["batch"], layout=layout)
        if "A" in s:
            s["adapters"] = pb.Adapters(s["A"], s["B"], s["scale"])
        if "gate" in case:
            s["gate"] = {"sigmoid": pb.PB_GATE_SIGMOID, "silu": pb.PB_GATE_SILU, "gelu": pb.PB_GATE_GELU,
                         "relu": pb.PB_GATE_RELU}[case["gate"]]
    else:
        s["codes"], s["step"] = _codes(W, case["bits"], case["used"])
    return s


# ---- the plain forms ----
def _fixed(X):
    return torch.trunc((X * FRAC).clamp(-2147483648.0, 2147483520.0)) / FRAC


def _act(gate, v):
    """The activation and its derivative."""
    if gate == "relu":
        return torch.where(v > 0, v, torch.zeros_like(v)), (v > 0).to(v.dtype)
    if gate == "gelu":
        k = math.sqrt(8.0 / math.pi)
        s = 1.0 / (1.0 + torch.exp(-k * (v + 0.044715 * v * v * v)))
        return v * s, s + v * s * (1.0 - s) * k * (1.0 + 3 * 0.044715 * v * v)
    s = 1.0 / (1.0 + torch.exp(-v))
    if gate == "sigmoid":
        return s, s * (1.0 - s)
    return v * s, s * (1.0 + v * (1.0 - s))


def _adapters_of(s):
    """A [count * rank, cols], B [rows, count * rank] in 32 bits, and per vector scale_k on the ranks of its adapter k, 0 on the others."""
    A, B, scale, index = s["A"].float(), s["B"].float(), s["scale"], s["index"]
    count, rank = A.shape[:2]
    mine = index[:, None] == torch.arange(count, device=index.device, dtype=index.dtype)[None, :]
    weight = torch.where(mine, scale[None, :], torch.zeros_like(scale)[None, :]).repeat_interleave(rank, dim=1)
    return A.reshape(count * rank, -1), B.permute(1, 0, 2).reshape(B.shape[1], -1), weight


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        layer, used = s["layer"], case["used"]
        if kind == "gated":
            return layer.gated(s["X"], s["gate"], used, keep=case["keep"])
        if kind == "gated_grad":
            return layer.gated_grad(s["pre"], s["dY"], s["gate"], used)
        if kind == "adapted":
            return layer.adapted(s["X"], s["adapters"], s["index"], used)
        if kind == "adapted_grad":
            return layer.adapted_grad(s["X"], s["dY"], s["adapters"], s["index"], used)
        return layer.grad(s["dY"], used)
    codes, step = s["codes"], s["step"]
    if kind == "gated":
        pre = torch.matmul(_fixed(s["X"]), codes.t()) * step
        F = case["units"]
        H = _act(case["gate"], pre[:, :F])[0] * pre[:, F:]
        return (H, pre) if case["keep"] else H
    if kind == "gated_grad":
        F = case["units"]
        g, u = s["pre"][:, :F], s["pre"][:, F:]
        a, da = _act(case["gate"], g)
        dpre = torch.cat([s["dY"] * u * da, s["dY"] * a], dim=1)
        return torch.matmul(dpre, codes) * step, dpre
    if kind == "grad":
        return torch.matmul(s["dY"], codes) * step
    A, B, weight = _adapters_of(s)
    if kind == "adapted":
        Y = torch.matmul(_fixed(s["X"]), codes.t()) * step
        return Y + torch.matmul(torch.matmul(s["X"], A.t()) * weight, B.t())
    count, rank = s["A"].shape[:2]
    u = torch.matmul(s["X"], A.t()) * weight
    t = torch.matmul(s["dY"], B) * weight
    dX = torch.matmul(s["dY"], codes) * step + torch.matmul(t, A)
    dA = torch.matmul(t.t(), s["X"]).reshape(s["A"].shape)
    dB = torch.matmul(s["dY"].t(), u).reshape(-1, count, rank).permute(1, 0, 2).contiguous()
    return dX, dA, dB


def work(case):
    kind, n, cols = case["kind"], case["batch"], case["cols"]
    rows = 2 * case["units"] if kind.startswith("gated") else case["rows"]
    nbytes = rows * cols * case["used"] / 8
    flops = 2.0 * n * rows * cols
    if kind == "gated":
        nbytes += 4.0 * n * (cols + rows / 2 + (rows if case["keep"] else 0))
    elif kind == "gated_grad":
        nbytes += 4.0 * n * (rows / 2 + rows + rows + cols)
    elif kind == "grad":
        nbytes += 4.0 * n * (rows + cols)
    else:
        size = {"float32": 4, "bfloat16": 2, "float16": 2}[case["type"]]
        per = case["rank"] * (rows + cols)          # values of an adapter
        nbytes += size * per * min(case["count"], n) + 4.0 * n * (cols + rows)
        flops += 2.0 * n * per
        if kind == "adapted_grad":
            nbytes += 4.0 * n * cols + 4.0 * per * case["count"]
            flops += 4.0 * n * per
    return {"bytes": nbytes, "flops": flops}


def exact(case, seed):
    """The definitions in 64 bits: the bitlayers one by one, every vector's own adapter."""
    s = _inputs(case, seed)
    bits, used = case["bits"], case["used"]
    W = s["W"]
    step = W.abs().max() / (2 ** (bits - 1) - 1 if bits > 1 else 1)
    q = torch.round(W / step).to(torch.int32).clamp(-(1 << (bits - 1)), (1 << (bits - 1)) - 1)
    layers = torch.zeros(W.shape, dtype=torch.float64, device=W.device)
    for i in range(used):
        weight = -(2.0 ** (bits - 1)) if i == 0 else 2.0 ** (bits - 1 - i)
        layers += weight * ((q >> (bits - 1 - i)) & 1).double()
    W = layers * step.double()
    kind = case["kind"]
    if "X" in s:
        X = s["X"].double()
        Xq = (X * FRAC).to(torch.int64).clamp(-(1 << 31), (1 << 31) - 1).double() / FRAC
    if "dY" in s:
        dY = s["dY"].double()
    if kind == "grad":
        return torch.matmul(dY, W)
    if kind.startswith("gated"):
        F, gate = case["units"], case["gate"]
        pre = torch.matmul(Xq, W.t()) if kind == "gated" else s["pre"].double()
        v, u = pre[:, :F], pre[:, F:]
        if gate == "relu":
            a, da = v.clamp(min=0), (v > 0).double()
        elif gate == "gelu":
            inner = math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)
            a = 0.5 * v * (1 + torch.tanh(inner))
            da = 0.5 * (1 + torch.tanh(inner)) + 0.5 * v * torch.cosh(inner) ** -2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * v ** 2)
        else:
            sig = torch.special.expit(v)
            a, da = (sig, sig * (1 - sig)) if gate == "sigmoid" else (v * sig, sig + v * sig * (1 - sig))
        if kind == "gated":
            return (a * u, pre) if case["keep"] else a * u
        dpre = torch.cat([dY * u * da, dY * a], dim=1)
        return torch.matmul(dpre, W), dpre
    A, B, scale, index = s["A"].double(), s["B"].double(), s["scale"].double(), s["index"].long()
    Y = torch.matmul(Xq, W.t())
    if kind == "adapted_grad":
        dX, dA, dB = torch.matmul(dY, W), torch.zeros_like(A), torch.zeros_like(B)
    for k in range(case["count"]):
        rows = torch.nonzero(index == k)[:, 0]
        x = X[rows]
        u = torch.matmul(x, A[k].t())
        if kind == "adapted":
            Y[rows] += scale[k] * torch.matmul(u, B[k].t())
            continue
        dy = dY[rows]
        t = scale[k] * torch.matmul(dy, B[k])
        dX[rows] += torch.matmul(t, A[k])
        dA[k] = torch.matmul(t.t(), x)
        dB[k] = scale[k] * torch.matmul(dy.t(), u)
    return Y if kind == "adapted" else (dX, dA, dB)
