"""The calls of a decoder layer in 8 bits whose speed is watched: the root mean square norm with the residual's addition, its
gradient, rows and weights into 8 bits with a scale for each block of 128 (behind a gate, too), and the product of such operands.
`listed` names them, `draw` gives more of the same ranges, `prepare` makes what a program holds before the call, `run` is the
call itself: the package's entry points where `own` is true, else the same in elementary torch operations.  `exact` computes it in 64
bits from the definition."""
from __future__ import annotations

import torch

own = False

DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "fp16": 2, "bf16": 2}
E4M3_MOST = 448.0
LEAST_SCALE = 2.0 ** -126
BLOCK = 128
EPS = 1e-6


def listed():
    return [
        # One decoder step in front of a product in 8 bits: the residual stream of a small batch (launch latency is what it costs).
        dict(name="norm_step", kind="norm", dtype="bf16", tokens=16, heads=0, dim=4096, residual=True, eight=True),
        # Queries and keys of a prompt inside their projection, each head by itself.
        dict(name="norm_heads", kind="norm", dtype="bf16", tokens=4111, heads=40, dim=128, residual=False, eight=False),
        # Prompts of a serving queue, an odd number of tokens: the residual stream goes on, its norm into 8 bits.
        dict(name="norm_prompt", kind="norm", dtype="bf16", tokens=16391, heads=0, dim=4096, residual=True, eight=True),
        # The gradient at training batch, what reaches the residual stream by other ways added.
        dict(name="grad_batch", kind="grad", dtype="bf16", tokens=16384, heads=0, dim=4096, extra=True),
        # The gradient of a small 32-bit run, rows of no whole 16 bytes.
        dict(name="grad_odd", kind="grad", dtype="fp32", tokens=1531, heads=0, dim=1001, extra=False),
        # Attention's output in front of its projection, one decoder step.
        dict(name="quantize_step", kind="quantize", dtype="bf16", rows=64, dim=2560, gate=False, tall=1),
        # Between the two products of a gated layer, prompts.
        dict(name="quantize_gate", kind="quantize", dtype="bf16", rows=8192, dim=10240, gate=True, tall=1),
        # A weight laid out, once a model is loaded: odd sizes, so that blocks at the edges are not whole.
        dict(name="quantize_weight", kind="quantize", dtype="bf16", rows=6100, dim=4080, gate=False, tall=128),
        # One request's token: the weight is streamed once.
        dict(name="gemm_one", kind="gemm", tokens=1, features=4096, k=4096, out="bf16"),
        # A decoder step of a batch through the projection of 32 + 2 * 8 heads of 128.
        dict(name="gemm_step", kind="gemm", tokens=64, features=6144, k=4096, out="bf16"),
        # A short prompt, odd in everything, the logits in 32 bits.
        dict(name="gemm_odd", kind="gemm", tokens=389, features=5003, k=2576, out="fp32"),
        # Prompts of a serving queue: what the matrix cores can do.
        dict(name="gemm_prompt", kind="gemm", tokens=16384, features=4096, k=8192, out="bf16"),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "grad", "quantize", "gemm", "gemm", "gemm"])
    while True:
        if kind in ("norm", "grad"):
            heads = rng.choice([0, 0, 0, 1, 5, 16, 40])
            c = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), tokens=_log(rng, 1, 65536), heads=heads,
                     dim=rng.choice([40, 64, 80, 96, 128, 128, 256]) if heads else rng.choice([_log(rng, 1, 20000), 8 * _log(rng, 8, 2048), 128 * _log(rng, 4, 128)]))
            if kind == "norm":
                c["residual"] = not heads and rng.random() < 0.6
                c["eight"] = not heads and rng.random() < 0.6
            else:
                c["extra"] = rng.random() < 0.5
            if work(c)["bytes"] <= 5e8:
                return c
        elif kind == "quantize":
            c = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), rows=_log(rng, 1, 65536), dim=rng.choice([_log(rng, 1, 30000), 128 * _log(rng, 1, 200)]),
                     gate=False, tall=rng.choice([1, 1, 128]))
            c["gate"] = c["tall"] == 1 and rng.random() < 0.5
            if work(c)["bytes"] <= 4e8:
                return c
        else:
            c = dict(kind=kind, tokens=rng.choice([_log(rng, 1, 64), _log(rng, 1, 512), _log(rng, 64, 16384)]), features=rng.choice([_log(rng, 1, 20000), 64 * _log(rng, 4, 256)]),
                     k=16 * rng.choice([_log(rng, 1, 1024), 8 * _log(rng, 2, 128)]), out=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
            w = work(c)
            if w["flops"] <= 1.0e12 and w["bytes"] <= 5e8:
                return c


def _blocks(n):
    return -(-n // BLOCK)


def work(case):
    kind = case["kind"]
    if kind == "gemm":
        m, n, k = case["tokens"], case["features"], case["k"]
        return {"bytes": m * k + n * k + m * n * BYTES[case["out"]] + 4 * _blocks(k) * (m + _blocks(n)), "flops": 2 * m * n * k}
    e = BYTES[case["dtype"]]
    if kind == "quantize":
        n = case["rows"] * case["dim"]
        return {"bytes": n * e * (2 if case["gate"] else 1) + n + 4 * _blocks(case["dim"]) * -(-case["rows"] // case["tall"]), "flops": n * (8 if case["gate"] else 3)}
    rows, d = case["tokens"] * max(1, case["heads"]), case["dim"]
    n = rows * d
    if kind == "grad":
        return {"bytes": n * e * (4 if case["extra"] else 3) + d * (e + 4), "flops": 10 * n}
    moved = n * e * (3 if case["residual"] else 1) + (n + 4 * rows * _blocks(d) if case["eight"] else n * e)
    return {"bytes": moved + d * e, "flops": 6 * n}


# ---- inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(shape, dt, g, std=1.0):
    """Values as a residual stream has them: some channels much larger than the others."""
    x = torch.empty(shape, dtype=dt, device="cuda")
    gain = std * torch.exp(0.5 * torch.randn(shape[-1], device="cuda", generator=g))
    flat = x.view(-1, shape[-1])
    step = max(1, (1 << 27) // shape[-1])   # in parts: 32-bit values of the whole would take more room than the rows
    for i in range(0, flat.size(0), step):
        part = flat[i:i + step]
        part.copy_(torch.randn(part.shape, device="cuda", generator=g).mul_(gain))
    return x


def _in_eight_bits(x, tall):
    """x [rows, k] as the product takes it: e4m3 and a scale for each tall x 128 block, scales of one block beside one another."""
    rows, k = x.shape
    q = torch.empty((rows, k), dtype=torch.float8_e4m3fn, device="cuda")
    scale = torch.empty((_blocks(k), -(-rows // tall)), dtype=torch.float32, device="cuda")
    step = max(tall, (1 << 26) // k // tall * tall)
    for i in range(0, rows, step):
        part = x[i:i + step].float()
        q[i:i + step], scale[:, i // tall:-(-(i + part.size(0)) // tall)] = _blockwise(part, tall)
    return q, scale.t()


def prepare(case, seed):
    g = _generator(seed)
    kind, state = case["kind"], {"case": case}
    if kind == "gemm":
        m, n, k = case["tokens"], case["features"], case["k"]
        state["a"], state["a_scale"] = _in_eight_bits(_rows((m, k), torch.bfloat16, g), 1)
        weight = torch.empty((n, k), dtype=torch.bfloat16, device="cuda").normal_(0.0, k ** -0.5, generator=g)
        state["w"], state["w_scale"] = _in_eight_bits(weight, BLOCK)
        return state
    dt = DTYPES[case["dtype"]]
    if kind == "quantize":
        if case["gate"]:   # both come out of one product
            both = _rows((case["rows"], 2 * case["dim"]), dt, g)
            state.update(gate=both[:, :case["dim"]], x=both[:, case["dim"]:])
        else:
            state["x"] = _rows((case["rows"], case["dim"]), dt, g, 0.02 if case["tall"] > 1 else 1.0)
        return state
    d = case["dim"]
    if case["heads"]:
        # the heads inside a packed projection that holds others behind them
        x = _rows((case["tokens"], case["heads"] + max(1, case["heads"] // 4), d), dt, g)[:, :case["heads"]]
    else:
        x = _rows((case["tokens"], d), dt, g)
    state.update(x=x, weight=(1.0 + 0.2 * torch.randn(d, device="cuda", generator=g)).to(dt))
    if kind == "grad":
        state["grad"] = _rows(tuple(x.shape), dt, g, 0.01)
        if case["extra"]:
            state["extra"] = _rows(tuple(x.shape), dt, g, 0.01)
    elif case["residual"]:
        state["residual"] = _rows((case["tokens"], d), dt, g, 3.0)
    return state


# ---- the plain forms

def _blockwise(x, tall):
    """x [rows, k] in 32 bits -> e4m3 values, scales [blocks of k, blocks of rows]."""
    rows, k = x.shape
    down, across = -(-rows // tall), _blocks(k)
    y = torch.nn.functional.pad(x, (0, across * BLOCK - k, 0, down * tall - rows)).view(down, tall, across, BLOCK)
    scale = (y.abs().amax((1, 3)) / E4M3_MOST).clamp(min=LEAST_SCALE)
    q = (y / scale[:, None, :, None]).clamp(-E4M3_MOST, E4M3_MOST).view(down * tall, across * BLOCK)[:rows, :k].to(torch.float8_e4m3fn)
    return q, scale.t()


def _norm(s):
    x = s["x"]
    h = x if "residual" not in s else (x.float() + s["residual"].float()).to(x.dtype)
    f = h.float()
    y = f * torch.rsqrt((f * f).sum(-1, keepdim=True) / f.size(-1) + EPS) * s["weight"].float()
    made = {"total": h} if "residual" in s else {}
    if not s["case"]["eight"]:
        return {"out": y.to(x.dtype), **made}
    q, scale = _blockwise(y, 1)
    return {"out": q, "scale": scale.t(), **made}


def _grad(s):
    h, g, w = s["x"].float(), s["grad"].float(), s["weight"].float()
    r = torch.rsqrt((h * h).sum(-1, keepdim=True) / h.size(-1) + EPS)
    gw = g * w
    c = (gw * h).sum(-1, keepdim=True)
    dx = r * (gw - h * (r * r * c / h.size(-1)))
    if "extra" in s:
        dx = dx + s["extra"].float()
    return {"x": dx.to(s["x"].dtype), "weight": (g * h * r).reshape(-1, h.size(-1)).sum(0)}


def _quantize(s):
    x = s["x"].float()
    if "gate" in s:
        gate = s["gate"].float()
        x = gate / (1.0 + torch.exp(-gate)) * x
    q, scale = _blockwise(x, s["case"]["tall"])
    return {"out": q, "scale": scale.t()}


def _gemm(s):
    a, w = s["a"].float(), s["w"].float()
    k = a.size(1)
    a = a * s["a_scale"].repeat_interleave(BLOCK, 1)[:, :k]
    w = w * s["w_scale"].repeat_interleave(BLOCK, 0)[:w.size(0)].repeat_interleave(BLOCK, 1)[:, :k]
    return torch.matmul(a, w.t()).to(DTYPES[s["case"]["out"]])


# ---- the framework's own

def run(state):
    s, kind = state, state["case"]["kind"]
    if not own:
        return {"norm": _norm, "grad": _grad, "quantize": _quantize, "gemm": _gemm}[kind](s)
    from paper_2002_12798_amd import device
    if kind == "norm":
        y = device.norm(s["x"], s["weight"], EPS, residual=s.get("residual"), eight=s["case"]["eight"])
        return {"out": y.out, **({"scale": y.scale} if s["case"]["eight"] else {}), **({"total": y.total} if "residual" in s else {})}
    if kind == "grad":
        dx, dw = device.norm_grad(s["x"], s["weight"], s["grad"], EPS, extra=s.get("extra"))
        return {"x": dx, "weight": dw}
    if kind == "quantize":
        y = device.quantize(s["x"], gate=s.get("gate"), tall=s["case"]["tall"])
        return {"out": y.out, "scale": y.scale}
    return device.gemm_scaled(s["a"], s["a_scale"], s["w"], s["w_scale"], dtype=DTYPES[s["case"]["out"]])


# ---- in 64 bits, from the definitions

def _values64(y, tall):
    """y [rows, k] -> y over its block's scale (not rounded to 8 bits), and the scales [blocks of rows, blocks of k]."""
    rows, k = y.shape
    scale = torch.empty((-(-rows // tall), _blocks(k)), dtype=torch.float64, device=y.device)
    out = torch.empty_like(y)
    for b in range(_blocks(k)):
        cols = slice(b * BLOCK, min(k, (b + 1) * BLOCK))
        top = y[:, cols].abs().amax(1)
        if tall > 1:
            top = torch.stack([top[i:i + tall].amax() for i in range(0, rows, tall)])
        scale[:, b] = torch.clamp(top / E4M3_MOST, min=LEAST_SCALE)
        out[:, cols] = y[:, cols] / torch.repeat_interleave(scale[:, b], tall)[:rows, None]
    return out, scale


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "gemm":
        m, n, k = case["tokens"], case["features"], case["k"]
        if 2.0 * m * n * k > 2e13:
            return None
        out = torch.zeros((m, n), dtype=torch.float64, device="cuda")
        row = torch.arange(n, device="cuda") // BLOCK
        for b in range(_blocks(k)):
            cols = slice(b * BLOCK, min(k, (b + 1) * BLOCK))
            part = s["a"][:, cols].double() @ s["w"][:, cols].double().t().contiguous()
            out += part * s["a_scale"][:, b].double()[:, None] * s["w_scale"][row, b].double()[None, :]
        return out
    if kind == "quantize":
        y = s["x"].double()
        if case["gate"]:
            y = y * s["gate"].double() * torch.sigmoid(s["gate"].double())
        q, scale = _values64(y, case["tall"])
        return {"out": q, "scale": scale}
    x, w = s["x"].double(), s["weight"].double()
    if kind == "grad":
        g = s["grad"].double()
        n = case["dim"]
        r = 1.0 / torch.sqrt(x.square().mean(-1) + EPS)[..., None]
        z = x * r   # (dz of it goes through the row's norm: what lies along z is taken out, but for eps)
        dz = g * w
        dx = r * (dz - z * (dz * z).sum(-1, keepdim=True) / n)
        dw = (g * z).flatten(0, -2).sum(0)
        return {"x": dx + s["extra"].double() if case["extra"] else dx, "weight": dw}
    made = {}
    if case["residual"]:
        made["total"] = x + s["residual"].double()
        x = made["total"].to(s["x"].dtype).double()   # the norm is of what goes on as the residual stream
    y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * w
    if not case["eight"]:
        return {"out": y, **made}
    q, scale = _values64(y, 1)
    return {"out": q, "scale": scale, **made}
