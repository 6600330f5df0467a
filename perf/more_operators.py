"""The operators of an encoder's feed-forward half, case by case: rows of a dense table looked up with a scale and
their gradient by sorted ids, root-mean-square norms after and before a block fused with its gate and residual, and
products with bias, activation and residual (``paper_2207_10731_gb300.sequence``), each with its plain form in
elementary torch operations and its definition in 64 bits.

Sizes are the embedding's own (rows of 16, 64 or 128 values, 26 tables and their concatenated row of 3328, batches
of 16384 and 65536) or generic ones.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5


def listed():
    return [
        # one token served: the weight is all that moves, latency counts
        {"name": "linear serving token", "op": "linear", "direction": "forward", "tokens": 1, "in": 4096, "out": 4096,
         "type": "bf16", "activation": "silu", "bias": True, "residual": False, "keep": False, "dense": "out",
         "gap": 0},
        # odd in every size, cut out of wider rows, with all that an epilogue can do
        {"name": "linear odd cut-out", "op": "linear", "direction": "forward", "tokens": 1001, "in": 333, "out": 517,
         "type": "f16", "activation": "gelu", "bias": True, "residual": True, "keep": True, "dense": "in", "gap": 5},
        # the product back onto the residual stream of a long batch
        {"name": "linear onto residual", "op": "linear", "direction": "forward", "tokens": 16384, "in": 4096,
         "out": 4096, "type": "bf16", "activation": None, "bias": True, "residual": True, "keep": False,
         "dense": "in", "gap": 0},
        # gradients of a feed-forward block's first product
        {"name": "linear backward feed-forward", "op": "linear", "direction": "backward", "tokens": 16384, "in": 1024,
         "out": 4096, "type": "bf16", "activation": "gelu", "bias": True, "residual": False, "keep": False,
         "dense": "out", "gap": 0},
        # gradients of the product that reads the concatenated row of all 26 tables: few outputs, a long sum over tokens
        {"name": "linear backward concatenated", "op": "linear", "direction": "backward", "tokens": 65536,
         "in": 26 * 128, "out": 512, "type": "bf16", "activation": "relu", "bias": True, "residual": False,
         "keep": False, "dense": "in", "gap": 0},
        # the newest items of eight users between two blocks: latency counts
        {"name": "norm serving rows", "op": "norm", "direction": "forward", "rows": 8, "cols": 1024, "type": "bf16",
         "stream": "bf16", "post": True, "pre": True, "gate": "none", "scale": 1.0, "gap": 0},
        # a long batch between two blocks, residual stream in 32 bits, gated value by value
        {"name": "norm gated long", "op": "norm", "direction": "forward", "rows": 131072, "cols": 1024, "type": "bf16",
         "stream": "f32", "post": True, "pre": True, "gate": "values", "scale": 0.5, "gap": 0},
        # its gradients on a 16-bit stream, with both weights' sums
        {"name": "norm backward gated", "op": "norm", "direction": "backward", "rows": 65536, "cols": 2048,
         "type": "bf16", "stream": "bf16", "post": True, "pre": True, "gate": "values", "scale": 0.5, "gap": 0},
        # an odd width, one gate to a token
        {"name": "norm backward odd width", "op": "norm", "direction": "backward", "rows": 40001, "cols": 333,
         "type": "f16", "stream": "f32", "post": True, "pre": True, "gate": "tokens", "scale": 1.0, "gap": 0},
        # every id of a Criteo-TB-shaped batch looked up in one dense table, popular ids first
        {"name": "embedding lookup batch", "op": "embedding", "direction": "forward", "tokens": 65536 * 26,
         "rows": 1000003, "cols": 128, "type": "f32", "to": "bf16", "skew": 3, "padding": 0.0, "scale": 11.5},
        # its gradient: a few ids carry a large part of the batch
        {"name": "embedding gradient batch", "op": "embedding", "direction": "backward", "tokens": 65536 * 26,
         "rows": 1000003, "cols": 128, "type": "f32", "to": "f32", "skew": 3, "padding": 0.0, "scale": 11.5},
        # a short padded batch into a vocabulary: most rows get nothing
        {"name": "embedding gradient vocabulary", "op": "embedding", "direction": "backward", "tokens": 2011,
         "rows": 50021, "cols": 1024, "type": "bf16", "to": "f32", "skew": 3, "padding": 0.1, "scale": 32.0},
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "norm", "embedding"])
    if op == "linear":
        case = {"op": op, "direction": rng.choice(["forward", "backward"]), "type": rng.choice(["bf16", "f16"]),
                "activation": rng.choice([None, "relu", "gelu", "silu"]), "bias": rng.random() < 0.75}
        for side in ("in", "out"):
            case[side] = rng.choice([64, 128, 512, 26 * 128, _between(rng, 8, 8192), _between(rng, 8, 8192)])
        most = 2**36 // (case["in"] * case["out"])
        case["tokens"] = _between(rng, 1, max(2, min(65536, most)))
        forward = case["direction"] == "forward"
        return dict(case, residual=forward and rng.random() < 0.5,
                    keep=forward and case["activation"] is not None and rng.random() < 0.5,
                    dense=rng.choice(["in", "out"]), gap=rng.choice([0, 0, 8, 5]))
    if op == "norm":
        cols = rng.choice([64, 128, 512, 26 * 128, _between(rng, 12, 8192), _between(rng, 12, 8192)])
        kind = rng.choice(["f32", "bf16", "f16"])
        post, pre = rng.choice([(True, True), (True, True), (False, True), (True, False)])
        return {"op": op, "direction": rng.choice(["forward", "backward"]), "cols": cols,
                "rows": _between(rng, 1, max(2, min(262144, 2**26 // cols))), "type": kind,
                "stream": rng.choice(["f32", kind]), "post": post, "pre": pre,
                "gate": rng.choice(["none", "values", "tokens"]), "scale": rng.choice([1.0, 0.5, 0.1]),
                "gap": rng.choice([0, 0, 8, 13])}
    cols = rng.choice([16, 64, 128, 512, _between(rng, 8, 4096), _between(rng, 8, 4096)])
    return {"op": op, "direction": rng.choice(["forward", "backward"]), "cols": cols,
            "tokens": _between(rng, 1, max(2, min(65536 * 26, 2**27 // cols))),
            "rows": _between(rng, 16, max(32, min(2**20, 2**27 // cols))), "type": rng.choice(["f32", "bf16", "f16"]),
            "to": rng.choice(["f32", "bf16", "f16"]), "skew": rng.choice([1, 3]), "padding": rng.choice([0.0, 0.1]),
            "scale": rng.choice([1.0, 11.5])}


def _normal(gen, *size, dtype=torch.float32, scale=1.0):
    return (torch.randn(*size, generator=gen, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _rows(gen, rows, cols, gap, dtype):
    """Normal rows, cut out of rows that are ``gap`` values wider."""
    return _normal(gen, rows, cols + gap, dtype=dtype)[:, :cols]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    state = dict(case)
    kind = TYPES[case["type"]]
    if case["op"] == "linear":
        tokens, n, m, gap = case["tokens"], case["in"], case["out"], case["gap"]
        state["x"] = _rows(gen, tokens, n, gap, kind)
        weight = _normal(gen, n, m, dtype=kind, scale=n ** -0.5)
        state["weight"] = weight if case["dense"] == "out" else weight.t().contiguous().t()
        state["bias_values"] = _normal(gen, m, scale=0.2) if case["bias"] else None
        if case["residual"]:
            state["residual_rows"] = _rows(gen, tokens, m, gap, kind)
        if case["direction"] == "backward":  # with what the forward pass kept
            state["grad"] = _rows(gen, tokens, m, gap, kind)
            if case["activation"]:
                z = state["x"].float() @ state["weight"].float()
                state["z"] = (z + state["bias_values"] if case["bias"] else z).to(kind)
        return state
    if case["op"] == "norm":
        rows, cols, gap, wide = case["rows"], case["cols"], case["gap"], TYPES[case["stream"]]
        size = 0.5 + torch.rand(rows, 1, generator=gen, device="cuda")
        state["x"] = _rows(gen, rows, cols, gap, torch.float32).mul_(size).to(kind)
        if gap:
            state["x"] = torch.nn.functional.pad(state["x"], (0, gap))[:, :cols]
        residual = _rows(gen, rows, cols, gap, wide)
        if case["gate"] != "none":  # logits
            state["gate_values"] = _normal(gen, rows, cols if case["gate"] == "values" else 1, dtype=kind)
        if case["post"]:
            state["post_weight"] = 1 + _normal(gen, cols, scale=0.2)
        if case["pre"]:
            state["pre_weight"] = 1 + _normal(gen, cols, scale=0.2)
        if case["direction"] == "forward":
            state["residual"] = residual
            return state
        # the stream after the block and the norms' scales, as the forward pass kept them
        state["total"] = residual
        if case["post"]:
            state["post_rstd"] = (state["x"].float().square().mean(1) + EPS).rsqrt()
        if case["pre"]:
            state["pre_rstd"] = (residual.float().square().mean(1) + EPS).rsqrt()
            state["grad_y"] = _normal(gen, rows, cols, dtype=kind)
        state["grad_total"] = _normal(gen, rows, cols, dtype=wide)
        return state
    tokens, rows, cols = case["tokens"], case["rows"], case["cols"]
    place = torch.rand(tokens, generator=gen, device="cuda", dtype=torch.float64)
    ids = (place ** case["skew"] * rows).long().clamp_(max=rows - 1)
    hidden = torch.rand(tokens, generator=gen, device="cuda") < case["padding"]
    state["ids"] = ids.masked_fill_(hidden, -1)
    if case["direction"] == "forward":
        state["weight"] = _normal(gen, rows, cols, dtype=kind)
    else:
        state["grad"] = _normal(gen, tokens, cols, dtype=kind)
    return state


# ---- plain forms ---------------------------------------------------------------------------------------------------


def _act(z, name):
    if name == "relu":
        return z * (z > 0)
    if name == "gelu":
        return 0.5 * z * torch.erfc(-math.sqrt(0.5) * z)
    return z / (1 + torch.exp(-z)) if name == "silu" else z


def _act_slope(z, name):
    if name == "relu":
        return (z > 0).float()
    if name == "gelu":
        return 0.5 * torch.erfc(-math.sqrt(0.5) * z) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s))


def _linear_forward(s):
    kind = TYPES[s["type"]]
    z = s["x"].float() @ s["weight"].float()
    if s["bias"]:
        z = z + s["bias_values"]
    y = _act(z, s["activation"])
    if s["residual"]:
        y = y + s["residual_rows"].float()
    return (y.to(kind), z.to(kind)) if s["keep"] else y.to(kind)


def _linear_backward(s):
    kind, g = TYPES[s["type"]], s["grad"].float()
    if s["activation"]:
        g = g * _act_slope(s["z"].float(), s["activation"])
    dx, dweight = g @ s["weight"].float().t(), s["x"].float().t() @ g
    return dx.to(kind), dweight.to(kind), g.sum(0, dtype=torch.float64).float()


def _norm_forward(s):
    u, answer = s["x"].float(), []
    if s["post"]:
        post = 1 / torch.sqrt((u * u).mean(1, keepdim=True) + EPS)
        u = u * post * s["post_weight"]
    if s["gate"] != "none":
        u = u / (1 + torch.exp(-s["gate_values"].float()))
    total = s["residual"].float() + s["scale"] * u
    answer.append(total.to(s["residual"].dtype))
    if s["pre"]:
        pre = 1 / torch.sqrt((total * total).mean(1, keepdim=True) + EPS)
        answer.append((total * pre * s["pre_weight"]).to(s["x"].dtype))
    return answer + ([post[:, 0]] if s["post"] else []) + ([pre[:, 0]] if s["pre"] else [])


def _norm_backward(s):
    kind, d = s["x"].dtype, s["grad_total"].float()
    weights = []
    if s["pre"]:
        rstd = s["pre_rstd"][:, None]
        hat, g = s["total"].float() * rstd, s["grad_y"].float()
        weights.append((g * hat).sum(0, dtype=torch.float64).float())
        g = g * s["pre_weight"]
        d = d + (g - hat * (g * hat).mean(1, keepdim=True)) * rstd
    answer = [d.to(s["total"].dtype)]
    x, du = s["x"].float(), d * s["scale"]
    hat = x * s["post_rstd"][:, None] if s["post"] else x
    if s["gate"] != "none":
        open_ = 1 / (1 + torch.exp(-s["gate_values"].float()))
        u = hat * s["post_weight"] if s["post"] else hat
        dgate = du * u * open_ * (1 - open_)
        answer.append((dgate if s["gate"] == "values" else dgate.sum(1, keepdim=True)).to(kind))
        du = du * open_
    if s["post"]:
        weights.insert(0, (du * hat).sum(0, dtype=torch.float64).float())
        g = du * s["post_weight"]
        du = (g - hat * (g * hat).mean(1, keepdim=True)) * s["post_rstd"][:, None]
    return [du.to(kind)] + answer + weights


def _embedding_forward(s):
    inside = s["ids"] >= 0
    y = s["weight"][s["ids"].clamp(min=0)].float() * s["scale"]
    return (y * inside[:, None]).to(TYPES[s["to"]])


def _embedding_backward(s):
    """In 64 bits: a popular id's sum is long."""
    inside = s["ids"] >= 0
    sums = torch.zeros(s["rows"], s["cols"], dtype=torch.float64, device="cuda")
    sums.index_add_(0, s["ids"][inside], s["grad"][inside].double())
    return (sums * s["scale"]).to(TYPES[s["to"]])


# ---- one pass ------------------------------------------------------------------------------------------------------


def run(state):
    s = state
    forward = s["direction"] == "forward"
    if not own:
        if s["op"] == "linear":
            return _linear_forward(s) if forward else _linear_backward(s)
        if s["op"] == "norm":
            return _norm_forward(s) if forward else _norm_backward(s)
        return _embedding_forward(s) if forward else _embedding_backward(s)
    from paper_2207_10731_gb300 import sequence

    if s["op"] == "linear":
        if forward:
            return sequence.linear_forward(s["x"], s["weight"], s["bias_values"], activation=s["activation"],
                                           residual=s.get("residual_rows"), keep=s["keep"])
        return sequence.linear_backward(s["grad"], s["x"], s["weight"], z=s.get("z"), activation=s["activation"])
    if s["op"] == "norm":
        more = {"post_weight": s.get("post_weight"), "pre_weight": s.get("pre_weight"), "gate": s.get("gate_values"),
                "scale": s["scale"]}
        if forward:
            answer = sequence.residual_norm_forward(s["x"], s["residual"], eps=EPS, **more)
        else:
            answer = sequence.residual_norm_backward(s["grad_total"], s.get("grad_y"), s["x"], s["total"],
                                                     s.get("post_rstd"), s.get("pre_rstd"), **more)
        return [t for t in answer if t is not None]
    if forward:
        return sequence.embedding_forward(s["weight"], s["ids"], scale=s["scale"], out_dtype=TYPES[s["to"]])
    return sequence.embedding_backward(s["grad"], s["ids"], s["rows"], scale=s["scale"], out_dtype=TYPES[s["to"]])


def work(case):
    a = SIZE[case["type"]]
    forward = case["direction"] == "forward"
    if case["op"] == "linear":
        t, n, m = case["tokens"], case["in"], case["out"]
        if forward:
            moved = a * (t * n + n * m + t * m * (1 + case["residual"] + case["keep"])) + 4 * m * case["bias"]
            return {"bytes": moved, "flops": 2 * t * n * m}
        return {"bytes": a * (2 * t * n + 2 * n * m + t * m * (1 + bool(case["activation"]))) + 4 * m,
                "flops": 4 * t * n * m}
    if case["op"] == "norm":
        b, n = SIZE[case["stream"]], case["rows"] * case["cols"]
        gate = {"none": 0, "values": n, "tokens": case["rows"]}[case["gate"]]
        norms = case["post"] + case["pre"]
        if forward:
            return {"bytes": n * (a * (1 + case["pre"]) + 2 * b) + a * gate + 4 * norms * (case["rows"] + case["cols"]),
                    "flops": 12 * n}
        # reads the stream's gradient, the block's output (where a norm or a gate needs it) and, with the second norm,
        # its gradient and the stream
        needed = case["post"] or case["gate"] != "none"
        return {"bytes": n * (a * (1 + needed + case["pre"]) + b * (2 + case["pre"])) + 2 * a * gate
                + 4 * norms * (case["rows"] + 2 * case["cols"]), "flops": 24 * n}
    tokens, rows, cols = case["tokens"], case["rows"], case["cols"]
    if forward:  # the rows that some id names are read once
        ends = torch.linspace(0, 1, rows + 1, dtype=torch.float64) ** (1 / case["skew"])
        touched = float((1 - torch.exp(-tokens * (1 - case["padding"]) * ends.diff())).sum())
        return {"bytes": int(8 * tokens + a * touched * cols + SIZE[case["to"]] * tokens * cols),
                "flops": tokens * cols}
    seen = int(tokens * (1 - case["padding"]))
    return {"bytes": 8 * tokens + a * seen * cols + SIZE[case["to"]] * rows * cols, "flops": (tokens + rows) * cols}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------


def _exact_linear(case, s):
    x, w, name = s["x"].double(), s["weight"].double(), case["activation"]
    root = 2 ** -0.5
    if case["direction"] == "forward":
        z = torch.addmm(s["bias_values"].double(), x, w) if case["bias"] else torch.mm(x, w)
        y = {None: lambda: z, "relu": lambda: z.clamp(min=0), "gelu": lambda: z * torch.special.erfc(-z * root) / 2,
             "silu": lambda: z * torch.sigmoid(z)}[name]()
        if case["residual"]:
            y = y + s["residual_rows"].double()
        return (y, z) if case["keep"] else y
    g = s["grad"].double()
    if name:
        z = s["z"].double()
        if name == "relu":
            g = torch.where(z > 0, g, 0.0)
        elif name == "gelu":
            g = g * (torch.special.erfc(-z * root) / 2 + z * torch.exp(-z ** 2 / 2) / (2 * math.pi) ** 0.5)
        else:
            s_ = torch.sigmoid(z)
            g = g * (s_ + z * s_ * torch.sigmoid(-z))
    return torch.einsum("tm,nm->tn", g, w), torch.einsum("tn,tm->nm", x, g), torch.einsum("tm->m", g)


def _exact_norm(case, s):
    cols, scale = case["cols"], case["scale"]
    x = s["x"].double()
    open_ = torch.sigmoid(s["gate_values"].double()) if case["gate"] != "none" else torch.ones_like(x[:, :1])
    if case["direction"] == "forward":
        post = (torch.einsum("rc,rc->r", x, x) / cols + EPS) ** -0.5
        u = torch.einsum("rc,r,c->rc", x, post, s["post_weight"].double()) if case["post"] else x
        total = torch.addcmul(s["residual"].double(), u, open_.expand_as(u), value=scale)
        answer = [total]
        pre = (torch.einsum("rc,rc->r", total, total) / cols + EPS) ** -0.5
        if case["pre"]:
            answer.append(torch.einsum("rc,r,c->rc", total, pre, s["pre_weight"].double()))
        return answer + ([post] if case["post"] else []) + ([pre] if case["pre"] else [])

    def through(g, values, rstd):  # the norm's Jacobian, without the weight
        along = torch.einsum("rc,rc->r", g, values) * rstd ** 3 / cols
        return g * rstd[:, None] - values * along[:, None]

    d, sums = s["grad_total"].double(), []
    if case["pre"]:
        g, total, rstd = s["grad_y"].double(), s["total"].double(), s["pre_rstd"].double()
        sums.append(torch.einsum("rc,rc,r->c", g, total, rstd))
        d = d + through(g * s["pre_weight"].double(), total, rstd)
    du = d * open_ * scale
    dx, u = du, x
    if case["post"]:
        rstd, w = s["post_rstd"].double(), s["post_weight"].double()
        sums.insert(0, torch.einsum("rc,rc,r->c", du, x, rstd))
        dx = through(du * w, x, rstd)
        u = x * rstd[:, None] * w
    answer = [dx, d]
    if case["gate"] != "none":
        dgate = d * u * (open_ - open_ ** 2) * scale
        answer.append(dgate if case["gate"] == "values" else torch.einsum("rc->r", dgate)[:, None])
    return answer + sums


def _exact_embedding(case, s):
    ids, rows, cols = s["ids"], case["rows"], case["cols"]
    if case["direction"] == "forward":
        padded = torch.cat([s["weight"], s["weight"].new_zeros(1, cols)])
        return padded[torch.where(ids < 0, rows, ids)].double() * case["scale"]
    order = torch.argsort(ids, stable=True)
    sums = torch.cat([torch.zeros(1, cols, dtype=torch.float64, device="cuda"),
                      s["grad"][order].double().cumsum(0)])
    ends = torch.searchsorted(ids[order], torch.arange(-1, rows, device="cuda"), right=True)
    return sums[ends].diff(dim=0) * case["scale"]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        return _exact_linear(case, s)
    return _exact_norm(case, s) if case["op"] == "norm" else _exact_embedding(case, s)
