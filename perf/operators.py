"""The operators of a sequence encoder over the pooled embeddings, case by case: layer norm, dropout and
attention over packed sequences (``paper_2207_10731_gb300.sequence``), each with its plain form in elementary
torch operations and its definition in 64 bits.

A user of the shared-array embedding holds rows of ``d`` values, one per id of a history: they are dropped out,
normalised and attended to inside each history.  Sizes are the embedding's own (rows of 16, 64 or 128 values, 26
tables, batches of 16384 and 65536) or generic ones.
"""
import functools
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5


def listed():
    return [
        # one serving batch of pooled rows, normalised for the next product: latency counts
        {"name": "norm forward serving rows", "op": "norm", "direction": "forward", "rows": 26, "cols": 128,
         "type": "f32", "to": "bf16"},
        # every pooled row of a Criteo-TB-shaped training batch, normalised as it leaves the embedding
        {"name": "norm forward pooled batch", "op": "norm", "direction": "forward", "rows": 65536 * 26, "cols": 128,
         "type": "f32", "to": "bf16"},
        # the concatenated row of all 26 tables, gradient into the embedding and into the norm's weights
        {"name": "norm backward concatenated", "op": "norm", "direction": "backward", "rows": 16384,
         "cols": 26 * 128, "type": "f32", "to": "f32"},
        # an odd width, 16-bit activations inside the encoder, gradient with the weights' reduction
        {"name": "norm backward odd width", "op": "norm", "direction": "backward", "rows": 40001, "cols": 333,
         "type": "bf16", "to": "bf16"},
        # dropout of one small batch's rows, odd in both sizes and cut out of a wider buffer
        {"name": "dropout small cut-out", "op": "dropout", "rows": 127, "cols": 129, "type": "f16", "p": 0.5,
         "residual": False, "gap": 31},
        # dropout of the pooled rows of a training batch in the embedding's own type
        {"name": "dropout pooled batch", "op": "dropout", "rows": 65536 * 26, "cols": 128, "type": "f32", "p": 0.1,
         "residual": False, "gap": 0},
        # a sublayer's output dropped out and added onto the residual stream
        {"name": "dropout onto residual", "op": "dropout", "rows": 262144, "cols": 512, "type": "bf16", "p": 0.2,
         "residual": True, "gap": 0},
        # serving: the newest item of one user against a short history
        {"name": "attention step one user", "op": "attention", "direction": "forward", "sequences": 1, "shortest": 200,
         "longest": 200, "queries": 1, "heads": 4, "kv_heads": 4, "dim": 64, "causal": True, "fused": False},
        # serving: the newest item of each user against long histories, shared key heads
        {"name": "attention step long", "op": "attention", "direction": "forward", "sequences": 48, "shortest": 512,
         "longest": 16384, "queries": 1, "heads": 16, "kv_heads": 4, "dim": 128, "causal": True, "fused": False},
        # training on packed histories of very different lengths, some of them empty
        {"name": "attention train histories", "op": "attention", "direction": "train", "sequences": 1024,
         "shortest": 0, "longest": 401, "queries": 0, "heads": 4, "kv_heads": 4, "dim": 64, "causal": True,
         "fused": True},
        # prefill of long sequences
        {"name": "attention forward long", "op": "attention", "direction": "forward", "sequences": 3,
         "shortest": 4096, "longest": 8192, "queries": 0, "heads": 16, "kv_heads": 4, "dim": 128, "causal": True,
         "fused": True},
        # training on long sequences, shared key heads: the largest
        {"name": "attention train long", "op": "attention", "direction": "train", "sequences": 4, "shortest": 2000,
         "longest": 7777, "queries": 0, "heads": 16, "kv_heads": 4, "dim": 128, "causal": True, "fused": True},
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "dropout", "attention", "attention", "attention"])
    if op == "norm":
        cols = rng.choice([16, 64, 128, 512, 26 * 128, _between(rng, 12, 8192)])
        return {"op": op, "direction": rng.choice(["forward", "backward"]),
                "rows": _between(rng, 1, max(2, min(65536 * 26, 2**27 // cols))), "cols": cols,
                "type": rng.choice(["f32", "bf16", "f16"]), "to": rng.choice(["f32", "bf16", "f16"])}
    if op == "dropout":
        cols = rng.choice([16, 64, 128, 512, _between(rng, 1, 8192)])
        return {"op": op, "rows": _between(rng, 1, max(2, min(65536 * 26, 2**27 // cols))), "cols": cols,
                "type": rng.choice(["f32", "bf16", "f16"]), "p": rng.choice([0.05, 0.1, 0.3, 0.5]),
                "residual": rng.random() < 0.5, "gap": rng.choice([0, 0, 8, 13])}
    kv_heads = rng.choice([1, 2, 4])
    case = {"op": op, "direction": rng.choice(["forward", "train"]), "queries": rng.choice([0, 0, 0, 1, 7]),
            "kv_heads": kv_heads, "heads": kv_heads * rng.choice([1, 2, 3, 4]), "dim": rng.choice([16, 64, 96, 128]),
            "causal": rng.random() < 0.75}
    longest = _between(rng, 16, 4096)
    case["fused"] = case["queries"] == 0 and rng.random() < 0.5
    return dict(case, longest=longest, shortest=rng.randint(0, longest),
                sequences=_between(rng, 1, max(2, min(1024, 2**31 // (4096 * longest * case["heads"])))))


def _lengths(case):
    """Lengths spread over the logarithm between the shortest and the longest; every 16th history is empty where the
    shortest is 0."""
    n, lo, hi = case["sequences"], case["shortest"], case["longest"]
    if hi == 0:
        return [0] * n
    got = []
    for i in range(n):
        if lo == 0 and i % 16 == 15:
            got.append(0)
            continue
        f = math.fmod(0.6180339887498949 * i, 1.0)
        got.append(int(round(hi * (max(lo, 1) / hi) ** f)))
    return got


def _query_lengths(case):
    return [case["queries"] or n for n in _lengths(case)]


def _pairs(case):
    """How many (query, key) pairs are not masked."""
    total = 0
    for n, q in zip(_lengths(case), _query_lengths(case)):
        if not case["causal"]:
            total += n * q
        else:  # query i sees the keys up to i + n - q: the queries stand at the end
            m = min(n, q)
            total += m * (n - m) + m * (m + 1) // 2
    return total


def _normal(gen, *size, dtype=torch.float32, scale=1.0):
    return (torch.randn(*size, generator=gen, device="cuda", dtype=torch.float32) * scale).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    state = dict(case)
    if case["op"] == "norm":
        rows, cols, kind = case["rows"], case["cols"], TYPES[case["type"]]
        x = _normal(gen, rows, cols) * (0.5 + torch.rand(rows, 1, generator=gen, device="cuda"))
        state["x"] = x.add_(_normal(gen, rows, 1, scale=0.5)).to(kind)
        state["weight"] = 1 + _normal(gen, cols, scale=0.2)
        state["bias"] = _normal(gen, cols, scale=0.2)
        if case["direction"] == "backward":  # with what the forward pass kept
            state["grad"] = _normal(gen, rows, cols, dtype=TYPES[case["to"]])
            x = state["x"].float()
            state["mean"] = x.mean(1)
            state["rstd"] = ((x - state["mean"][:, None]).square().mean(1) + EPS).rsqrt()
        return state
    if case["op"] == "dropout":
        rows, cols, kind = case["rows"], case["cols"], TYPES[case["type"]]
        state["x"] = _normal(gen, rows, cols + case["gap"], dtype=kind)[:, :cols]
        if case["residual"]:
            state["residual_rows"] = _normal(gen, rows, cols + case["gap"], dtype=kind)[:, :cols]
        state["seed"] = 0x9E3779B97F4A7C15 ^ seed
        state["offset"] = 2**33 + seed
        return state
    keys, queries = _lengths(case), _query_lengths(case)
    order = torch.randperm(len(keys), generator=gen, device="cuda").tolist()
    keys, queries = [keys[i] for i in order], [queries[i] for i in order]
    state["k_offsets"] = torch.tensor([0] + keys, dtype=torch.int64).cumsum(0).cuda()
    state["q_offsets"] = torch.tensor([0] + queries, dtype=torch.int64).cumsum(0).cuda()
    state["most_keys"], state["most_queries"] = max(keys), max(queries)
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    kind = torch.bfloat16
    if case["fused"]:  # views of one projection's output
        rows = _normal(gen, sum(keys), heads + 2 * kv_heads, dim, dtype=kind)
        state["q"], state["k"], state["v"] = rows.split([heads, kv_heads, kv_heads], dim=1)
    else:
        state["q"] = _normal(gen, sum(queries), heads, dim, dtype=kind)
        state["k"] = _normal(gen, sum(keys), kv_heads, dim, dtype=kind)
        state["v"] = _normal(gen, sum(keys), kv_heads, dim, dtype=kind)
    if case["direction"] == "train":
        state["grad"] = _normal(gen, sum(queries), heads, dim, dtype=kind)
    return state


# ---- plain forms ---------------------------------------------------------------------------------------------------


def _norm_forward(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    x = x - mean
    rstd = 1 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    y = x * rstd * s["weight"] + s["bias"]
    return y.to(TYPES[s["to"]]), mean[:, 0], rstd[:, 0]


def _norm_backward(s):
    g, rstd = s["grad"].float(), s["rstd"][:, None]
    hat = (s["x"].float() - s["mean"][:, None]) * rstd
    h = g * s["weight"]
    dx = (h - h.mean(1, keepdim=True) - hat * (h * hat).mean(1, keepdim=True)) * rstd
    return dx.to(s["x"].dtype), (g * hat).sum(0), g.sum(0)


def _round(c, step):
    """One round of the counter-based generator Philox 4x32 (Salmon, Moraes, Dror and Shaw 2011) on 32-bit words
    held in 64 bits."""
    low = 0xFFFFFFFF
    a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
    return ((b >> 32) & low) ^ c[1] ^ step[0], b & low, ((a >> 32) & low) ^ c[3] ^ step[1], a & low


def _kept(n, p, seed, offset):
    """The 0/1 mask of elements 0 .. n-1: element e takes 16 bits of the counter (e // 8, offset)."""
    low = 0xFFFFFFFF
    g = torch.arange((n + 7) // 8, device="cuda", dtype=torch.int64)
    zero = torch.zeros_like(g)
    steps = [((seed + i * 0x9E3779B9) & low, ((seed >> 32) + i * 0xBB67AE85) & low) for i in range(10)]
    words = functools.reduce(_round, steps, (g & low, g >> 32, zero + (offset & low), zero + (offset >> 32)))
    words = torch.stack(words, 1)
    bits = torch.stack((words & 0xFFFF, words >> 16), 2).view(-1)[:n]
    return bits >= round(p * 65536)


def _dropout(s):
    x = s["x"]
    keep = _kept(x.numel(), s["p"], s["seed"], s["offset"]).view(x.shape)
    y = torch.where(keep, x.float() * (65536 / (65536 - round(s["p"] * 65536))), 0.0)
    if s["residual"]:
        y = y + s["residual_rows"].float()
    return y.to(x.dtype)


def _padded(x, offsets, n):
    """Packed rows [tokens, heads, dim] as [sequences, heads, n, dim] in 32 bits, zero past each sequence's end."""
    at = offsets[:-1, None] + torch.arange(n, device="cuda")
    inside = at < offsets[1:, None]
    rows = x[at.clamp_(max=max(0, x.shape[0] - 1))].float() if x.shape[0] else x.new_zeros(*at.shape, *x.shape[1:]).float()
    return (rows * inside[:, :, None, None]).transpose(1, 2), inside


def _attention(s):
    heads, kv_heads, dim, n, m = s["heads"], s["kv_heads"], s["dim"], s["most_queries"], s["most_keys"]
    group, scale = heads // kv_heads, 1 / math.sqrt(dim)
    q, real = _padded(s["q"], s["q_offsets"], n)
    k, there = _padded(s["k"], s["k_offsets"], m)
    v, _ = _padded(s["v"], s["k_offsets"], m)
    q = q.reshape(-1, kv_heads, group * n, dim)
    seen = real[:, :, None] & there[:, None, :]
    if s["causal"]:
        ahead = (s["k_offsets"].diff() - s["q_offsets"].diff())[:, None, None]
        i, j = torch.arange(n, device="cuda")[:, None], torch.arange(m, device="cuda")
        seen = seen & (j <= i + ahead)
    hidden = ~seen[:, None, None].expand(-1, 1, group, n, m).reshape(-1, 1, group * n, m)
    scores = (q @ k.transpose(2, 3)).mul_(scale).masked_fill_(hidden, -math.inf)
    top = scores.amax(3, keepdim=True) if m else scores.new_full((*scores.shape[:3], 1), -math.inf)
    p = scores.sub_(top.clamp(min=torch.finfo(torch.float32).min)).exp_()
    total = p.sum(3, keepdim=True)
    lse = top + total.log()
    p = p.div_(total.clamp(min=1e-30))
    out = p @ v

    def packed(x, rows, inside):
        return x.reshape(x.shape[0], -1, rows, x.shape[-1]).transpose(1, 2)[inside]

    answer = [packed(out, n, real).to(s["q"].dtype), packed(lse, n, real)[..., 0]]
    if s["direction"] == "train":
        g = _padded(s["grad"], s["q_offsets"], n)[0].reshape(-1, kv_heads, group * n, dim)
        dv = p.transpose(2, 3) @ g
        ds = (g @ v.transpose(2, 3)).sub_((g * out).sum(3, keepdim=True)).mul_(p).mul_(scale)
        answer += [packed(ds @ k, n, real).to(s["q"].dtype), packed(ds.transpose(2, 3) @ q, m, there).to(s["k"].dtype),
                   packed(dv, m, there).to(s["v"].dtype)]
    return answer


# ---- one pass ------------------------------------------------------------------------------------------------------


def run(state):
    s = state
    if not own:
        if s["op"] == "norm":
            return _norm_forward(s) if s["direction"] == "forward" else _norm_backward(s)
        return _dropout(s) if s["op"] == "dropout" else _attention(s)
    from paper_2207_10731_gb300 import sequence

    if s["op"] == "norm":
        if s["direction"] == "forward":
            return sequence.layer_norm_forward(s["x"], s["weight"], s["bias"], eps=EPS, out_dtype=TYPES[s["to"]])
        return sequence.layer_norm_backward(s["grad"], s["x"], s["weight"], s["mean"], s["rstd"])
    if s["op"] == "dropout":
        return sequence.dropout(s["x"], s["p"], seed=s["seed"], offset=s["offset"], residual=s.get("residual_rows"))
    out, lse = sequence.attention_forward(s["q"], s["k"], s["v"], s["q_offsets"], s["k_offsets"], causal=s["causal"])
    if s["direction"] == "forward":
        return out, lse
    return (out, lse) + tuple(sequence.attention_backward(s["grad"], s["q"], s["k"], s["v"], out, lse, s["q_offsets"],
                                                          s["k_offsets"], causal=s["causal"]))


def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}
    if case["op"] == "norm":
        n, a, b = case["rows"] * case["cols"], size[case["type"]], size[case["to"]]
        if case["direction"] == "forward":
            return {"bytes": n * (a + b) + 8 * case["rows"] + 8 * case["cols"], "flops": 8 * n}
        return {"bytes": n * (2 * a + b) + 8 * case["rows"] + 12 * case["cols"], "flops": 14 * n}
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": n * size[case["type"]] * (3 if case["residual"] else 2), "flops": 2 * n}
    keys, queries = sum(_lengths(case)), sum(_query_lengths(case))
    row, kv_row = 2 * case["heads"] * case["dim"], 2 * case["kv_heads"] * case["dim"]
    moved = queries * (2 * row + 4 * case["heads"]) + 2 * keys * kv_row
    products = 2
    if case["direction"] == "train":  # reads the upstream gradient, writes three gradients; five products more
        moved += queries * 2 * row + 2 * keys * kv_row
        products = 7
    return {"bytes": moved, "flops": 2 * products * case["dim"] * case["heads"] * _pairs(case)}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------


def _mix64(n, p, seed, offset):
    """The mask again, with the 32 x 32 bit products put together from 16-bit parts."""
    low = 0xFFFFFFFF

    def product(x, m):
        mh, ml, xh, xl = m >> 16, m & 0xFFFF, x >> 16, x & 0xFFFF
        mid = xh * ml + ((xl * ml) >> 16)
        mid2 = xl * mh + (mid & 0xFFFF)
        return xh * mh + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | ((xl * ml) & 0xFFFF)

    g = torch.arange((n + 7) // 8, device="cuda", dtype=torch.int64)
    c0, c1, c2, c3 = g & low, g >> 32, torch.full_like(g, offset & low), torch.full_like(g, offset >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        h0, l0 = product(c0, 0xD2511F53)
        h1, l1 = product(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    bits = torch.empty(g.numel(), 8, dtype=torch.int64, device="cuda")
    for i, c in enumerate((c0, c1, c2, c3)):
        bits[:, 2 * i], bits[:, 2 * i + 1] = c % 65536, c // 65536
    return bits.view(-1)[:n] >= round(p * 65536)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        x, w = s["x"].double(), s["weight"].double()
        if case["direction"] == "forward":
            var, mean = torch.var_mean(x, 1, correction=0)
            rstd = (var + EPS) ** -0.5
            return (x - mean[:, None]) * rstd[:, None] * w + s["bias"].double(), mean, rstd
        g, rstd = s["grad"].double(), s["rstd"].double()
        hat = (x - s["mean"].double()[:, None]) * rstd[:, None]
        g_weight, g_bias = torch.einsum("rc,rc->c", g, hat), g.sum(0)
        g = g * w
        along = torch.einsum("rc,rc->r", g, hat) / case["cols"]
        return (g - g.mean(1)[:, None] - hat * along[:, None]) * rstd[:, None], g_weight, g_bias
    if case["op"] == "dropout":
        x = s["x"].double()
        y = x * _mix64(x.numel(), s["p"], s["seed"], s["offset"]).view(x.shape)
        y = y * (1 / (1 - round(s["p"] * 65536) / 65536))
        return y + s["residual_rows"].double() if case["residual"] else y
    group, scale = case["heads"] // case["kv_heads"], case["dim"] ** -0.5
    train = case["direction"] == "train"
    outs, lses, dq, dk, dv = [], [], [], [], []
    qo, ko = s["q_offsets"].tolist(), s["k_offsets"].tolist()
    for i in range(case["sequences"]):
        q = s["q"][qo[i]:qo[i + 1]].double().transpose(0, 1)
        k, v = (s[name][ko[i]:ko[i + 1]].double().transpose(0, 1).repeat_interleave(group, 0) for name in "kv")
        n, m = q.shape[1], k.shape[1]
        z = torch.einsum("hid,hjd->hij", q, k) * scale
        if case["causal"]:
            z = z + torch.full((n, m), -math.inf, dtype=torch.float64, device="cuda").triu(m - n + 1)
        lse = torch.logsumexp(z, 2)
        p = torch.where(torch.isinf(lse)[:, :, None], 0.0, torch.exp(z - lse[:, :, None]))
        out = torch.einsum("hij,hjd->hid", p, v)
        outs.append(out.transpose(0, 1))
        lses.append(lse.transpose(0, 1))
        if train:
            g = s["grad"][qo[i]:qo[i + 1]].double().transpose(0, 1)
            dz = torch.einsum("hid,hjd->hij", g, v)
            dz = p * (dz - (p * dz).sum(2, keepdim=True)) * scale
            dq.append(torch.einsum("hij,hjd->hid", dz, k).transpose(0, 1))
            sums = [torch.einsum("hij,hid->jhd", dz, q), torch.einsum("hij,hid->jhd", p, g)]
            for to, x in zip((dk, dv), sums):
                to.append(x.reshape(m, case["kv_heads"], group, case["dim"]).sum(2))
    answer = [torch.cat(outs), torch.cat(lses)]
    return answer + [torch.cat(x) for x in (dq, dk, dv)] if train else answer
