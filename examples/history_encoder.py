"""Training and serving a small sequence encoder over the shared-array embedding.

Every user has a history of item ids, of any length.  An item and its position
are two tables of one PSS embedding; the packed rows go through dropout and one
attention block (layer norm, fused projection, causal attention inside each
history, output projection dropped out onto the residual stream, layer norm),
and a linear head answers, at every item, whether it has occurred in the
history before -- which only attention can see.  All gradients are explicit
calls; the projections are plain torch products.  FeedForwardEncoder is the larger
model: positions in a dense table of their own, projections with their epilogues, and a
gated feed-forward block behind the attention, root-mean-square norms between them.

    python examples/history_encoder.py [steps [small|feed-forward]]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2207_10731_gb300 import binding, sequence  # noqa: E402


class HistoryEncoder:
    def __init__(self, items=1000, positions=512, d=64, heads=4, kv_heads=2, dim=16, M=1 << 17,
                 p=0.1, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*size, scale):
            return torch.randn(*size, generator=gen, device="cuda") * scale

        self.d, self.heads, self.kv_heads, self.dim, self.p, self.seed = d, heads, kv_heads, dim, p, seed
        self.embedding = binding.PSS([items, positions], dim=d, M=M, Z=16, G=4, seed=seed,
                                     optimizer="adagrad")
        self.embedding.set_weights(normal(M, scale=0.5))
        width = (heads + 2 * kv_heads) * dim
        self.w = {"norm": torch.ones(d, device="cuda"), "norm_bias": torch.zeros(d, device="cuda"),
                  "qkv": normal(d, width, scale=d ** -0.5),
                  "out": normal(heads * dim, d, scale=(heads * dim) ** -0.5),
                  "last": torch.ones(d, device="cuda"), "last_bias": torch.zeros(d, device="cuda"),
                  "head": normal(d, scale=d ** -0.5)}
        self.moments = {k: (torch.zeros_like(v), torch.zeros_like(v)) for k, v in self.w.items()}
        self.steps = 0

    def _split(self, rows):
        rows = rows.view(-1, self.heads + 2 * self.kv_heads, self.dim)
        return rows.split([self.heads, self.kv_heads, self.kv_heads], dim=1)

    def embed(self, ids, offsets):
        """Sum of the item's and the position's rows, [tokens, d] fp32."""
        tokens = ids.numel()
        lengths = offsets.diff()
        positions = torch.arange(tokens, device="cuda") - offsets[:-1].repeat_interleave(lengths)
        bags = torch.arange(2 * tokens + 1, device="cuda")
        return self.embedding.forward(torch.cat([ids, positions]), bags, tokens).sum(1)

    def forward(self, ids, offsets, train):
        """Logits per token, and what the backward pass needs."""
        p = self.p if train else 0.0
        salt = 2 * self.steps
        h = sequence.dropout(self.embed(ids, offsets), p, self.seed, salt)
        y, mean, rstd = sequence.layer_norm_forward(h, self.w["norm"], self.w["norm_bias"],
                                                    out_dtype=torch.bfloat16)
        qkv = y @ self.w["qkv"].bfloat16()
        q, k, v = self._split(qkv)
        out, lse = sequence.attention_forward(q, k, v, offsets)
        o = out.reshape(-1, self.heads * self.dim) @ self.w["out"].bfloat16()
        h2 = sequence.dropout(o.float(), p, self.seed, salt + 1, residual=h)
        z, mean2, rstd2 = sequence.layer_norm_forward(h2, self.w["last"], self.w["last_bias"])
        return z @ self.w["head"], (h, y, mean, rstd, qkv, out, lse, h2, z, mean2, rstd2)

    def step(self, ids, offsets, labels, lr=0.01):
        """One training step; the mean logistic loss, on the device."""
        logits, (h, y, mean, rstd, qkv, out, lse, h2, z, mean2, rstd2) = \
            self.forward(ids, offsets, True)
        salt, n = 2 * self.steps, ids.numel()
        loss = torch.nn.functional.binary_cross_entropy_with_logits(logits, labels)
        g = {}
        d_logits = (torch.sigmoid(logits) - labels) / n
        g["head"] = d_logits @ z
        d_h2, g["last"], g["last_bias"] = sequence.layer_norm_backward(
            d_logits[:, None] * self.w["head"], h2, self.w["last"], mean2, rstd2)
        d_o = sequence.dropout(d_h2, self.p, self.seed, salt + 1).bfloat16()
        flat = out.reshape(n, -1)
        g["out"] = (flat.t() @ d_o).float()
        d_out = (d_o @ self.w["out"].bfloat16().t()).view_as(out)
        d_qkv = torch.empty_like(qkv)
        sequence.attention_backward(d_out, *self._split(qkv), out, lse, offsets,
                                    grads=self._split(d_qkv))
        g["qkv"] = (y.t() @ d_qkv).float()
        d_h, g["norm"], g["norm_bias"] = sequence.layer_norm_backward(
            d_qkv @ self.w["qkv"].bfloat16().t(), h, self.w["norm"], mean, rstd)
        d_x = sequence.dropout(d_h + d_h2, self.p, self.seed, salt)
        self.embedding.backward_update(d_x[:, None].expand(-1, 2, -1).contiguous(), lr)
        self.update(g, lr)
        return loss

    def update(self, g, lr):
        self.steps += 1
        for name, grad in g.items():   # Adam
            m, s = self.moments[name]
            m.mul_(0.9).add_(grad, alpha=0.1)
            s.mul_(0.99).addcmul_(grad, grad, value=0.01)
            size = (s / (1 - 0.99 ** self.steps)).sqrt_().add_(1e-8)
            self.w[name].addcdiv_(m / (1 - 0.9 ** self.steps), size, value=-lr)

    def serve(self, ids, offsets):
        """Logits of each history's newest item: one query per user over the
        keys and values of the whole history.  NaN for an empty history, which
        has no newest item."""
        some = offsets.diff() > 0
        if ids.numel() == 0:
            return torch.full(some.shape, float("nan"), device="cuda")
        h = self.embed(ids, offsets)
        y, _, _ = sequence.layer_norm_forward(h, self.w["norm"], self.w["norm_bias"],
                                              out_dtype=torch.bfloat16)
        newest = (offsets[1:] - 1).clamp_(min=0)   # an empty history's is another's: not used
        q, k, v = self._split(y @ self.w["qkv"].bfloat16())
        steps = torch.arange(newest.numel() + 1, device="cuda")
        out, _ = sequence.attention_forward(q[newest], k, v, steps, offsets)
        o = out.reshape(newest.numel(), -1) @ self.w["out"].bfloat16()
        h2 = o.float() + h[newest]
        z, _, _ = sequence.layer_norm_forward(h2, self.w["last"], self.w["last_bias"])
        return torch.where(some, z @ self.w["head"], float("nan"))


class FeedForwardEncoder(HistoryEncoder):
    def __init__(self, items=1000, positions=512, hidden=128, seed=0, **sizes):
        super().__init__(items=items, positions=positions, seed=seed, **sizes)
        d, gen = self.d, torch.Generator(device="cuda").manual_seed(seed + 1)

        def normal(*size, scale):
            return torch.randn(*size, generator=gen, device="cuda") * scale
        M = self.embedding.M
        self.embedding = binding.PSS([items], dim=d, M=M, Z=16, G=4, seed=seed, optimizer="adagrad")
        self.embedding.set_weights(normal(M, scale=0.5))
        self.positions, self.scale = positions, d ** 0.5
        for name in ("last", "last_bias"):
            del self.w[name]
        ones = {name: torch.ones(d, device="cuda") for name in ("post", "pre", "last_post", "last_pre")}
        self.w.update(ones, table=normal(positions, d, scale=0.5 / self.scale),
                      up=normal(d, hidden, scale=d ** -0.5), up_bias=torch.zeros(hidden, device="cuda"),
                      down=normal(hidden, d, scale=hidden ** -0.5),
                      down_bias=torch.zeros(d, device="cuda"), gate=normal(d, 1, scale=d ** -0.5))
        self.moments = {k: (torch.zeros_like(v), torch.zeros_like(v)) for k, v in self.w.items()}

    def places(self, offsets, tokens):
        return torch.arange(tokens, device="cuda") - offsets[:-1].repeat_interleave(offsets.diff())

    def embed(self, ids, offsets):
        """Sum of the item's row and the position's, scaled, [tokens, d] fp32."""
        tokens = ids.numel()
        rows = self.embedding.forward(ids, torch.arange(tokens + 1, device="cuda"), tokens)
        return rows.view(tokens, self.d) + sequence.embedding_forward(
            self.w["table"], self.places(offsets, tokens), scale=self.scale)

    def block(self, o, h):
        """Logits for the attention's projected output and the stream, and what the
        backward pass needs."""
        w = {k: v.bfloat16() for k, v in self.w.items() if k in ("up", "down", "gate")}
        total, n, a, b = sequence.residual_norm_forward(o, h, self.w["post"], self.w["pre"])
        u, z = sequence.linear_forward(n, w["up"], self.w["up_bias"], "gelu", keep=True)
        f = sequence.linear_forward(u, w["down"], self.w["down_bias"])
        gate = sequence.linear_forward(n, w["gate"])
        total2, last, c, e = sequence.residual_norm_forward(f, total, self.w["last_post"],
                                                            self.w["last_pre"], gate, scale=0.5)
        return last.float() @ self.w["head"], (w, total, n, a, b, u, z, f, gate, total2, last, c, e)

    def forward(self, ids, offsets, train):
        h = sequence.dropout(self.embed(ids, offsets), self.p if train else 0.0, self.seed, self.steps)
        y, mean, rstd = sequence.layer_norm_forward(h, self.w["norm"], self.w["norm_bias"],
                                                    out_dtype=torch.bfloat16)
        qkv = sequence.linear_forward(y, self.w["qkv"].bfloat16())
        out, lse = sequence.attention_forward(*self._split(qkv), offsets)
        o = sequence.linear_forward(out.view(ids.numel(), -1), self.w["out"].bfloat16())
        logits, kept = self.block(o, h)
        return logits, (h, y, mean, rstd, qkv, out, lse, o, kept)

    def gradients(self, ids, offsets, labels, lr=0.0):
        """(loss, the weights' gradients) of one training batch; the embedding takes its step."""
        logits, (h, y, mean, rstd, qkv, out, lse, o, kept) = self.forward(ids, offsets, True)
        w, total, n, a, b, u, z, f, gate, total2, last, c, e = kept
        loss = torch.nn.functional.binary_cross_entropy_with_logits(logits, labels)
        tokens, kind, g = ids.numel(), torch.float32, {}
        d_logits = (torch.sigmoid(logits) - labels) / tokens
        g["head"] = d_logits @ last.float()
        d_last = (d_logits[:, None] * self.w["head"]).bfloat16()
        d_f, d_total, d_gate, g["last_post"], g["last_pre"] = sequence.residual_norm_backward(
            None, d_last, f, total2, c, e, self.w["last_post"], self.w["last_pre"], gate, scale=0.5)
        d_u, g["down"], g["down_bias"] = sequence.linear_backward(d_f, u, w["down"], dweight_dtype=kind)
        d_n, g["up"], g["up_bias"] = sequence.linear_backward(d_u, n, w["up"], z, "gelu",
                                                              dweight_dtype=kind)
        more, g["gate"], _ = sequence.linear_backward(d_gate, n, w["gate"], dbias=False,
                                                      dweight_dtype=kind)
        d_o, d_h, _, g["post"], g["pre"] = sequence.residual_norm_backward(
            d_total, d_n + more, o, total, a, b, self.w["post"], self.w["pre"])
        d_out, g["out"], _ = sequence.linear_backward(d_o, out.view(tokens, -1),
                                                      self.w["out"].bfloat16(), dbias=False,
                                                      dweight_dtype=kind)
        d_qkv = torch.empty_like(qkv)
        sequence.attention_backward(d_out.view_as(out), *self._split(qkv), out, lse, offsets,
                                    grads=self._split(d_qkv))
        d_y, g["qkv"], _ = sequence.linear_backward(d_qkv, y, self.w["qkv"].bfloat16(), dbias=False,
                                                    dweight_dtype=kind)
        d_x, g["norm"], g["norm_bias"] = sequence.layer_norm_backward(d_y, h, self.w["norm"], mean, rstd)
        d_x = sequence.dropout(d_x + d_h, self.p, self.seed, self.steps)
        g["table"] = sequence.embedding_backward(d_x, self.places(offsets, tokens), self.positions,
                                                 scale=self.scale)
        self.embedding.backward_update(d_x, lr)
        return loss, g

    def step(self, ids, offsets, labels, lr=0.01):
        loss, g = self.gradients(ids, offsets, labels, lr)
        self.update(g, lr)
        return loss

    def serve(self, ids, offsets):
        some = offsets.diff() > 0
        if ids.numel() == 0:
            return torch.full(some.shape, float("nan"), device="cuda")
        h = self.embed(ids, offsets)
        y, _, _ = sequence.layer_norm_forward(h, self.w["norm"], self.w["norm_bias"],
                                              out_dtype=torch.bfloat16)
        newest = (offsets[1:] - 1).clamp_(min=0)
        q, k, v = self._split(sequence.linear_forward(y, self.w["qkv"].bfloat16()))
        steps = torch.arange(newest.numel() + 1, device="cuda")
        out, _ = sequence.attention_forward(q[newest], k, v, steps, offsets)
        o = sequence.linear_forward(out.view(newest.numel(), -1), self.w["out"].bfloat16())
        return torch.where(some, self.block(o, h[newest])[0], float("nan"))


def histories(seed, users=256, items=1000, longest=64):
    """(ids, offsets, labels): random histories in which items come back."""
    gen = torch.Generator().manual_seed(seed)
    lengths = torch.randint(1, longest + 1, (users,), generator=gen)
    ids, labels = [], []
    for n in lengths.tolist():
        row, seen = [], set()
        for _ in range(n):
            again = row and torch.rand((), generator=gen) < 0.5
            pick = row[int(torch.randint(len(row), (), generator=gen))] if again else \
                int(torch.randint(items, (), generator=gen))
            labels.append(float(pick in seen))
            seen.add(pick)
            row.append(pick)
        ids += row
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), lengths.cumsum(0)])
    return torch.tensor(ids).cuda(), offsets.cuda(), torch.tensor(labels).cuda()


def main(steps=300, kind="small"):
    model = HistoryEncoder() if kind == "small" else FeedForwardEncoder()
    batches = [histories(s) for s in range(8)]
    for i in range(steps):
        loss = model.step(*batches[i % len(batches)])
        if i % 50 == 0 or i == steps - 1:
            print(f"step {i}: loss {loss.item():.4f}")
    ids, offsets, labels = histories(1000)
    logits, _ = model.forward(ids, offsets, False)
    right = ((logits > 0) == (labels > 0.5)).float().mean().item()
    served = model.serve(ids, offsets)
    print(f"unseen histories: {100 * right:.1f} % of the items answered right; "
          f"served newest items differ by at most "
          f"{(served - logits[offsets[1:] - 1]).abs().max().item():.3g}")


if __name__ == "__main__":
    main(*(int(a) for a in sys.argv[1:2]), *sys.argv[2:3])
