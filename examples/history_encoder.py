"""Training and serving a small sequence encoder over the shared-array embedding.

Every user has a history of item ids, of any length.  An item and its position
are two tables of one PSS embedding; the packed rows go through dropout and one
attention block (layer norm, fused projection, causal attention inside each
history, output projection dropped out onto the residual stream, layer norm),
and a linear head answers, at every item, whether it has occurred in the
history before -- which only attention can see.  All gradients are explicit
calls; the projections are plain torch products.

    python examples/history_encoder.py [steps]
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
        self.steps += 1
        for name, grad in g.items():   # Adam
            m, s = self.moments[name]
            m.mul_(0.9).add_(grad, alpha=0.1)
            s.mul_(0.99).addcmul_(grad, grad, value=0.01)
            size = (s / (1 - 0.99 ** self.steps)).sqrt_().add_(1e-8)
            self.w[name].addcdiv_(m / (1 - 0.9 ** self.steps), size, value=-lr)
        return loss

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


def main(steps=300):
    model = HistoryEncoder()
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
    main(*(int(a) for a in sys.argv[1:2]))
