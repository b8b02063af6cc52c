"""A behaviour-sequence encoder on the embedding step: training and serving.

Training, one step: ids -> Table.forward (padded copy) -> layer norm -> q, k, v projection -> attention over the ragged
sequences (causal, falling off with distance by learned slopes) -> output projection and residual -> mean over the
sequence -> logistic loss; then back through all of it, the gradient of the padded copy into Table.backward_optimizer.

Serving: the keys and values of a user's history are kept, and candidates are scored against them, a few queries over a
long history in one attention call.

    python examples/sequence_encoder.py [--steps 20] [--bags 512] [--pad 256] [--dim 64] [--heads 4]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2509_20883_amd import recis as R  # noqa: E402


class Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, op, mask):
        y, mean, rstd = op.forward(x, weight, bias, mask=mask)
        ctx.save_for_backward(x, weight, mean, rstd, mask)
        ctx.op = op
        return y

    @staticmethod
    def backward(ctx, grad):
        x, weight, mean, rstd, mask = ctx.saved_tensors
        return (*ctx.op.backward(grad, x, mean, rstd, weight, mask=mask), None, None)


class Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, slopes, op, offsets):
        out, stats = op.forward(q, k, v, offsets, slopes=slopes)
        ctx.save_for_backward(q, k, v, out, *stats, slopes, offsets)
        ctx.op = op
        return out

    @staticmethod
    def backward(ctx, grad):
        q, k, v, out, lse, rest, slopes, offsets = ctx.saved_tensors
        return (*ctx.op.backward(grad, q, k, v, out, R.AttnStats(lse, rest), offsets, slopes=slopes), None, None)


class Encoder:
    """Pre-norm attention block over padded sequences [bags, pad, dim] in bf16."""

    def __init__(self, dim, heads, kv_heads, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(rows, cols):
            w = torch.randn(rows, cols, generator=g, device="cuda") / rows ** 0.5
            return w.bfloat16().requires_grad_()

        self.heads, self.kv_heads, self.d = heads, kv_heads, dim // heads
        self.gain = torch.ones(dim, device="cuda", requires_grad=True)
        self.shift = torch.zeros(dim, device="cuda", requires_grad=True)
        self.qkv = weight(dim, (heads + 2 * kv_heads) * self.d)
        self.proj = weight(dim, dim)
        self.head = weight(dim, 1)
        self.slopes = torch.pow(2.0, -1.0 - 4.0 * torch.arange(heads, device="cuda") / heads).requires_grad_()
        self.norm, self.attend = R.LayerNorm(), R.SeqAttention(causal=True)
        self.parameters = [self.gain, self.shift, self.qkv, self.proj, self.head, self.slopes]

    def split(self, x):
        """q, k, v of rows [..., dim], as column blocks of one projection."""
        y = (x.reshape(-1, x.shape[-1]) @ self.qkv).view(*x.shape[:-1], self.heads + 2 * self.kv_heads, self.d)
        return y.split([self.heads, self.kv_heads, self.kv_heads], -2)

    def scores(self, rows, mask, offsets):
        x = Norm.apply(rows, self.gain, self.shift, self.norm, mask)
        out = Attention.apply(*self.split(x), self.slopes, self.attend, offsets)
        h = rows + (out.reshape(-1, rows.shape[-1]) @ self.proj).view_as(rows)
        live = mask[..., None].to(h.dtype)
        pooled = (h * live).float().sum(1) / mask.sum(1, keepdim=True).clamp(min=1)
        return (pooled.bfloat16() @ self.head).float().squeeze(1)


def train(steps=20, bags=512, pad=256, dim=64, heads=4, vocab=20000, lr=0.05, seed=0):
    """Learns which users' sequences hold more even than odd ids; returns the encoder, the table and the losses."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    table = R.Table(dim, R.BF16, R.ADAGRAD, seed=1, init_lo=-0.05, init_hi=0.05, capacity_slots=1 << 17)
    model = Encoder(dim, heads, max(1, heads // 2), seed)
    opt = torch.optim.Adam(model.parameters, lr=3e-3)
    lens = torch.randint(1, pad + 1, (bags,), generator=g, device="cuda")
    offsets = torch.zeros(bags + 1, dtype=torch.int64, device="cuda")
    torch.cumsum(lens, 0, out=offsets[1:])
    taste = torch.rand(bags, generator=g, device="cuda") < 0.5
    owner = torch.repeat_interleave(torch.arange(bags, device="cuda"), lens)
    losses = []
    for _ in range(steps):
        n = int(offsets[-1])
        even = torch.where(taste[owner], 0.8, 0.2) > torch.rand(n, generator=g, device="cuda")
        values = 2 * torch.randint(0, vocab // 2, (n,), generator=g, device="cuda") + (~even).long()
        rows, mask, ctx = table.forward(values, offsets, R.NONE, pad)
        rows.requires_grad_()
        loss = torch.nn.functional.binary_cross_entropy_with_logits(model.scores(rows, mask, offsets), taste.float())
        opt.zero_grad()
        loss.backward()
        opt.step()
        table.backward_optimizer(ctx, rows.grad.contiguous(), lr)
        losses.append(loss.detach())
    table.check()
    return model, table, [float(x) for x in losses]


@torch.no_grad()
def serve(model, table, history, candidates):
    """Scores of candidate ids against one user's history: its keys and values once, then every candidate as one query
    that sees the whole history (a candidate is not part of it, so nothing is causal)."""
    ids = torch.cat([history, candidates])
    rows, _, _ = table.forward(ids, torch.tensor([0, ids.numel()], device="cuda"), R.NONE, ids.numel())
    x = model.norm.forward(rows[0], model.gain, model.shift)[0]
    q, k, v = model.split(x)
    n = history.numel()
    look = R.SeqAttention(causal=False)
    out, _ = look.forward(q[n:], k[:n], v[:n], torch.tensor([0, candidates.numel()], device="cuda"),
                          kv_offsets=torch.tensor([0, n], device="cuda"), max_q=candidates.numel())
    h = rows[0, n:] + out.reshape(candidates.numel(), -1) @ model.proj
    return (h @ model.head).float().squeeze(1)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--bags", type=int, default=512)
    ap.add_argument("--pad", type=int, default=256)
    ap.add_argument("--dim", type=int, default=64)
    ap.add_argument("--heads", type=int, default=4)
    a = ap.parse_args()
    model, table, losses = train(a.steps, a.bags, a.pad, a.dim, a.heads)
    print("loss " + " ".join(f"{x:.3f}" for x in losses), flush=True)
    history = torch.arange(0, 20000, 2, device="cuda")
    scores = serve(model, table, history, torch.arange(8, device="cuda"))
    print("candidates " + " ".join(f"{x:+.3f}" for x in scores.tolist()), flush=True)
    table.close()


if __name__ == "__main__":
    main()
