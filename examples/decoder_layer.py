"""A decoder layer, attention and experts, trained on packed sequences and then served token by token from a cache of pages.

    python examples/decoder_layer.py

norm -> q, k, v -> attention with a window and first tokens that stay visible -> experts (examples/moe_layer.py), forward and
backward on the library's operators; the projections and the optimiser are PyTorch's.  Served, the prompts go through the same
attention, their keys and values into pages that are planned on the GPU, and each new token attends over its pages.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from moe_layer import AddNorm, MoELayer, moe  # noqa: E402


class Attend(torch.autograd.Function):
    """Attention within each sequence; q, k and v are parts of x [rows, heads + 2 kv_heads, dim]."""

    @staticmethod
    def forward(ctx, x, offsets, kv_heads, window, sinks):
        q, k, v = split(x, kv_heads)
        y, kept = moe.attend_rows(q, k, v, offsets, window=window, sinks=sinks, keep=True)
        ctx.save_for_backward(x, offsets, y, *kept)
        ctx.sees = dict(window=window, sinks=sinks)
        ctx.kv_heads = kv_heads
        return y

    @staticmethod
    def backward(ctx, dy):
        x, offsets, y, *kept = ctx.saved_tensors
        d = moe.attend_rows_backward(*split(x, ctx.kv_heads), offsets, y, moe.KeptAttention(*kept), dy.contiguous(), **ctx.sees)
        return torch.cat(d, 1), None, None, None, None


def split(x, kv_heads):
    heads = x.shape[1] - 2 * kv_heads
    return x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]


class DecoderLayer(torch.nn.Module):
    def __init__(self, hidden, heads, kv_heads, dim, inter, experts, top_k, window=0, sinks=0, device="cuda"):
        super().__init__()
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        self.sees = dict(window=window, sinks=sinks)
        self.gain = torch.nn.Parameter(torch.ones(hidden, device=device))
        self.to_qkv = torch.nn.Parameter((torch.randn((heads + 2 * kv_heads) * dim, hidden, device=device) * hidden ** -0.5).bfloat16())
        self.to_out = torch.nn.Parameter((torch.randn(hidden, heads * dim, device=device) * (heads * dim) ** -0.5).bfloat16())
        self.experts = MoELayer(hidden, inter, experts, top_k, device)

    def qkv(self, x):
        return (x @ self.to_qkv.t()).view(-1, self.heads + 2 * self.kv_heads, self.dim)

    def out(self, h, y):
        """(h + the attention's output, the experts' output on it): the next layer adds them"""
        return self.experts(h, y.reshape(-1, self.heads * self.dim) @ self.to_out.t())

    def forward(self, h, offsets):
        h, x = AddNorm.apply(h, None, self.gain)
        return self.out(h, Attend.apply(self.qkv(x), offsets, self.kv_heads, *self.sees.values()))


class Served:
    """The layer with a cache of pages for `requests` sequences; cache: torch.bfloat16 or torch.int8."""

    @torch.no_grad()
    def __init__(self, layer, requests, longest, page=16, cache=torch.bfloat16):
        self.layer, self.page = layer, page
        device, per = layer.gain.device, -(-longest // page)
        n = requests * per
        shape = (n, layer.kv_heads, page, layer.dim)
        self.pages = [torch.zeros(shape, dtype=cache, device=device) for _ in range(2)]
        self.scales = [torch.zeros(shape[:3], device=device) if cache == torch.int8 else None for _ in range(2)]
        self.table = torch.full((requests, per), -1, dtype=torch.int32, device=device)
        self.free = torch.arange(n, dtype=torch.int32, device=device)
        self.lengths = torch.zeros(requests, dtype=torch.int32, device=device)
        self.used = torch.zeros(1, dtype=torch.int32, device=device)

    def take(self, h, more):
        """(h, its q, the plan): `more` new tokens of each request, rows of h, are in the cache"""
        n = moe.norm_rows(h, None, self.layer.gain)
        q, k, v = split(self.layer.qkv(n.x), self.layer.kv_heads)
        plan = moe.plan_pages(self.lengths, more, self.table, self.free, self.page, h.shape[0], used=self.used)
        moe.store_pages(k, v, plan.slots, *self.pages, *self.scales)
        self.lengths, self.used = plan.lengths, plan.used
        return q, k, v, plan

    @torch.no_grad()
    def prompts(self, h, more):
        """The requests' first tokens, `more` of each (int32), row after row."""
        q, k, v, plan = self.take(h, more)
        return self.layer.out(h, moe.attend_rows(q, k, v, plan.offsets, **self.layer.sees))

    @torch.no_grad()
    def token(self, h):
        """One more token of each request."""
        q, _, _, _ = self.take(h, torch.ones_like(self.lengths))
        return self.layer.out(h, moe.attend_pages(q, *self.pages, self.table, self.lengths, *self.scales, **self.layer.sees))


def main(hidden=1024, heads=8, kv_heads=2, dim=64, inter=256, experts=8, top_k=2, tokens=1500, steps=30, window=256, sinks=4):
    torch.manual_seed(0)
    teacher, layer = (DecoderLayer(hidden, heads, kv_heads, dim, inter, experts, top_k, window, sinks) for _ in range(2))
    h = torch.randn(tokens, hidden, device="cuda")
    offsets = torch.tensor([0, tokens // 3, tokens], dtype=torch.int32, device="cuda")
    with torch.no_grad():
        layer.experts.load_state_dict(teacher.experts.state_dict())
        target = sum(t.float() for t in teacher(h, offsets))
    trained = [layer.gain, layer.to_qkv, layer.to_out]
    wide = [p.detach().float() for p in trained]  # (the optimiser's steps are smaller than the roundings of bf16)
    adam, losses = torch.optim.Adam(wide, lr=2e-3), []
    for _ in range(steps):
        loss = (sum(t.float() for t in layer(h, offsets)) - target).square().mean()
        for w, p, g in zip(wide, trained, torch.autograd.grad(loss, trained)):
            w.grad = g.float()
        adam.step()
        with torch.no_grad():
            for w, p in zip(wide, trained):
                p.copy_(w)
        losses.append(float(loss.detach()))
    print(f"{tokens} tokens in two sequences, {heads} heads of {dim}: loss {losses[0]:.4f} -> {losses[-1]:.4f} in {steps} steps")
    with torch.no_grad():
        want = sum(t.float() for t in layer(h, offsets))
    for cache in (torch.bfloat16, torch.int8):
        served = Served(layer, 2, tokens, cache=cache)
        lens = offsets[1:] - offsets[:-1]
        a, b = (offsets[1:] - 20).tolist()  # the last 20 tokens of each come one by one
        served.prompts(torch.cat((h[:a], h[tokens // 3:b])), lens - 20)
        got = torch.stack([sum(t.float() for t in served.token(h[[a + t, b + t]])) for t in range(20)])
        ref = torch.stack([want[[a + t, b + t]] for t in range(20)])
        print(f"served from {cache}: tokens differ by {(got - ref).norm() / ref.norm():.4f} of their size")
    return losses


if __name__ == "__main__":
    main()
